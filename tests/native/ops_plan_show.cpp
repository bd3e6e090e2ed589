// The plans that the operators' host runtime makes (paper_2411_17866_amd/csrc/ops_runtime.cpp),
// one line for each problem of the cross entropy named on the command line as
// tokens,dim,vocab,dtype,grads: form, tile, tile columns of 256 and of them those taken by
// tiles of 256, pieces, parts of dh, sampled tile columns; one for each batch of matrices
// named as ortho,count,rows,cols: whether it is iterated in LDS, the tiles of its
// symmetric products and of its update.  Compiled with g++ against stubs of the launchers
// and of the HIP calls.
#include <algorithm>
#include <cstdio>

#include "dsm.h"
#include "ops_internal.h"
#include "ortho_plan.h"

static dsm::CePlan seen;

namespace dsm {
dsm_status set_thread_error(dsm_status st, const char* message) {
    std::fprintf(stderr, "%s\n", message);
    return st;
}
hipError_t launch_linear_ce(const CePlan& plan, const CeBuffers&, hipStream_t) {
    seen = plan;
    return hipSuccess;
}
int64_t ortho_group_bytes(int, int, int, bool) { return 0; }
hipError_t launch_ortho(const OrthoGroup&, const float*, const OrthoScales*, int, hipStream_t) { return hipSuccess; }
}  // namespace dsm

extern "C" hipError_t hipGetDeviceCount(int* n) {
    *n = 1;
    return hipSuccess;
}
extern "C" const char* hipGetErrorString(hipError_t) { return "stub"; }

int main(int argc, char** argv) {
    for (int i = 1; i < argc; ++i) {
        long long tokens, dim, vocab;
        int dtype, grads, count, rows, cols;
        if (std::sscanf(argv[i], "ortho,%d,%d,%d", &count, &rows, &cols) == 3) {
            const int m = std::min(rows, cols), n = std::max(rows, cols);
            std::printf("%d %d %d\n", dsm::is_small(m, n), dsm::ortho_tile(count, m, n, true),
                        dsm::ortho_tile(count, m, n, false));
            continue;
        }
        if (std::sscanf(argv[i], "%lld,%lld,%lld,%d,%d", &tokens, &dim, &vocab, &dtype, &grads) != 5) return 1;
        const dsm_ce_problem p{tokens, dim, vocab, dtype, grads};
        dsm_ce_buffers b{};
        const auto at = [](int k) { return reinterpret_cast<void*>(static_cast<uintptr_t>(k) << 40); };
        b.h = at(1);
        b.w = at(2);
        b.target = static_cast<const int64_t*>(at(3));
        b.total = static_cast<float*>(at(4));
        b.loss = static_cast<float*>(at(5));
        b.dh = grads ? at(6) : nullptr;
        b.dw = grads ? at(7) : nullptr;
        b.workspace = at(8);
        b.h_stride = b.w_stride = b.dh_stride = b.dw_stride = dim;
        if (dsm_ce_workspace(&p, &b.workspace_bytes) != DSM_OK || dsm_linear_ce(&p, &b, 1) != DSM_OK) return 1;
        static const char* const forms[] = {"bf16", "half", "halves", "f32"};
        const long long pieces = seen.piece > 0 ? (vocab + seen.piece - 1) / seen.piece : 0;
        std::printf("%s %d %lld %d %lld %d %d\n", forms[seen.form], seen.tile, (vocab + 255) / 256, seen.front, pieces,
                    seen.dh_splits, seen.sample);
    }
    return 0;
}
