// The plans that the host runtime makes of linear layers
// (paper_2411_17866_amd/csrc/block_runtime.cpp), one line for each problem named on the
// command line as tokens,dim,wide,dtype,act,dw_dtype; compiled with g++ against stubs of
// the launchers and of the HIP calls.
#include <cstdio>

#include "block_internal.h"

static dsm::LinearPlan seen;

namespace dsm {
dsm_status set_thread_error(dsm_status st, const char* message) {
    std::fprintf(stderr, "%s\n", message);
    return st;
}
hipError_t launch_linear(const LinearCall& c, hipStream_t) {
    seen = c.p;
    return hipSuccess;
}
hipError_t launch_linear_backward(const LinearCall&, hipStream_t) { return hipSuccess; }
hipError_t launch_norm(const NormCall&, hipStream_t) { return hipSuccess; }
hipError_t launch_norm_backward(const NormCall&, hipStream_t) { return hipSuccess; }
hipError_t launch_clip_squares(const ClipTable&, int64_t, double*, hipStream_t) { return hipSuccess; }
hipError_t launch_clip_norms(const ClipGroups&, const double*, float*, double*, hipStream_t) { return hipSuccess; }
hipError_t launch_clip_scale(const ClipTable&, const double*, hipStream_t) { return hipSuccess; }
hipError_t launch_clip_rest(const ClipTable&, const ClipFew&, const double*, float*, hipStream_t) { return hipSuccess; }
int norm_groups(int64_t, int64_t) { return 1; }
}  // namespace dsm

extern "C" hipError_t hipGetDeviceCount(int* n) {
    *n = 1;
    return hipSuccess;
}
extern "C" const char* hipGetErrorString(hipError_t) { return "stub"; }

int main(int argc, char** argv) {
    for (int i = 1; i < argc; ++i) {
        long long tokens, dim, wide;
        int dtype, act, dw;
        if (std::sscanf(argv[i], "%lld,%lld,%lld,%d,%d,%d", &tokens, &dim, &wide, &dtype, &act, &dw) != 6) return 1;
        const dsm_linear_problem p{tokens, dim, wide, dtype, act, dw, 1};
        dsm_linear_buffers b{};
        const auto at = [](int k) { return reinterpret_cast<void*>(static_cast<uintptr_t>(k) << 44); };
        b.x = at(1);
        b.w = at(2);
        b.y = at(3);
        b.workspace = at(4);
        b.x_stride = b.w_stride = dim;
        b.y_stride = wide;
        if (dsm_linear_workspace(&p, &b.workspace_bytes) != DSM_OK || dsm_linear(&p, &b) != DSM_OK) return 1;
        static const char* const forms[] = {"bf16", "halves", "single"};
        std::printf("form %s back_form %s few %d tile %d splits %d front %d back_tile %d dx_splits %d dw_splits %d "
                    "split_rows %d dz_halves %d back_few %d\n",
                    forms[seen.form], forms[seen.back_form], seen.few, seen.tile, seen.splits, seen.front, seen.back_tile,
                    seen.dx_splits, seen.dw_splits, seen.split_rows, seen.dz_halves, seen.back_few);
    }
    return 0;
}
