// Host checks of the operators' runtime (paper_2411_17866_amd/csrc/ops_runtime.cpp):
// compiled with g++ under sanitizers against stubs of the launchers and of the HIP
// calls, so that every plan, argument check and launch argument can be looked at
// without a GPU.  Prints "all checks passed".
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <random>
#include <string>
#include <vector>

#include "dsm.h"
#include "dsm_internal.h"
#include "ops_internal.h"

static long checks = 0;
#define CHECK(c)                                                                \
    do {                                                                        \
        ++checks;                                                               \
        if (!(c)) {                                                             \
            std::printf("FAILED %s:%d: %s\n", __FILE__, __LINE__, #c);          \
            std::exit(1);                                                       \
        }                                                                       \
    } while (0)

// ---- Stubs ----

static std::string last_message;
static int devices = 1;
static hipError_t launch_result = hipSuccess;
struct CeCall {
    dsm::CePlan plan;
    dsm::CeBuffers buf;
};
static std::vector<CeCall> ce_calls;
struct OrthoCall {
    dsm::OrthoGroup group;
    std::vector<float> coeffs;
    std::vector<dsm::OrthoScales> scales;
};
static std::vector<OrthoCall> ortho_calls;

namespace dsm {
dsm_status set_thread_error(dsm_status st, const char* message) {
    last_message = message;
    return st;
}
hipError_t launch_linear_ce(const CePlan& plan, const CeBuffers& buf, hipStream_t) {
    ce_calls.push_back({plan, buf});
    return launch_result;
}
// The kernels' own rule is not compiled here: any size that grows with the problem.
int64_t ortho_group_bytes(int count, int m, int n, bool bf16) {
    if (m <= 32 && n <= 64) return 0;
    return static_cast<int64_t>(count) * m * (n + m) * (bf16 ? 4 : 8);
}
hipError_t launch_ortho(const OrthoGroup& g, const float* coeffs, const OrthoScales* scales, int steps, hipStream_t) {
    ortho_calls.push_back({g, {coeffs, coeffs + 3 * steps}, {scales, scales + steps}});
    return launch_result;
}
}  // namespace dsm

extern "C" hipError_t hipGetDeviceCount(int* n) {
    *n = devices;
    return devices > 0 ? hipSuccess : hipErrorNoDevice;
}
extern "C" const char* hipGetErrorString(hipError_t) { return "stub"; }

static std::mt19937_64 rng(5);
static int64_t pick(int64_t lo, int64_t hi) { return lo + static_cast<int64_t>(rng() % static_cast<uint64_t>(hi - lo + 1)); }
static int64_t spread(int64_t hi) {
    const double u = std::uniform_real_distribution<double>(0, std::log(static_cast<double>(hi)))(rng);
    return std::min<int64_t>(hi, static_cast<int64_t>(std::lround(std::exp(u))));
}
static void* at(uint64_t v) { return reinterpret_cast<void*>(v); }

// ---- Cross entropy ----

static dsm_ce_buffers ce_buffers(const dsm_ce_problem& p, int64_t ws) {
    dsm_ce_buffers b{};
    b.h = at(uint64_t(1) << 40);
    b.w = at(uint64_t(2) << 40);
    b.target = static_cast<const int64_t*>(at(uint64_t(3) << 40));
    b.total = static_cast<float*>(at(uint64_t(4) << 40));
    b.loss = static_cast<float*>(at(uint64_t(5) << 40));
    b.dh = p.grads ? at(uint64_t(6) << 40) : nullptr;
    b.dw = p.grads ? at(uint64_t(7) << 40) : nullptr;
    b.workspace = at(uint64_t(8) << 40);
    b.workspace_bytes = ws;
    b.h_stride = b.w_stride = b.dh_stride = b.dw_stride = p.dim;
    return b;
}

static void check_plan(const dsm_ce_problem& p, const dsm::CePlan& q, int64_t ws) {
    const int64_t T = p.tokens, D = p.dim, V = p.vocab;
    CHECK(q.tokens == T && q.dim == D && q.vocab == V && q.bytes == ws && q.grads == p.grads);
    const bool f32 = q.form == dsm::kCeF32 || q.form == dsm::kCeHalves;
    CHECK(f32 == (p.dtype == DSM_F32));
    CHECK(q.tile == 32 || q.tile == 64 || q.tile == 128 || q.tile == 256);
    // The instantiations that the launcher has.
    if (q.form == dsm::kCeF32) CHECK(q.tile <= 64);
    if (q.form == dsm::kCeHalf) CHECK(q.tile >= 128 && p.grads);
    if (q.form == dsm::kCeHalves) CHECK(q.tile >= 128);
    if (q.form == dsm::kCeBf16 && p.grads) CHECK(q.tile <= 128);
    const int64_t units = f32 ? 2 : 1, square = q.tile == 256 ? 256 : 128;
    const int64_t wide = (D + 63) / 64 * 64 * units, high = (T + 63) / 64 * 64;
    CHECK(q.ld_h == wide && q.ld_w == wide);
    // Losses alone: columns by tiles of 256, then by 128.
    const int64_t columns = (V + 255) / 256;
    CHECK(q.front >= 1 && q.front <= columns && (q.front == columns || (q.tile == 256 && !p.grads)));
    const int64_t slots = q.front == columns ? (V + square - 1) / square
                                             : q.front + (V - 256 * int64_t(q.front) + 127) / 128;
    // Parts in order, at 256 bytes, each long enough for what the kernels write.
    struct Part {
        int64_t at, bytes;
    };
    std::vector<Part> parts = {{q.scalars, dsm::kCeScalars}, {q.coef, 4 * T}, {q.lse, 4 * T}, {q.hit, 4 * T},
                               {q.stats, slots * T * 8}, {q.h, high * wide * 2}, {q.w, V * wide * 2}};
    if (p.grads && T > 0) {
        CHECK(q.piece > 0 && q.piece % square == 0 && q.piece < V + square);
        CHECK(q.dh_splits >= 1 && q.dh_splits <= 128);
        CHECK(q.ld_p == q.piece * units && q.ld_dh >= D && q.ld_dh % 4 == 0);
        const int64_t g = T * q.ld_p * 2;
        if (q.form == dsm::kCeBf16) CHECK(q.p_lo == T * q.ld_p);
        const int64_t all = q.form == dsm::kCeBf16 ? 2 * g : g;
        CHECK(all <= (int64_t(1) << 30) || q.piece == square);
        // A launch has a group for each 2048 columns of each row.
        CHECK(T * ((q.piece + 2047) / 2048) < (int64_t(1) << 31));
        parts.push_back({q.tops, T * (q.piece / square) * 16});
        if (q.sample > 0) {
            CHECK(q.tile == 256 && (q.form == dsm::kCeHalf || q.form == dsm::kCeHalves));
            // Sampled tile columns lie inside the vocabulary, and are a 64th of it.
            CHECK(q.every >= 4 && int64_t(q.sample) * q.every <= (V + 255) / 256);
            CHECK(int64_t(q.sample) * 64 * 256 >= V);
            CHECK(q.ld_ht == high * units);
            parts.push_back({q.refs, T * 4});
            parts.push_back({q.rows, T * 8});
            parts.push_back({q.ht, D * q.ld_ht * 2});
            CHECK((q.form == dsm::kCeHalf) == (q.ld_wt > 0));
            if (q.ld_wt > 0) {
                CHECK(q.ld_wt >= V && q.ld_wt % 64 == 0);
                parts.push_back({q.wt, D * q.ld_wt * 2});
            }
        }
        parts.push_back({q.p, all});
        parts.push_back({q.dh, q.dh_splits * T * q.ld_dh * 4});
    }
    int64_t end = 0;
    for (const Part& part : parts) {
        CHECK(part.at % 256 == 0 && part.at >= end);
        end = part.at + part.bytes;
    }
    CHECK(end <= q.bytes);
    // Tiles of a launch fit a grid's 32 bits.
    CHECK((T + q.tile - 1) / q.tile * ((V + square - 1) / square) < (int64_t(1) << 31));
}

static void cross_entropy() {
    for (int k = 0; k < 4000; ++k) {
        dsm_ce_problem p{};
        p.tokens = k % 50 == 0 ? 0 : spread(1 << 16);
        p.dim = spread(8192);
        p.vocab = spread(1 << 18);
        p.dtype = static_cast<int32_t>(pick(0, 1));
        p.grads = static_cast<int32_t>(pick(0, 1));
        int64_t ws = -1;
        CHECK(dsm_ce_workspace(&p, &ws) == DSM_OK && ws > 0);
        dsm_ce_buffers b = ce_buffers(p, ws);
        const int64_t elem = p.dtype == DSM_F32 ? 4 : 2;
        const int64_t skip = pick(0, 3) ? 0 : pick(0, 15) * elem;
        b.w = at((uint64_t(2) << 40) + skip);
        b.w_stride += pick(0, 3) ? 0 : pick(0, 70);
        b.h_stride += pick(0, 3) ? 0 : pick(0, 70);
        ce_calls.clear();
        CHECK(dsm_linear_ce(&p, &b, 1) == DSM_OK && ce_calls.size() == 1);
        const CeCall& c = ce_calls[0];
        check_plan(p, c.plan, ws);
        // Direct reads are 16 bytes at whole steps of k.
        const bool aligned = skip % 16 == 0 && b.w_stride * elem % 16 == 0 && p.dim % 64 == 0;
        const bool whole = c.plan.form == dsm::kCeBf16 || c.plan.form == dsm::kCeF32;
        CHECK(c.buf.w_direct == (aligned && whole));
        CHECK(c.buf.h_direct == (c.buf.w_direct && !p.grads && b.h_stride * elem % 16 == 0));
        CHECK(!c.buf.w_vector || (p.dim % 4 == 0 && b.w_stride % 4 == 0 && skip % (4 * elem) == 0));
        CHECK(c.buf.mean == 1);
        b.workspace_bytes = ws - 1;
        CHECK(dsm_linear_ce(&p, &b, 1) == DSM_ERR_INVALID_ARG && ce_calls.size() == 1);
    }
    // Refusals: nothing is launched.
    const dsm_ce_problem good{100, 64, 1000, DSM_F32, 1};
    int64_t ws = 0;
    CHECK(dsm_ce_workspace(&good, &ws) == DSM_OK);
    CHECK(dsm_ce_workspace(&good, nullptr) == DSM_ERR_INVALID_ARG && dsm_ce_workspace(nullptr, &ws) == DSM_ERR_INVALID_ARG);
    ce_calls.clear();
    const auto refused = [&](const dsm_ce_problem& p, const dsm_ce_buffers* b, const char* what) {
        CHECK(dsm_linear_ce(&p, b, 0) == DSM_ERR_INVALID_ARG);
        CHECK(last_message.find(what) != std::string::npos);
        CHECK(ce_calls.empty());
    };
    const dsm_ce_buffers fine = ce_buffers(good, ws);
    refused(good, nullptr, "buffers");
    dsm_ce_problem p = good;
    for (int64_t bad : {int64_t(-1), (int64_t(1) << 20) + 1}) refused((p = good, p.tokens = bad, p), &fine, "tokens");
    for (int64_t bad : {int64_t(0), (int64_t(1) << 16) + 1}) refused((p = good, p.dim = bad, p), &fine, "dim");
    for (int64_t bad : {int64_t(0), (int64_t(1) << 20) + 1}) refused((p = good, p.vocab = bad, p), &fine, "vocab");
    refused((p = good, p.dtype = 2, p), &fine, "dtype");
    refused((p = good, p.grads = 2, p), &fine, "grads");
    dsm_ce_buffers b = fine;
    refused(good, (b = fine, b.h = nullptr, &b), "NULL");
    refused(good, (b = fine, b.w = nullptr, &b), "NULL");
    refused(good, (b = fine, b.target = nullptr, &b), "NULL");
    refused(good, (b = fine, b.total = nullptr, &b), "NULL");
    refused(good, (b = fine, b.loss = nullptr, &b), "NULL");
    refused(good, (b = fine, b.dh = nullptr, &b), "NULL");
    refused(good, (b = fine, b.dw = nullptr, &b), "NULL");
    refused(good, (b = fine, b.workspace = nullptr, &b), "workspace");
    refused(good, (b = fine, b.workspace = at((uint64_t(8) << 40) + 128), &b), "aligned");
    refused(good, (b = fine, b.h_stride = 63, &b), "stride");
    refused(good, (b = fine, b.w_stride = 63, &b), "stride");
    refused(good, (b = fine, b.dh_stride = 63, &b), "stride");
    refused(good, (b = fine, b.dw_stride = 63, &b), "stride");
    refused(good, (b = fine, b.h = at((uint64_t(1) << 40) + 2), &b), "aligned");
    refused(good, (b = fine, b.dw = at((uint64_t(7) << 40) + 1), &b), "aligned");
    refused(good, (b = fine, b.target = static_cast<const int64_t*>(at((uint64_t(3) << 40) + 4)), &b), "aligned");
    refused(good, (b = fine, b.weight = static_cast<const float*>(at((uint64_t(9) << 40) + 2)), &b), "aligned");
    devices = 0;
    CHECK(dsm_linear_ce(&good, &fine, 0) == DSM_ERR_HIP && ce_calls.empty());
    devices = 1;
    launch_result = hipErrorInvalidValue;
    CHECK(dsm_linear_ce(&good, &fine, 0) == DSM_ERR_HIP);
    launch_result = hipSuccess;
}

// ---- Orthogonalised updates ----

static dsm_ortho_buffers ortho_buffers(int64_t ws) {
    dsm_ortho_buffers b{};
    b.in = at(uint64_t(1) << 40);
    b.out = at(uint64_t(2) << 40);
    b.workspace = at(uint64_t(3) << 40);
    b.workspace_bytes = ws;
    return b;
}

// Every stored operand of every iteration stays under fp16's largest number, for
// singular values anywhere in their range.
static void check_scales(const OrthoCall& c) {
    const size_t steps = c.scales.size();
    for (int k = 0; k <= 400; ++k) {
        double s = 1.0005 * k / 400.0;
        for (size_t i = 0; i < steps; ++i) {
            const double a = c.coeffs[3 * i], b = c.coeffs[3 * i + 1], q = c.coeffs[3 * i + 2], l = s * s;
            const dsm::OrthoScales& e = c.scales[i];
            CHECK(std::fabs(s) * std::ldexp(1.0, e.x) < 65504);
            CHECK(l * std::ldexp(1.0, e.a) < 65504);
            CHECK(std::fabs(b * l + q * l * l) * std::ldexp(1.0, e.b) < 65504);
            CHECK(e.x_next == (i + 1 < steps ? c.scales[i + 1].x : 0));
            CHECK(std::fabs(a) + std::fabs(b) + std::fabs(q) <= std::ldexp(1.0, e.growth));
            s = a * s + b * s * l + q * s * l * l;
        }
    }
}

static void orthogonalised() {
    for (int k = 0; k < 1500; ++k) {
        dsm_ortho_problem p{};
        p.rows = spread(5000);
        p.cols = spread(5000);
        p.row_stride = p.cols + (pick(0, 2) ? 0 : pick(0, 9));
        p.count = static_cast<int32_t>(spread(200));
        p.dtype = static_cast<int32_t>(pick(0, 1));
        p.steps = static_cast<int32_t>(pick(1, 8));
        p.eps = 1e-7f;
        std::vector<float> coeffs;
        for (int i = 0; i < 3 * p.steps; ++i) coeffs.push_back(std::uniform_real_distribution<float>(-3, 3)(rng));
        p.coeffs = pick(0, 1) ? coeffs.data() : nullptr;
        std::vector<int64_t> offsets;
        for (int i = 0; i < p.count; ++i) offsets.push_back(i * (p.rows * p.row_stride + (k % 3)));
        p.offsets = offsets.data();
        int64_t ws = -1;
        const dsm_status st = dsm_ortho_workspace(&p, &ws);
        CHECK(st == DSM_OK || (st == DSM_ERR_UNSUPPORTED && p.coeffs));
        if (st != DSM_OK) continue;
        const bool none = dsm::ortho_group_bytes(1, static_cast<int>(std::min(p.rows, p.cols)),
                                                 static_cast<int>(std::max(p.rows, p.cols)), p.dtype == DSM_BF16) == 0;
        CHECK(none ? ws == 0 : ws > 0);
        dsm_ortho_buffers b = ortho_buffers(ws);
        if (none) b.workspace = nullptr;
        ortho_calls.clear();
        CHECK(dsm_orthogonalize(&p, &b) == DSM_OK);
        int done = 0;
        for (const OrthoCall& c : ortho_calls) {
            const dsm::OrthoGroup& g = c.group;
            CHECK(g.count >= 1 && g.count <= dsm::kOrthoGroup);
            CHECK(g.m == std::min(p.rows, p.cols) && g.n == std::max(p.rows, p.cols));
            CHECK(g.tall == (p.rows > p.cols) && g.bf16 == (p.dtype == DSM_BF16) && g.row_stride == p.row_stride);
            CHECK(dsm::ortho_group_bytes(g.count, g.m, g.n, g.bf16) <= ws);
            CHECK(!g.mom && !g.x && g.scale == 1.0f);
            for (int i = 0; i < g.count; ++i) {
                CHECK(g.off.at[i] == offsets[done + i]);
                if (g.vector) CHECK(offsets[done + i] % 4 == 0 && p.row_stride % 4 == 0);
            }
            done += g.count;
        }
        CHECK(done == p.count);
        check_scales(ortho_calls[0]);
        if (ws > 0) {
            b.workspace_bytes = ws - 1;
            CHECK(dsm_orthogonalize(&p, &b) == DSM_ERR_INVALID_ARG);
        }
    }
    const int64_t offsets[2] = {0, 4096};
    dsm_ortho_problem good{};
    good.rows = 40;
    good.cols = good.row_stride = 100;
    good.offsets = offsets;
    good.count = 2;
    good.steps = 5;
    int64_t ws = 0;
    CHECK(dsm_ortho_workspace(&good, &ws) == DSM_OK && ws > 0);
    const dsm_ortho_buffers fine = ortho_buffers(ws);
    const dsm_ortho_hparams hp{0.1f, 0.9f, 1.0f, 0.1f, 1};
    ortho_calls.clear();
    const auto refused = [&](dsm_status got, dsm_status want, const char* what) {
        CHECK(got == want);
        CHECK(last_message.find(what) != std::string::npos);
        CHECK(ortho_calls.empty());
    };
    dsm_ortho_problem p = good;
    dsm_ortho_buffers b = fine;
    const auto run = [&] { return dsm_orthogonalize(&p, &b); };
    refused((p = good, p.rows = -1, run()), DSM_ERR_INVALID_ARG, "rows");
    refused((p = good, p.cols = p.row_stride = (1 << 20) + 1, run()), DSM_ERR_INVALID_ARG, "cols");
    refused((p = good, p.rows = p.cols = p.row_stride = (1 << 14) + 1, run()), DSM_ERR_INVALID_ARG, "smaller");
    refused((p = good, p.row_stride = 99, run()), DSM_ERR_INVALID_ARG, "row_stride");
    refused((p = good, p.count = -1, run()), DSM_ERR_INVALID_ARG, "count");
    refused((p = good, p.dtype = 3, run()), DSM_ERR_INVALID_ARG, "dtype");
    refused((p = good, p.steps = 0, run()), DSM_ERR_INVALID_ARG, "steps");
    refused((p = good, p.steps = 33, run()), DSM_ERR_INVALID_ARG, "steps");
    refused((p = good, p.eps = -1.0f, run()), DSM_ERR_INVALID_ARG, "eps");
    refused((p = good, p.eps = NAN, run()), DSM_ERR_INVALID_ARG, "eps");
    refused((p = good, p.offsets = nullptr, run()), DSM_ERR_INVALID_ARG, "offsets");
    const int64_t negative[2] = {0, -4};
    refused((p = good, p.offsets = negative, run()), DSM_ERR_INVALID_ARG, "offsets[1]");
    const float grows[6] = {100, 0, 0, 100, 0, 0}, infinite[3] = {INFINITY, 0, 0};
    refused((p = good, p.steps = 2, p.coeffs = grows, run()), DSM_ERR_UNSUPPORTED, "grow");
    refused((p = good, p.steps = 1, p.coeffs = infinite, run()), DSM_ERR_INVALID_ARG, "finite");
    p = good;
    refused((b = fine, b.in = nullptr, run()), DSM_ERR_INVALID_ARG, "NULL");
    refused((b = fine, b.out = nullptr, run()), DSM_ERR_INVALID_ARG, "NULL");
    refused((b = fine, b.in = at((uint64_t(1) << 40) + 2), run()), DSM_ERR_INVALID_ARG, "aligned");
    refused((b = fine, b.m = static_cast<float*>(at(256)), run()), DSM_ERR_INVALID_ARG, "dsm_ortho_step");
    refused((b = fine, b.workspace = nullptr, run()), DSM_ERR_INVALID_ARG, "workspace");
    refused(dsm_orthogonalize(&p, nullptr), DSM_ERR_INVALID_ARG, "buffers");
    dsm_ortho_hparams h = hp;
    float* x = static_cast<float*>(at(uint64_t(5) << 40));
    const auto step = [&] { return dsm_ortho_step(&p, &b, &h); };
    b = fine;
    b.x = x;
    refused(step(), DSM_ERR_INVALID_ARG, "exactly one");
    b.out = nullptr;
    refused((h = hp, h.lr = 0, step()), DSM_ERR_INVALID_ARG, "lr");
    refused((h = hp, h.mu = 1.5f, step()), DSM_ERR_INVALID_ARG, "mu");
    refused((h = hp, h.scale = INFINITY, step()), DSM_ERR_INVALID_ARG, "scale");
    refused((h = hp, h.weight_decay = -1, step()), DSM_ERR_INVALID_ARG, "weight_decay");
    refused(dsm_ortho_step(&p, &b, nullptr), DSM_ERR_INVALID_ARG, "hparams");
    refused((h = hp, p.dtype = DSM_BF16, step()), DSM_ERR_INVALID_ARG, "fp32");
    p = good;
    b.x = nullptr;
    refused(step(), DSM_ERR_INVALID_ARG, "exactly one");
    b.x = x;
    CHECK(step() == DSM_OK && ortho_calls.size() == 1 && ortho_calls[0].group.x == x && ortho_calls[0].group.lr == 0.1f);
    ortho_calls.clear();
    // Nothing to do: nothing is launched, no device is needed.
    devices = 0;
    for (int64_t dsm_ortho_problem::*size : {&dsm_ortho_problem::rows, &dsm_ortho_problem::cols}) {
        p = good;
        p.*size = 0;
        CHECK(dsm_orthogonalize(&p, &fine) == DSM_OK && step() == DSM_OK);
    }
    p = good;
    p.count = 0;
    CHECK(dsm_orthogonalize(&p, &fine) == DSM_OK && ortho_calls.empty());
    CHECK(dsm_orthogonalize(&good, &fine) == DSM_ERR_HIP && ortho_calls.empty());
    devices = 1;
    launch_result = hipErrorInvalidValue;
    CHECK(dsm_orthogonalize(&good, &fine) == DSM_ERR_HIP);
}

int main() {
    cross_entropy();
    orthogonalised();
    std::printf("all checks passed (%ld)\n", checks);
    return 0;
}
