// Host checks of the runtime of the linear layer, the norms and clipping
// (paper_2411_17866_amd/csrc/block_runtime.cpp): compiled with g++ under sanitizers against
// stubs of the launchers and of the HIP calls, so that every plan, argument check and
// launch argument can be looked at without a GPU.  Prints "all checks passed".
#include <algorithm>
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <random>
#include <string>
#include <vector>

#include "block_internal.h"

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
static std::vector<dsm::LinearCall> linear_calls;
static std::vector<dsm::NormCall> norm_calls;
enum Step { kSquares, kNorms, kScale, kRest };
struct ClipCall {
    Step step;
    dsm::ClipTable table;
    std::vector<int64_t> starts;
    const double *parts, *factor;
};
static std::vector<ClipCall> clip_calls;
static int64_t clip_bytes = 0;

template <class Groups>
static std::vector<int64_t> starts_of(const Groups& g) {
    return {g.start, g.start + g.count + 1};
}

namespace dsm {
dsm_status set_thread_error(dsm_status st, const char* message) {
    last_message = message;
    return st;
}
hipError_t launch_linear(const LinearCall& c, hipStream_t) { return linear_calls.push_back(c), launch_result; }
hipError_t launch_linear_backward(const LinearCall& c, hipStream_t) { return linear_calls.push_back(c), launch_result; }
hipError_t launch_norm(const NormCall& c, hipStream_t) { return norm_calls.push_back(c), launch_result; }
hipError_t launch_norm_backward(const NormCall& c, hipStream_t) { return norm_calls.push_back(c), launch_result; }
// The kernels' own rule is not compiled here.
int norm_groups(int64_t tokens, int64_t) { return static_cast<int>(std::min<int64_t>(tokens, 700)); }
hipError_t launch_clip_squares(const ClipTable& t, int64_t bytes, double* parts, hipStream_t) {
    clip_bytes = bytes;
    return clip_calls.push_back({kSquares, t, {}, parts, nullptr}), launch_result;
}
hipError_t launch_clip_norms(const ClipGroups& g, const double* parts, float*, double* factor, hipStream_t) {
    return clip_calls.push_back({kNorms, {}, starts_of(g), parts, factor}), launch_result;
}
hipError_t launch_clip_scale(const ClipTable& t, const double* factor, hipStream_t) {
    return clip_calls.push_back({kScale, t, {}, nullptr, factor}), launch_result;
}
hipError_t launch_clip_rest(const ClipTable& t, const ClipFew& g, const double* parts, float*, hipStream_t) {
    return clip_calls.push_back({kRest, t, starts_of(g), parts, nullptr}), launch_result;
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
static void* place(int k) { return at(static_cast<uint64_t>(k) << 44); }

static void refused(dsm_status got, const char* what, dsm_status want = DSM_ERR_INVALID_ARG) {
    if (got != want || last_message.find(what) == std::string::npos)
        std::printf("status %d, message %s, wanted %s\n", got, last_message.c_str(), what);
    CHECK(got == want && last_message.find(what) != std::string::npos);
    CHECK(linear_calls.empty() && norm_calls.empty() && clip_calls.empty());
}

// ---- Linear layer ----

static dsm_linear_buffers linear_buffers(const dsm_linear_problem& p, int64_t ws) {
    dsm_linear_buffers b{};
    b.x = place(1);
    b.w = place(2);
    b.bias = static_cast<const float*>(place(3));
    b.residual = place(4);
    b.y = place(5);
    b.z = place(6);
    b.dy = place(7);
    b.dx = place(8);
    b.dw = place(9);
    b.dbias = static_cast<float*>(place(10));
    b.workspace = place(11);
    b.workspace_bytes = ws;
    b.x_stride = b.w_stride = b.dx_stride = b.dw_stride = p.dim;
    b.residual_stride = b.y_stride = b.z_stride = b.dy_stride = p.wide;
    return b;
}

struct Region {
    int64_t at, bytes;
};
// Regions that a pass's kernels use at once: none meets another, all end before `end`.
static void check_regions(std::vector<Region> all, int64_t end) {
    all.erase(std::remove_if(all.begin(), all.end(), [](const Region& r) { return r.bytes == 0; }), all.end());
    std::sort(all.begin(), all.end(), [](const Region& a, const Region& b) { return a.at < b.at; });
    int64_t from = 0;
    for (const Region& r : all) {
        CHECK(r.at >= from && r.at % 256 == 0);
        from = r.at + r.bytes;
    }
    CHECK(from <= end);
}
static int64_t up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }
static bool reads_whole(int64_t address, int64_t stride, int64_t cols, int64_t size, int64_t run) {
    return address % 16 == 0 && stride * size % 16 == 0 && cols * size % (run * 2) == 0 && stride * size < (int64_t(1) << 23);
}

static void check_forward(const dsm_linear_problem& p, const dsm_linear_buffers& b, const dsm::LinearCall& c, int64_t ws) {
    const dsm::LinearPlan& q = c.p;
    const int64_t T = p.tokens, D = p.dim, N = p.wide, size = p.dtype == DSM_F32 ? 4 : 2;
    CHECK(q.tokens == T && q.dim == D && q.wide == N && q.act == p.act && q.f32 == (p.dtype == DSM_F32));
    CHECK(q.forward_bytes <= ws && q.splits >= 1 && q.splits <= 16);
    CHECK((q.form == dsm::kLinearBf16) == !q.f32);
    CHECK(q.ld_y >= N && q.ld_y % 8 == 0);
    if (q.few) {
        CHECK(T <= 64 && (q.splits == 1 || (N + 15) / 16 * q.splits <= (q.f32 && T <= 32 ? 512 : 256)));
        check_regions({{q.y_parts, q.splits > 1 ? q.splits * T * q.ld_y * 4 : 0}}, q.forward_bytes);
        return;
    }
    // The instantiations that the launcher has.
    CHECK(q.tile == 64 || (q.form != dsm::kLinearSingle && (q.tile == 128 || q.tile == 256)));
    CHECK(q.front >= 1 && q.front <= (N + q.tile - 1) / q.tile);
    if (q.tile != 256 || q.splits > 1) CHECK(q.front == (N + q.tile - 1) / q.tile);
    const int64_t units = q.f32 ? 2 : 1;
    CHECK(q.ld_dim >= up(D, 64) * units && q.ld_dim % (64 * units) == 0);
    // What is read where it lies is whole runs of 64 16-bit elements.
    const bool may = q.form != dsm::kLinearHalves;
    CHECK(c.x_direct == (may && reads_whole(reinterpret_cast<int64_t>(b.x), b.x_stride, D, size, 64)));
    CHECK(c.w_direct == (may && reads_whole(reinterpret_cast<int64_t>(b.w), b.w_stride, D, size, 64)));
    const bool exps = q.form == dsm::kLinearHalves;
    check_regions({{q.x, c.x_direct ? 0 : T * q.ld_dim * 2}, {q.w, c.w_direct ? 0 : N * q.ld_dim * 2}, {q.x_exp, exps ? T * 4 : 0},
                   {q.w_exp, exps ? N * 4 : 0}, {q.y_parts, q.splits > 1 ? q.splits * T * q.ld_y * 4 : 0}}, q.forward_bytes);
    // Work-groups of at most 512 threads: fewer than 2^32 in a launch.
    CHECK((T + q.tile - 1) / q.tile * ((N + q.tile - 1) / q.tile) * q.splits < (int64_t(1) << 23));
}

static void check_backward(const dsm_linear_problem& p, const dsm_linear_buffers& b, const dsm::LinearCall& c, int64_t ws) {
    const dsm::LinearPlan& q = c.p;
    const int64_t T = p.tokens, D = p.dim, N = p.wide, size = p.dtype == DSM_F32 ? 4 : 2, units = size / 2;
    CHECK(q.backward_bytes <= ws);
    CHECK(c.z_in == (p.act ? b.z : nullptr));
    if (T == 0) return;
    CHECK(q.dx_splits >= 1 && q.dx_splits <= 16 && q.dw_splits >= 1 && q.dw_splits <= 16);
    CHECK(q.dz_halves == (!q.f32 && p.dw_dtype == DSM_F32 && p.act != 0));
    CHECK(q.pad_tokens % 64 == 0 && q.pad_tokens >= T);
    CHECK(q.ld_wide >= up(N, 64) * units && q.ld_wide % (64 * units) == 0 && q.ld_dx >= D && q.ld_dx % 8 == 0);
    const bool few = q.back_few, halves = q.back_form == dsm::kLinearHalves;
    if (few) CHECK(T <= (q.f32 ? 64 : 32) && q.dw_splits == 1 && q.bias_parts == 1);
    CHECK(few || q.back_form != dsm::kLinearSingle);
    if (!few) CHECK(q.back_tile == 64 || q.back_tile == 128 || q.back_tile == 256);
    if (halves) CHECK(q.split_rows == 8 || (q.split_rows == 2 && N <= 8192));
    // dbias's parts: of the kernels that make dz.
    CHECK(q.bias_parts == (halves ? (T + q.split_rows - 1) / q.split_rows : q.pad_tokens / dsm::kDzRows));
    // dz's rows past the tokens meet x's last one, and have to be zeros.
    CHECK(c.dz_direct == (!p.act && q.back_form == dsm::kLinearBf16 &&
                          (few || (T % 64 == 0 && reads_whole(reinterpret_cast<int64_t>(b.dy), b.dy_stride, N, size, 64)))));
    CHECK(c.x_direct == (!halves && !q.dz_halves && reads_whole(reinterpret_cast<int64_t>(b.x), b.x_stride, D, size, 8)));
    CHECK(c.w_direct == (!halves && reads_whole(reinterpret_cast<int64_t>(b.w), b.w_stride, D, size, 8)));
    const int64_t twice = q.dz_halves ? 2 : 1;
    check_regions({{q.x, c.x_direct || few ? 0 : (q.dz_halves ? 2 * q.pad_tokens : T) * q.ld_dim * 2},
                   {q.w, c.w_direct || few ? 0 : N * q.ld_dim * 2}, {q.x_exp, halves ? 4 : 0}, {q.w_exp, halves ? 4 : 0},
                   {q.dz, c.dz_direct ? 0 : q.pad_tokens * q.ld_wide * 2 * twice}, {q.z_exp, halves ? T * 4 : 0},
                   {q.w_tops, halves ? dsm::kLinearTopParts * 4 : 0}, {q.tops, halves ? q.pad_tokens / q.split_rows * 4 : 0},
                   {q.dx_parts, q.dx_splits > 1 ? q.dx_splits * T * q.ld_dx * 4 : 0},
                   {q.dw_parts, q.dw_splits > 1 ? q.dw_splits * N * q.ld_dx * 4 : 0}, {q.bias_sums, q.bias_parts * N * 4}},
                  q.backward_bytes);
    if (few) return;
    const int64_t of = q.back_tile, across = (D + of - 1) / of;
    CHECK(((T + of - 1) / of * q.dx_splits + (N + of - 1) / of * q.dw_splits) * across + (N + 127) / 128 * (q.pad_tokens / 64) <
          (int64_t(1) << 24));
}

static void linear() {
    for (int round = 0; round < 6000; ++round) {
        dsm_linear_problem p{};
        p.tokens = round % 50 == 0 ? int64_t(1) << 20 : round % 3 ? spread(8192) : pick(0, 200);
        p.dim = round % 70 == 0 ? 1 << 16 : spread(8192);
        p.wide = round % 90 == 0 ? 1 << 16 : spread(12000);
        if (round % 4 == 0) p.dim = up(p.dim, 64), p.wide = up(p.wide, 64);
        if (round % 8 == 0) p.tokens = std::min<int64_t>(up(p.tokens, 64), 1 << 20);
        p.dtype = round % 2;
        p.act = round / 2 % 5;
        p.dw_dtype = round / 10 % 2 ? DSM_F32 : p.dtype;
        p.grads = round % 7 != 0;
        int64_t ws = -1, again = -1;
        CHECK(dsm_linear_workspace(&p, &ws) == DSM_OK && ws >= 0);
        dsm_linear_buffers b = linear_buffers(p, ws);
        const int64_t pad = pick(0, 3) == 0 ? pick(1, 40) : pick(0, 1) * 64;
        b.x_stride += pad;
        b.w_stride += pick(0, 1) * 8;
        b.dy_stride += pad;
        if (round % 11 == 0) b.w_stride = (int64_t(1) << 22) + 64;
        if (round % 13 == 0) b.x = at((uint64_t(1) << 44) + 4);
        if (round % 17 == 0) b.dy = at((uint64_t(7) << 44) + 8);
        linear_calls.clear();
        CHECK(dsm_linear(&p, &b) == DSM_OK);
        CHECK(linear_calls.size() == (p.tokens > 0));
        for (const auto& c : linear_calls) {
            CHECK(c.x == b.x && c.w == b.w && c.y == b.y && c.z == b.z && c.residual == b.residual && c.bias == b.bias);
            CHECK(c.x_stride == b.x_stride && c.w_stride == b.w_stride && c.y_stride == b.y_stride && c.workspace == b.workspace);
            check_forward(p, b, c, ws);
            if (c.p.forward_bytes > 0) {
                linear_calls.clear();
                b.workspace_bytes = c.p.forward_bytes - 1;
                refused(dsm_linear(&p, &b), "workspace_bytes");
                b.workspace_bytes = ws;
                break;
            }
        }
        linear_calls.clear();
        if (!p.grads) {
            refused(dsm_linear_backward(&p, &b), "without gradients");
            continue;
        }
        CHECK(dsm_linear_backward(&p, &b) == DSM_OK && linear_calls.size() == 1);
        const dsm::LinearCall c = linear_calls[0];
        CHECK(c.dx == b.dx && c.dw == b.dw && c.dbias == b.dbias && c.dy == b.dy && c.dy_stride == b.dy_stride);
        check_backward(p, b, c, ws);
        linear_calls.clear();
        if (c.p.backward_bytes > 0) {
            b.workspace_bytes = c.p.backward_bytes - 1;
            refused(dsm_linear_backward(&p, &b), "workspace_bytes");
        }
        // Plans of problems that differ in one field are their own.
        dsm_linear_problem other = p;
        if (p.dtype == DSM_BF16) other.dw_dtype = p.dw_dtype == DSM_F32 ? DSM_BF16 : DSM_F32;
        other.act = (p.act + 1) % 5;
        for (const dsm_linear_problem& one : {dsm_linear_problem{p.tokens, p.dim, p.wide, p.dtype, other.act, p.dw_dtype, 1},
                                              dsm_linear_problem{p.tokens, p.dim, p.wide, p.dtype, p.act, other.dw_dtype, 1}}) {
            int64_t bytes = 0;
            CHECK(dsm_linear_workspace(&one, &bytes) == DSM_OK);
            b.workspace_bytes = bytes;
            CHECK(dsm_linear_backward(&one, &b) == DSM_OK);
            check_backward(one, b, linear_calls[0], bytes);
            linear_calls.clear();
        }
        // A plan is the same whenever it is asked for, among others or again.
        CHECK(dsm_linear_workspace(&p, &again) == DSM_OK && again == ws);
    }
    const dsm_linear_problem good{100, 40, 60, DSM_F32, DSM_ACT_GELU, DSM_F32, 1};
    int64_t ws = 0;
    CHECK(dsm_linear_workspace(&good, &ws) == DSM_OK && ws > 0);
    const dsm_linear_buffers fine = linear_buffers(good, ws);
    dsm_linear_problem p = good;
    dsm_linear_buffers b = fine;
    for (int back = 0; back < 2; ++back) {
        const auto run = [&] { return back ? dsm_linear_backward(&p, &b) : dsm_linear(&p, &b); };
        refused((p = good, p.tokens = -1, run()), "tokens");
        refused((p = good, p.tokens = (1 << 20) + 1, run()), "tokens");
        refused((p = good, p.dim = 0, run()), "dim");
        refused((p = good, p.dim = (1 << 16) + 1, run()), "dim");
        refused((p = good, p.wide = 0, run()), "wide");
        refused((p = good, p.wide = (1 << 16) + 1, run()), "wide");
        refused((p = good, p.dtype = 2, run()), "dtype");
        refused((p = good, p.act = 5, run()), "act");
        refused((p = good, p.act = -1, run()), "act");
        refused((p = good, p.dw_dtype = DSM_BF16, run()), "dw_dtype");
        refused((p = good, p.grads = 2, run()), "grads");
        p = good;
        refused((b = fine, b.x = nullptr, run()), "x is NULL");
        refused((b = fine, b.w = nullptr, run()), "w is NULL");
        refused((b = fine, b.x_stride = 39, run()), "x_stride");
        refused((b = fine, b.w_stride = 39, run()), "w_stride");
        refused((b = fine, b.z_stride = 59, run()), "z_stride");
        refused((b = fine, b.x = at((uint64_t(1) << 44) + 2), run()), "x is not aligned");
        refused((b = fine, b.z = at((uint64_t(6) << 44) + 1), run()), "z is not aligned");
        refused((b = fine, b.workspace = nullptr, run()), "workspace is NULL");
        refused((b = fine, b.workspace = at((uint64_t(11) << 44) + 128), run()), "workspace is not");
        refused(back ? dsm_linear_backward(&good, nullptr) : dsm_linear(&good, nullptr), "buffers");
        refused(back ? dsm_linear_backward(nullptr, &fine) : dsm_linear(nullptr, &fine), "problem");
    }
    const auto forward = [&] { return dsm_linear(&p, &b); };
    refused((b = fine, b.y = nullptr, forward()), "y is NULL");
    refused((b = fine, b.y_stride = 59, forward()), "y_stride");
    refused((b = fine, b.residual_stride = 59, forward()), "residual_stride");
    refused((b = fine, b.bias = static_cast<const float*>(at((uint64_t(3) << 44) + 2)), forward()), "bias");
    for (const void* in : {b.x, b.w, static_cast<const void*>(fine.z)})
        refused((b = fine, b.y = const_cast<void*>(in), forward()), "y is x, w or z");
    for (const void* in : {fine.x, fine.w, fine.residual})
        refused((b = fine, b.z = const_cast<void*>(in), forward()), "z is x, w or residual");
    refused((b = fine, b.y = const_cast<void*>(b.residual), b.y_stride = 61, forward()), "another stride");
    const auto backward = [&] { return dsm_linear_backward(&p, &b); };
    refused((b = fine, b.dy = nullptr, backward()), "dy is NULL");
    refused((b = fine, b.z = nullptr, backward()), "z is NULL");
    refused((b = fine, b.dy_stride = 59, backward()), "dy_stride");
    refused((b = fine, b.dx_stride = 39, backward()), "dx_stride");
    refused((b = fine, b.dw_stride = 39, backward()), "dw_stride");
    refused((b = fine, b.dbias = static_cast<float*>(at((uint64_t(10) << 44) + 2)), backward()), "dbias");
    refused((b = fine, b.dw = b.dx, backward()), "dx is dw");
    for (const void* in : {fine.x, fine.w, fine.dy, static_cast<const void*>(fine.z)}) {
        refused((b = fine, b.dx = const_cast<void*>(in), backward()), "dx or dw is");
        refused((b = fine, b.dw = const_cast<void*>(in), backward()), "dx or dw is");
    }
    refused(dsm_linear_workspace(&good, nullptr), "workspace_bytes");
    // What is not wanted need not be there; nothing wanted: no device is needed.
    b = fine;
    b.dx = nullptr;
    b.w = nullptr;
    CHECK(backward() == DSM_OK && linear_calls.size() == 1);
    b = fine;
    b.dw = nullptr;
    b.x = nullptr;
    CHECK(backward() == DSM_OK && linear_calls.size() == 2);
    linear_calls.clear();
    devices = 0;
    b.dx = nullptr;
    b.dbias = nullptr;
    CHECK(backward() == DSM_OK);
    p.tokens = 0;
    CHECK((b = fine, forward()) == DSM_OK && linear_calls.empty());
    p = good;
    refused(forward(), "no HIP device", DSM_ERR_HIP);
    refused(backward(), "no HIP device", DSM_ERR_HIP);
    devices = 1;
    launch_result = hipErrorInvalidValue;
    CHECK(forward() == DSM_ERR_HIP && backward() == DSM_ERR_HIP);
    launch_result = hipSuccess;
    linear_calls.clear();
}

// ---- Norms ----

static dsm_norm_buffers norm_buffers(const dsm_norm_problem& p, int64_t ws) {
    dsm_norm_buffers b{};
    b.h = place(1);
    b.f = place(2);
    b.s = place(3);
    b.y = p.norm ? place(4) : nullptr;
    b.dy = p.norm ? place(5) : nullptr;
    b.ds = place(6);
    b.dh = place(7);
    b.df = place(8);
    float** vectors[] = {&b.dgate, &b.dweight, &b.dbias, &b.dpost_weight, &b.dpost_bias};
    const bool there[] = {true, p.norm != 0, p.norm != 0, p.post != 0, p.post != 0};
    for (int i = 0; i < 5; ++i) *vectors[i] = there[i] ? static_cast<float*>(place(10 + i)) : nullptr;
    b.workspace = place(20);
    b.workspace_bytes = ws;
    b.h_stride = b.f_stride = b.s_stride = b.y_stride = b.dy_stride = b.ds_stride = b.dh_stride = b.df_stride = p.dim;
    return b;
}

static void norms() {
    for (int round = 0; round < 500; ++round) {
        dsm_norm_problem p{spread(1 << 30), spread(8192), round % 2, round / 2 % 3, round / 6 % 3, round % 5 != 0, 1e-5f, 1e-6f, 0.5f};
        int64_t ws = -1;
        CHECK(dsm_norm_workspace(&p, &ws) == DSM_OK);
        const int64_t groups = dsm::norm_groups(p.tokens, p.dim);
        CHECK(ws >= (p.grads ? 5 * groups * p.dim * 4 : 0) && (p.grads || ws == 0));
        const dsm_norm_buffers b = norm_buffers(p, ws);
        norm_calls.clear();
        CHECK(dsm_residual_norm(&p, &b) == DSM_OK && norm_calls.size() == 1);
        const dsm::NormCall& c = norm_calls[0];
        CHECK(c.tokens == p.tokens && c.dim == p.dim && c.norm == p.norm && c.post == p.post && c.eps == p.eps &&
              c.post_eps == p.post_eps && c.scale == p.scale && c.f32 == (p.dtype == DSM_F32) && c.s == b.s && c.y == b.y);
        norm_calls.clear();
        if (!p.grads) {
            refused(dsm_residual_norm_backward(&p, &b), "without gradients");
            continue;
        }
        CHECK(dsm_residual_norm_backward(&p, &b) == DSM_OK && norm_calls.size() == 1);
        const dsm::NormCall& d = norm_calls[0];
        CHECK(d.groups == groups && d.parts == b.workspace && d.sums[0] == b.dweight && d.sums[1] == b.dbias && d.sums[2] == b.dgate &&
              d.sums[3] == b.dpost_weight && d.sums[4] == b.dpost_bias && d.f == b.f && d.dh == b.dh && d.df == b.df);
        norm_calls.clear();
        dsm_norm_buffers less = b;
        less.workspace_bytes = ws - 1;
        refused(dsm_residual_norm_backward(&p, &less), "workspace_bytes");
        // Without the vectors' gradients there are no sums, and f is not read unless post is taken back.
        less.dweight = less.dbias = less.dgate = less.dpost_weight = less.dpost_bias = nullptr;
        CHECK(dsm_residual_norm_backward(&p, &less) == DSM_OK && norm_calls.size() == 1);
        CHECK((norm_calls[0].f != nullptr) == (p.post != 0));
        norm_calls.clear();
    }
    const dsm_norm_problem good{100, 40, DSM_BF16, DSM_NORM_RMS, DSM_NORM_LAYER, 1, 1e-5f, 1e-5f, 1.0f};
    int64_t ws = 0;
    CHECK(dsm_norm_workspace(&good, &ws) == DSM_OK);
    const dsm_norm_buffers fine = norm_buffers(good, ws);
    dsm_norm_problem p = good;
    dsm_norm_buffers b = fine;
    for (int back = 0; back < 2; ++back) {
        const auto run = [&] { return back ? dsm_residual_norm_backward(&p, &b) : dsm_residual_norm(&p, &b); };
        b = fine;
        refused((p = good, p.tokens = -1, run()), "tokens");
        refused((p = good, p.tokens = (int64_t(1) << 30) + 1, run()), "tokens");
        refused((p = good, p.dim = 0, run()), "dim");
        refused((p = good, p.dim = 8193, run()), "dim");
        refused((p = good, p.dtype = -1, run()), "dtype");
        refused((p = good, p.norm = 3, run()), "norm");
        refused((p = good, p.post = -1, run()), "norm");
        refused((p = good, p.grads = 3, run()), "grads");
        refused((p = good, p.eps = -1.0f, run()), "eps");
        refused((p = good, p.eps = NAN, run()), "eps");
        refused((p = good, p.post_eps = INFINITY, run()), "eps");
        refused((p = good, p.scale = INFINITY, run()), "scale");
        p = good;
        refused((b = fine, b.h = nullptr, run()), "h is NULL");
        refused((b = fine, b.f = nullptr, run()), "f is NULL");
        refused((b = fine, b.h_stride = 39, run()), "h_stride");
        refused((b = fine, b.f_stride = 39, run()), "f_stride");
        refused((b = fine, b.h = at((uint64_t(1) << 44) + 1), run()), "h is not aligned");
        refused((b = fine, b.post_bias = static_cast<const float*>(at(258)), run()), "vector");
        refused(back ? dsm_residual_norm_backward(&good, nullptr) : dsm_residual_norm(&good, nullptr), "buffers");
        refused(back ? dsm_residual_norm_backward(nullptr, &fine) : dsm_residual_norm(nullptr, &fine), "problem");
    }
    const auto forward = [&] { return dsm_residual_norm(&p, &b); };
    refused((b = fine, b.y = nullptr, forward()), "y is NULL");
    refused((b = fine, b.y = b.s, forward()), "y is s");
    refused((p = good, p.norm = 0, b = fine, forward()), "y without a norm");
    p = good;
    p.post = 0;
    refused((b = fine, b.f = nullptr, forward()), "s without f");
    p = good;
    for (const void* in : {fine.h, fine.f}) {
        refused((b = fine, b.s = const_cast<void*>(in), b.s_stride = 41, forward()), "another stride");
        refused((b = fine, b.y = const_cast<void*>(in), b.y_stride = 41, forward()), "another stride");
        b = fine;
        b.s = const_cast<void*>(in);
        CHECK(forward() == DSM_OK);
        norm_calls.clear();
    }
    const auto backward = [&] { return dsm_residual_norm_backward(&p, &b); };
    refused((b = fine, b.dy = nullptr, backward()), "dy is NULL");
    refused((p = good, p.norm = 0, b = fine, backward()), "without a norm");
    refused((p = good, p.norm = 0, b = fine, b.dy = nullptr, b.dweight = b.dbias = nullptr, b.ds = nullptr, backward()), "ds is NULL");
    refused((p = good, p.post = 0, b = fine, backward()), "without a post norm");
    p = good;
    refused((b = fine, b.dh = b.df, backward()), "dh is df");
    refused((b = fine, b.dh = const_cast<void*>(b.f), backward()), "dh is f");
    refused((b = fine, b.dgate = b.dpost_bias, backward()), "one array");
    refused((b = fine, b.dweight = b.dbias, backward()), "one array");
    refused((b = fine, b.df = const_cast<void*>(b.dy), b.df_stride = 44, backward()), "another stride");
    refused((b = fine, b.workspace = nullptr, backward()), "workspace is NULL");
    refused(dsm_norm_workspace(&good, nullptr), "workspace_bytes");
    devices = 0;
    p.tokens = 0;
    CHECK((b = fine, forward()) == DSM_OK);
    b.dweight = b.dbias = b.dgate = b.dpost_weight = b.dpost_bias = nullptr;
    CHECK(backward() == DSM_OK);
    p = good;
    refused((b = fine, forward()), "no HIP device", DSM_ERR_HIP);
    refused(backward(), "no HIP device", DSM_ERR_HIP);
    devices = 1;
    // Sums over no tokens are written all the same.
    p.tokens = 0;
    CHECK(backward() == DSM_OK && norm_calls.size() == 1 && norm_calls[0].groups == 0);
    norm_calls.clear();
    p = good;
    launch_result = hipErrorInvalidValue;
    CHECK(forward() == DSM_ERR_HIP && backward() == DSM_ERR_HIP);
    launch_result = hipSuccess;
    norm_calls.clear();
}

// ---- Clipping ----

// Elements that lie side by side, of one type and group.
struct Stretch {
    int64_t from, bytes, size;
    int group;
    bool operator==(const Stretch& o) const { return from == o.from && bytes == o.bytes && size == o.size && group == o.group; }
};
// Those of an entry.
template <class Entry>
static void runs(const Entry& e, int64_t size, std::vector<Stretch>* out) {
    for (int64_t i = e.first; i < e.first + e.numel;) {
        const int64_t row = i / e.block, col = i % e.block, n = std::min(e.block - col, e.first + e.numel - i);
        const int64_t from = reinterpret_cast<int64_t>(e.data) + (row * e.stride + col) * size;
        const int group = static_cast<int>(e.group);
        if (!out->empty() && out->back().from + out->back().bytes == from && out->back().size == size && out->back().group == group)
            out->back().bytes += n * size;
        else
            out->push_back({from, n * size, size, group});
        i += n;
    }
}

static void clipping() {
    for (int round = 0; round < 1500; ++round) {
        const int n = static_cast<int>(round % 10 == 0 ? pick(0, 400) : pick(0, 20));
        const int groups = static_cast<int>(round % 6 == 0 ? pick(1, 256) : pick(1, 5));
        std::vector<dsm_clip_tensor> t(n);
        int64_t address = int64_t(1) << 44;
        int group = 0;
        for (int i = 0; i < n; ++i) {
            if (pick(0, 5) == 0) group = static_cast<int>(std::min<int64_t>(group + pick(0, 2), groups - 1));
            dsm_clip_tensor& e = t[i];
            e.dtype = pick(0, 3) == 0 ? DSM_BF16 : DSM_F32;
            e.group = group;
            e.numel = pick(0, 8) == 0 ? 0 : spread(round % 9 == 0 ? 3000000 : 100000);
            const int64_t size = e.dtype == DSM_F32 ? 4 : 2;
            if (i > 0 && pick(0, 3) == 0) {  // the next part of the last one's rows
                e = t[i - 1];
                const int64_t gap = pick(0, 2) == 0 ? pick(1, 9) : 0;
                e.first += e.numel + gap;
                e.numel = spread(50000);
                if (gap == 0 && t[i - 1].block >= t[i - 1].first + t[i - 1].numel && t[i - 1].block == t[i - 1].stride)
                    t[i - 1].block = t[i - 1].stride = e.block = e.stride = e.first + e.numel;
                if (e.block < e.first + e.numel) address = reinterpret_cast<int64_t>(e.data) + ((e.first + e.numel) / e.block + 1) * e.stride * size;
                else address = reinterpret_cast<int64_t>(e.data) + (e.first + e.numel) * size;
                continue;
            }
            address = up(address, size) + pick(0, 2) * 256;  // 0: right behind the last
            e.data = reinterpret_cast<void*>(address);
            if (pick(0, 2) == 0) {
                e.block = spread(5000);
                e.stride = e.block + pick(0, 100);
                e.first = pick(0, 1) * pick(0, 300);
                address += ((e.first + e.numel) / e.block + 1) * e.stride * size;
            } else {
                e.block = e.stride = std::max<int64_t>(e.numel, 1);
                address += e.numel * size;
            }
        }
        int64_t ws = 0;
        CHECK(dsm_clip_workspace(t.data(), n, groups, &ws) == DSM_OK);
        char* workspace = static_cast<char*>(at(uint64_t(1) << 60));
        float* norm = static_cast<float*>(place(2));
        const float max_norm = round % 5 == 0 ? INFINITY : 1.0f;
        clip_calls.clear();
        CHECK(dsm_grad_clip(t.data(), n, groups, max_norm, 1e-6f, norm, workspace, ws, nullptr) == DSM_OK);
        // Each pass's entries together are the tensors, in order; chunks follow each other.
        std::vector<Stretch> want, got[2];
        std::vector<int64_t> starts, chunks(groups, 0);
        for (const auto& e : t) runs(e, e.dtype == DSM_F32 ? 4 : 2, &want);
        int64_t slot[2] = {0, 0};
        int tables[2] = {0, 0};
        for (const auto& c : clip_calls) {
            if (!c.starts.empty()) starts = c.starts;
            if (c.step == kNorms) {
                CHECK(c.parts == reinterpret_cast<double*>(workspace));
                CHECK(reinterpret_cast<const char*>(c.factor) + groups * 8 <= workspace + ws);
                continue;
            }
            const int pass = c.step != kSquares;
            CHECK(c.table.count > 0 && c.table.count <= dsm::kClipEntries && c.table.slot == slot[pass]);
            int32_t chunk = 0;
            for (int k = 0; k < c.table.count; ++k) {
                const dsm::ClipEntry& e = c.table.e[k];
                CHECK(e.chunk == chunk && e.numel > 0);
                const auto n_chunks = static_cast<int32_t>((e.numel + dsm::kClipChunk - 1) / dsm::kClipChunk);
                chunk += n_chunks;
                if (!pass) chunks[e.group] += n_chunks;
                runs(e, e.bf16 ? 2 : 4, &got[pass]);
            }
            CHECK(c.table.chunks == chunk);
            slot[pass] += chunk;
            ++tables[pass];
        }
        CHECK(got[0] == want);
        int64_t bytes = 0;
        for (const Stretch& r : want) bytes += r.bytes;
        CHECK(want.empty() || clip_bytes == bytes);
        CHECK(got[1] == (max_norm < INFINITY ? want : std::vector<Stretch>()));
        CHECK(static_cast<int>(starts.size()) == groups + 1 && starts[0] == 0);
        for (int g = 0; g < groups; ++g) CHECK(starts[g + 1] - starts[g] == chunks[g]);
        // The sums end before the factors.
        const int64_t factors = max_norm < INFINITY && tables[0] == 1 && groups <= 64 && starts[groups] <= 2048 ? ws : ws - 256 * 8;
        CHECK(slot[0] * 8 <= factors);
        for (const auto& c : clip_calls) {
            if (c.factor) CHECK(reinterpret_cast<const char*>(c.factor) - workspace >= slot[0] * 8);
            CHECK((c.step == kRest) == (c.step != kSquares && factors == ws));
        }
        clip_calls.clear();
        refused(dsm_grad_clip(t.data(), n, groups, max_norm, 1e-6f, norm, workspace, ws - 1, nullptr), "workspace_bytes");
    }
    const dsm_clip_tensor good[2] = {{place(1), 0, 100, 100, 100, DSM_F32, 0}, {place(2), 5, 90, 10, 12, DSM_BF16, 1}};
    dsm_clip_tensor t[2];
    int64_t ws = 0;
    CHECK(dsm_clip_workspace(good, 2, 2, &ws) == DSM_OK);
    float* norm = static_cast<float*>(place(3));
    int32_t n = 2, groups = 2;
    float max_norm = 1.0f, eps = 0.0f;
    const auto run = [&] { return dsm_grad_clip(t, n, groups, max_norm, eps, norm, place(4), ws, nullptr); };
    const auto reset = [&] { t[0] = good[0], t[1] = good[1]; };
    reset();
    refused((n = -1, run()), "n_tensors");
    n = 2;
    refused((groups = 0, run()), "n_groups");
    refused((groups = 257, run()), "n_groups");
    refused((groups = 1, run()), "group 1");
    groups = 2;
    refused((t[0].group = 1, t[1].group = 0, run()), "group 0");
    refused((reset(), t[0].group = -1, run()), "group -1");
    refused((reset(), t[1].first = -1, run()), "first");
    refused((reset(), t[1].numel = -1, run()), "numel");
    refused((reset(), t[1].numel = (int64_t(1) << 48) + 1, run()), "numel");
    refused((reset(), t[1].numel = int64_t(1) << 48, run()), "2^37");
    refused((reset(), t[1].block = 0, run()), "block");
    refused((reset(), t[1].stride = 9, run()), "stride");
    refused((reset(), t[0].dtype = 2, run()), "dtype");
    refused((reset(), t[0].data = nullptr, run()), "data is NULL");
    refused((reset(), t[0].data = at(258), run()), "aligned");
    refused((reset(), t[1].data = at(257), run()), "aligned");
    reset();
    refused((max_norm = -1.0f, run()), "max_norm");
    refused((max_norm = NAN, run()), "max_norm");
    max_norm = 1.0f;
    refused((eps = -1.0f, run()), "eps");
    refused((eps = INFINITY, run()), "eps");
    eps = 0.0f;
    refused((norm = nullptr, run()), "norm is NULL");
    refused((norm = static_cast<float*>(at(258)), run()), "norm is not");
    norm = static_cast<float*>(place(3));
    refused(dsm_grad_clip(nullptr, 1, 1, 1.0f, 0.0f, norm, place(4), ws, nullptr), "tensors");
    refused(dsm_grad_clip(good, 2, 2, 1.0f, 0.0f, norm, nullptr, ws, nullptr), "workspace is NULL");
    refused(dsm_clip_workspace(good, 2, 2, nullptr), "workspace_bytes");
    devices = 0;
    refused(run(), "no HIP device", DSM_ERR_HIP);
    devices = 1;
    launch_result = hipErrorInvalidValue;
    CHECK(run() == DSM_ERR_HIP && clip_calls.size() == 1);
}

int main() {
    linear();
    norms();
    clipping();
    std::printf("all checks passed (%ld)\n", checks);
    return 0;
}
