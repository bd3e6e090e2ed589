// Host runtime of the language-model operators in include/dsm.h: argument
// checks, workspace plans, the powers of two of the iteration's operands, and
// launches.  The runtime owns no memory of any kind; nothing here throws.
#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>

#include "dsm.h"
#include "ops_internal.h"
#include "thread_error.h"

namespace {

constexpr int64_t kMaxTokens = int64_t(1) << 20, kMaxVocab = int64_t(1) << 20, kMaxDim = 1 << 16;
constexpr int64_t kMaxSide = int64_t(1) << 20, kMaxShort = 1 << 14;
constexpr int kMaxSteps = dsm::kOrthoMaxSteps;

dsm_status bad(dsm_status st, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
dsm_status bad(dsm_status st, const char* fmt, ...) {
    char msg[512];
    va_list ap;
    va_start(ap, fmt);
    std::vsnprintf(msg, sizeof msg, fmt, ap);
    va_end(ap);
    return dsm::set_thread_error(st, msg);
}

dsm_status invalid(const char* what) { return bad(DSM_ERR_INVALID_ARG, "%s", what); }

bool aligned(const void* p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }

int64_t round_up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }

dsm_status check_device() {
    int n = 0;
    if (hipGetDeviceCount(&n) != hipSuccess || n < 1) return bad(DSM_ERR_HIP, "no HIP device");
    return DSM_OK;
}

dsm_status launched(const char* what, hipError_t e) {
    if (e == hipSuccess) return DSM_OK;
    return bad(DSM_ERR_HIP, "%s: %s (%d)", what, hipGetErrorString(e), static_cast<int>(e));
}

dsm_status check_workspace(const void* ws, int64_t bytes, int64_t need) {
    if (!ws) return invalid("workspace is NULL");
    if (!aligned(ws, 256)) return invalid("workspace is not 256-byte aligned");
    if (bytes < need)
        return bad(DSM_ERR_INVALID_ARG, "workspace_bytes %lld < %lld", static_cast<long long>(bytes),
                   static_cast<long long>(need));
    return DSM_OK;
}

// ---- Linear layer with softmax cross entropy ----

// G of a piece takes at most this much memory.  (8192 tokens of 50257 x 768 in bf16
// take 0.8 GB for all of it; by two pieces half of the logits are computed twice.)
constexpr int64_t kPieceBytes = int64_t(1) << 30;
constexpr int kMaxSplits = 128;

// How the second pass is cut: pieces of the vocabulary, and parts of a piece's
// columns that dh is summed over side by side.  Estimated microseconds decide,
// from how many turns the 256 CUs take over a product's tiles (two tiles of 128 fit
// a CU, one of 256), what a step of 64 columns of k costs a tile, and what adding
// to dh's fp32 parts moves at 4 TB/s.
void cut(dsm::CePlan* q, int64_t T, int64_t D, int64_t V) {
    const int64_t square = q->tile == 256 ? 256 : 128, width = q->form == dsm::kCeHalf ? 1 : 2;
    const double slots = square == 256 ? 256 : 512;
    double step = square == 256 ? 0.62 : 0.38;
    if (q->form != dsm::kCeHalf) step *= q->form == dsm::kCeBf16 ? 2.0 : 3.0;
    const auto tiles = [](int64_t n, int64_t of) { return (n + of - 1) / of; };
    const auto turns = [&](int64_t n) { return std::ceil(static_cast<double>(n) / slots); };
    const double dh_pass = 4e-6 * static_cast<double>(T * D) / 4.0;  // a read or write of one part
    const int64_t all = tiles(V, square), t = tiles(T, q->tile), d = tiles(D, square);
    const int64_t most = std::max<int64_t>(kPieceBytes / (T * 2 * width) / square, 1);
    const int64_t fewest = tiles(all, most);
    double best = 0.0;
    for (int64_t pieces = fewest; pieces <= std::min(all, fewest + 16); ++pieces) {
        const int64_t per = tiles(all, pieces), n = tiles(all, per);
        const double logits = turns(t * per) * (static_cast<double>(D) / 64 * step + 5.0);
        // dh and dw run side by side: the work over the CUs, and half a tile of the
        // longer kind for the uneven end.
        const double dw_tile = std::ceil(static_cast<double>(T) / 64) * step + 5.0;
        for (int s = 1; s <= kMaxSplits && (s == 1 || s * 256 <= per * square); ++s) {
            const double dh_tile = std::ceil(static_cast<double>(per * square) / 64 / s) * step + 5.0;
            const double work = (static_cast<double>(t * d * s) * dh_tile + static_cast<double>(per * d) * dw_tile) / slots;
            const double both = std::max(work, std::max(dh_tile, dw_tile)) + 0.5 * std::max(dh_tile, dw_tile) +
                                s * dh_pass * (n > 1 ? 2 : 1);
            // (The first piece's logits are there.)
            const double cost = static_cast<double>(n - 1) * logits + static_cast<double>(n) * (both + 6.0) + s * dh_pass;
            if (best == 0.0 || cost < best) {
                best = cost;
                q->piece = static_cast<int32_t>(per * square);
                q->dh_splits = s;
            }
        }
    }
    // Whether rows get a reference from a sample (linear_ce.hip), which takes a turn of
    // the logits' tiles (at least a 64th of the vocabulary) and saves reading and
    // writing G of the first piece at 5.8 TB/s.  8192 tokens of 50257 x 768 in bf16:
    // 1.96 ms with references and what they allow (dw, dh from operands transposed), 2.35
    // without; rows that all miss their reference 2.19 and 2.26.
    if (square == 256) {
        const int64_t n = std::max(std::max<int64_t>(256 / t, 1), tiles(V, 64 * 256));
        const double sample = turns(n * t) * (static_cast<double>(D) / 64 * step + 5.0) + 12.0;
        const double settle = static_cast<double>(T * q->piece * width) * 4.0 / 5.8e6;
        if (all / n >= 4 && sample < settle) {
            q->sample = static_cast<int32_t>(n);
            q->every = static_cast<int32_t>(all / n);
        }
    }
    q->ld_p = q->piece * (q->form == dsm::kCeHalves || q->form == dsm::kCeF32 ? 2 : 1);
}

dsm_status check_ce(const dsm_ce_problem* p) {
    if (!p) return invalid("problem is NULL");
    if (p->tokens < 0 || p->tokens > kMaxTokens) return invalid("tokens outside [0, 2^20]");
    if (p->dim < 1 || p->dim > kMaxDim) return invalid("dim outside [1, 2^16]");
    if (p->vocab < 1 || p->vocab > kMaxVocab) return invalid("vocab outside [1, 2^20]");
    if (p->dtype != DSM_F32 && p->dtype != DSM_BF16) return bad(DSM_ERR_INVALID_ARG, "unknown dtype %d", p->dtype);
    if (p->grads != 0 && p->grads != 1) return invalid("grads must be 0 or 1");
    return DSM_OK;
}

dsm::CePlan make_plan(const dsm_ce_problem* p) {
    dsm::CePlan q{};
    q.tokens = static_cast<int32_t>(p->tokens);
    q.dim = static_cast<int32_t>(p->dim);
    q.vocab = static_cast<int32_t>(p->vocab);
    q.grads = p->grads;
    const int64_t T = p->tokens, V = p->vocab;
    // Few tokens: the passes over w that make its fp16 form cost more than the matrix
    // cores lose without it.  Of 50257 x 768, in us, without those passes and with:
    // bf16 with gradients, 128 tokens 117 and 129, 160 tokens 163 and 152, 512 tokens
    // 327 and 231; fp32 with gradients, 64 tokens 235 and 250; fp32 losses alone, 128
    // tokens 124 and 148, 192 tokens 157 and 154, 256 tokens 210 and 156.
    if (p->dtype == DSM_F32)
        q.form = T <= (p->grads ? 64 : 128) ? dsm::kCeF32 : dsm::kCeHalves;
    else
        q.form = p->grads && T > 128 ? dsm::kCeHalf : dsm::kCeBf16;
    const int64_t width = p->dtype == DSM_F32 ? 2 : 1;
    const int64_t tokens_pad = round_up(T, 64);
    if (T <= 64 || q.form == dsm::kCeF32) {
        q.tile = T <= 32 ? 32 : 64;
    } else {
        // 256 where it takes the CUs no longer over the logits (a turn of two tiles of
        // 128 a CU takes 0.62 of a turn of one of 256): 1024 tokens of 4001 x 384 in
        // bf16 with gradients 79 us by 128, 111 us by 256; 8192 of 50257 x 768 by 256.
        const auto tiles = [&](int64_t of) { return ((T + of - 1) / of) * ((V + of - 1) / of); };
        const double t128 = 0.62 * std::ceil(static_cast<double>(tiles(128)) / 512);
        const double t256 = std::ceil(static_cast<double>(tiles(256)) / 256);
        q.tile = T > 128 && t256 <= t128 ? 256 : 128;
    }
    q.front = static_cast<int32_t>((V + 255) / 256);
    if (q.tile == 256 && !p->grads) {
        // Where the last turn of tiles of 256 leaves most CUs idle, its columns go by
        // tiles of 128 (0.62 of a turn as above, and a launch).  1024 tokens of 50257 x
        // 1600: 3.1 turns, 168 us in 4, 159 as 3 and 72 tiles of 128.
        const auto tiles = [](int64_t n, int64_t of) { return (n + of - 1) / of; };
        const int64_t t = tiles(T, 256), all = q.front, front = t * all / 256 * 256 / t;
        const int64_t rest = tiles(T, 128) * tiles(V - front * 256, 128);
        const double saved = static_cast<double>(tiles(t * all, 256) - tiles(t * front, 256)) -
                             0.62 * static_cast<double>(tiles(rest, 512));
        if (front > 0 && saved * (0.0016 * static_cast<double>(p->dim) + 0.5) > 0.4) q.front = static_cast<int32_t>(front);
    }
    const int64_t square = q.tile == 256 ? 256 : 128;
    q.ld_h = q.ld_w = round_up(p->dim, 64) * width;
    int64_t at = 0;
    auto take = [&](int64_t bytes) {
        const int64_t here = at;
        at = round_up(at + bytes, 256);
        return here;
    };
    q.scalars = take(dsm::kCeScalars);
    q.coef = take(T * 4);
    q.lse = take(T * 4);
    q.hit = take(T * 4);
    const int64_t behind = std::max<int64_t>(V - static_cast<int64_t>(q.front) * 256, 0);
    q.stats = take(((V + square - 1) / square + (behind + 127) / 128) * T * 8);
    q.h = take(tokens_pad * q.ld_h * 2);
    q.w = take(V * q.ld_w * 2);
    if (p->grads && T > 0) {
        cut(&q, T, p->dim, V);
        q.tops = take(T * (q.piece / square) * 4 * 4);  // four columns of waves a tile
        if (q.sample > 0) {
            q.refs = take(T * 4);
            q.rows = take(T * 8);
            q.ld_ht = tokens_pad * width;
            q.ht = take(p->dim * q.ld_ht * 2);
            if (q.form == dsm::kCeHalf) {
                q.ld_wt = round_up(V, 64);
                q.wt = take(p->dim * q.ld_wt * 2);
            }
        }
        // (In the bf16 form G is two arrays of halves.)
        q.p_lo = T * q.ld_p;
        q.p = take(T * q.ld_p * (q.form == dsm::kCeBf16 ? 4 : 2));
        q.ld_dh = round_up(p->dim, 4);
        q.dh = take(q.dh_splits * T * q.ld_dh * 4);
    }
    q.bytes = at;
    return q;
}

// ---- Orthogonalised updates ----

constexpr float kCoeffs[3] = {3.4445f, -4.7750f, 2.0315f};
// The matrices that one set of launches takes have at most this much workspace
// between them (one matrix may need more).
constexpr int64_t kGroupBytes = int64_t(4) << 30;

struct Iteration {
    float coeffs[3 * kMaxSteps];
    dsm::OrthoScales scales[kMaxSteps];
};

// The power of two that brings `bound` to at most 60000 (fp16 holds 65504).
int exponent_under(double bound) {
    int e = 0;
    std::frexp(60000.0 / std::max(bound, 1e-6), &e);
    return std::min(e - 1, 15);
}

// Bounds of |X|, |A| and |B| in each iteration from the singular values' range:
// they start in [0, 1] (divided by the Frobenius norm), and go through
// s -> |a s + b s^3 + c s^5|; A has s^2, B has b s^2 + c s^4.  1% covers rounding.
dsm_status plan_iteration(const dsm_ortho_problem* p, Iteration* it) {
    double r = 1.01;
    for (int k = 0; k < p->steps; ++k) {
        double f[3];
        for (int j = 0; j < 3; ++j) {
            const float v = p->coeffs ? p->coeffs[3 * k + j] : kCoeffs[j];
            if (!std::isfinite(v)) return invalid("coeffs hold a number that is not finite");
            it->coeffs[3 * k + j] = v;
            f[j] = v;
        }
        const double a = f[0], b = f[1], c = f[2], l = r * r;
        double top_b = std::fabs(b * l + c * l * l);
        if (c != 0.0) {
            const double z = -b / (2 * c);
            if (z > 0 && z < l) top_b = std::max(top_b, std::fabs(b * z + c * z * z));
        }
        double next = std::fabs(a * r + b * r * l + c * r * l * l);
        auto extremum = [&](double z) {  // of s -> a s + b s^3 + c s^5 at s^2 = z
            if (z > 0 && z < l) next = std::max(next, std::fabs(std::sqrt(z) * (a + b * z + c * z * z)));
        };
        if (c != 0.0) {
            const double disc = 9 * b * b - 20 * a * c;
            if (disc >= 0) {
                extremum((-3 * b + std::sqrt(disc)) / (10 * c));
                extremum((-3 * b - std::sqrt(disc)) / (10 * c));
            }
        } else if (b != 0.0) {
            extremum(-a / (3 * b));
        }
        next *= 1.01;
        if (!(r <= 1024.0 && top_b <= 1048576.0 && next <= 1024.0))
            return bad(DSM_ERR_UNSUPPORTED, "coeffs: the iterates of step %d grow beyond 2^10", k);
        dsm::OrthoScales& s = it->scales[k];
        s.x = exponent_under(r);
        s.a = exponent_under(l);
        s.b = exponent_under(top_b * 1.01);
        s.growth = std::max(0, static_cast<int>(std::ceil(std::log2(1.01 * (std::fabs(a) + std::fabs(b) + std::fabs(c)) + 1e-30))));
        if (k > 0) it->scales[k - 1].x_next = s.x;
        s.x_next = 0;  // the last result as it is
        r = next;
    }
    return DSM_OK;
}

dsm_status check_ortho(const dsm_ortho_problem* p, Iteration* it) {
    if (!p) return invalid("problem is NULL");
    if (p->rows < 0 || p->rows > kMaxSide || p->cols < 0 || p->cols > kMaxSide)
        return invalid("rows or cols outside [0, 2^20]");
    if (std::min(p->rows, p->cols) > kMaxShort) return invalid("the smaller of rows and cols exceeds 2^14");
    if (p->row_stride < p->cols) return invalid("row_stride < cols");
    if (p->count < 0) return invalid("count < 0");
    if (p->dtype != DSM_F32 && p->dtype != DSM_BF16) return bad(DSM_ERR_INVALID_ARG, "unknown dtype %d", p->dtype);
    if (p->steps < 1 || p->steps > kMaxSteps) return invalid("steps outside [1, 32]");
    if (!std::isfinite(p->eps) || p->eps < 0) return invalid("eps must be finite and >= 0");
    return plan_iteration(p, it);
}

bool is_empty(const dsm_ortho_problem* p) { return p->rows == 0 || p->cols == 0 || p->count == 0; }

int group_size(const dsm_ortho_problem* p) {
    const int m = static_cast<int>(std::min(p->rows, p->cols)), n = static_cast<int>(std::max(p->rows, p->cols));
    const int64_t one = dsm::ortho_group_bytes(1, m, n, p->dtype == DSM_BF16);
    const int64_t fit = one == 0 ? dsm::kOrthoGroup : std::max<int64_t>(1, kGroupBytes / one);
    return static_cast<int>(std::min<int64_t>(std::min<int64_t>(fit, p->count), dsm::kOrthoGroup));
}

int64_t ortho_bytes(const dsm_ortho_problem* p) {
    if (is_empty(p)) return 0;
    const int m = static_cast<int>(std::min(p->rows, p->cols)), n = static_cast<int>(std::max(p->rows, p->cols));
    return dsm::ortho_group_bytes(group_size(p), m, n, p->dtype == DSM_BF16);
}

dsm_status run_ortho(const dsm_ortho_problem* p, const dsm_ortho_buffers* b, const dsm_ortho_hparams* hp,
                     const Iteration& it) {
    if (!p->offsets) return invalid("offsets is NULL");
    for (int i = 0; i < p->count; ++i)
        if (p->offsets[i] < 0) return bad(DSM_ERR_INVALID_ARG, "offsets[%d] < 0", i);
    const int64_t need = ortho_bytes(p);
    if (need > 0)
        if (dsm_status st = check_workspace(b->workspace, b->workspace_bytes, need)) return st;
    if (dsm_status st = check_device()) return st;
    const int group = group_size(p);
    dsm::OrthoGroup g{};
    g.m = static_cast<int32_t>(std::min(p->rows, p->cols));
    g.n = static_cast<int32_t>(std::max(p->rows, p->cols));
    g.tall = p->rows > p->cols;
    g.bf16 = p->dtype == DSM_BF16;
    g.row_stride = p->row_stride;
    g.workspace = b->workspace;
    g.in = b->in;
    g.out = b->out;
    g.eps = p->eps;
    g.scale = 1.0f;
    if (hp) {
        g.mom = b->m;
        g.x = b->x;
        g.mu = hp->mu;
        g.lr = hp->lr;
        g.scale = hp->scale;
        g.weight_decay = hp->weight_decay;
        g.nesterov = hp->nesterov;
    }
    const size_t four = p->dtype == DSM_F32 ? 16 : 8;
    bool vector = p->row_stride % 4 == 0 && aligned(g.in, four) && aligned(g.out, four) && aligned(g.mom, 16) &&
                  aligned(g.x, 16);
    for (int i = 0; i < p->count; ++i) vector = vector && p->offsets[i] % 4 == 0;
    g.vector = vector;
    for (int first = 0; first < p->count; first += group) {
        g.count = std::min(group, p->count - first);
        for (int i = 0; i < g.count; ++i) g.off.at[i] = p->offsets[first + i];
        const hipError_t e = dsm::launch_ortho(g, it.coeffs, it.scales, p->steps, static_cast<hipStream_t>(b->stream));
        if (e != hipSuccess) return launched("launching the orthogonalisation", e);
    }
    return DSM_OK;
}

}  // namespace

extern "C" {

dsm_status dsm_ce_workspace(const dsm_ce_problem* problem, int64_t* workspace_bytes) {
    if (dsm_status st = check_ce(problem)) return st;
    if (!workspace_bytes) return invalid("workspace_bytes is NULL");
    *workspace_bytes = make_plan(problem).bytes;
    return DSM_OK;
}

dsm_status dsm_linear_ce(const dsm_ce_problem* problem, const dsm_ce_buffers* buffers, int32_t mean) {
    if (dsm_status st = check_ce(problem)) return st;
    if (!buffers) return invalid("buffers is NULL");
    const dsm_ce_problem& p = *problem;
    const dsm_ce_buffers& b = *buffers;
    const size_t elem = p.dtype == DSM_F32 ? 4 : 2;
    if (!b.w || !b.total) return invalid("w or total is NULL");
    if (p.tokens > 0 && (!b.h || !b.target || !b.loss)) return invalid("h, target or loss is NULL");
    if (p.grads && (!b.dw || (p.tokens > 0 && !b.dh))) return invalid("dh or dw is NULL");
    if ((p.tokens > 0 && b.h_stride < p.dim) || b.w_stride < p.dim) return invalid("h_stride or w_stride < dim");
    if (p.grads && ((p.tokens > 0 && b.dh_stride < p.dim) || b.dw_stride < p.dim)) return invalid("dh_stride or dw_stride < dim");
    if (!aligned(b.h, elem) || !aligned(b.w, elem) || !aligned(b.dh, elem) || !aligned(b.dw, elem))
        return invalid("h, w, dh or dw is not aligned to its elements");
    if (!aligned(b.target, 8) || !aligned(b.weight, 4) || !aligned(b.total, 4) || !aligned(b.loss, 4) ||
        !aligned(b.lse, 4))
        return invalid("target, weight, total, loss or lse is not aligned to its elements");
    const dsm::CePlan plan = make_plan(problem);
    if (dsm_status st = check_workspace(b.workspace, b.workspace_bytes, plan.bytes)) return st;
    if (dsm_status st = check_device()) return st;
    dsm::CeBuffers q{};
    q.h = b.h;
    q.w = b.w;
    q.target = b.target;
    q.weight = b.weight;
    q.total = b.total;
    q.loss = b.loss;
    q.lse = b.lse;
    q.dh = b.dh;
    q.dw = b.dw;
    q.h_stride = b.h_stride;
    q.w_stride = b.w_stride;
    q.dh_stride = b.dh_stride;
    q.dw_stride = b.dw_stride;
    q.workspace = static_cast<char*>(b.workspace);
    q.mean = mean != 0;
    // 16-byte loads of whole steps of 64 columns (fp32: 32), with 32-bit offsets
    // inside a tile.
    q.w_direct = (plan.form == dsm::kCeBf16 || plan.form == dsm::kCeF32) && p.dim % 64 == 0 &&
                 b.w_stride * elem % 16 == 0 && aligned(b.w, 16) && b.w_stride < (int64_t(1) << 22);
    // Without gradients nothing but a token's own loss meets its row of h, so rows
    // without a valid target need no zeros.
    q.h_direct = q.w_direct && !p.grads && b.h_stride * elem % 16 == 0 && aligned(b.h, 16) &&
                 b.h_stride < (int64_t(1) << 22);
    const size_t four = 4 * elem;
    q.h_vector = p.dim % 4 == 0 && b.h_stride % 4 == 0 && aligned(b.h, four);
    q.w_vector = p.dim % 4 == 0 && b.w_stride % 4 == 0 && aligned(b.w, four);
    q.dh_vector = p.dim % 4 == 0 && b.dh_stride % 4 == 0 && aligned(b.dh, four);
    q.dw_vector = p.dim % 4 == 0 && b.dw_stride % 4 == 0 && aligned(b.dw, four);
    return launched("launching the cross entropy", dsm::launch_linear_ce(plan, q, static_cast<hipStream_t>(b.stream)));
}

dsm_status dsm_ortho_workspace(const dsm_ortho_problem* problem, int64_t* workspace_bytes) {
    Iteration it;
    if (dsm_status st = check_ortho(problem, &it)) return st;
    if (!workspace_bytes) return invalid("workspace_bytes is NULL");
    *workspace_bytes = ortho_bytes(problem);
    return DSM_OK;
}

dsm_status dsm_orthogonalize(const dsm_ortho_problem* problem, const dsm_ortho_buffers* buffers) {
    Iteration it;
    if (dsm_status st = check_ortho(problem, &it)) return st;
    if (!buffers) return invalid("buffers is NULL");
    if (buffers->m || buffers->x) return invalid("m and x belong to dsm_ortho_step");
    if (is_empty(problem)) return DSM_OK;
    const size_t elem = problem->dtype == DSM_F32 ? 4 : 2;
    if (!buffers->in || !buffers->out) return invalid("in or out is NULL");
    if (!aligned(buffers->in, elem) || !aligned(buffers->out, elem))
        return invalid("in or out is not aligned to its elements");
    return run_ortho(problem, buffers, nullptr, it);
}

dsm_status dsm_ortho_step(const dsm_ortho_problem* problem, const dsm_ortho_buffers* buffers,
                          const dsm_ortho_hparams* hp) {
    Iteration it;
    if (dsm_status st = check_ortho(problem, &it)) return st;
    if (!buffers) return invalid("buffers is NULL");
    if (!hp) return invalid("hparams is NULL");
    if (problem->dtype != DSM_F32) return invalid("dsm_ortho_step takes fp32 buffers");
    if (!std::isfinite(hp->mu) || hp->mu < 0 || hp->mu > 1) return invalid("mu outside [0, 1]");
    if (!std::isfinite(hp->scale)) return invalid("scale is not finite");
    if (is_empty(problem)) return DSM_OK;
    if (!buffers->in) return invalid("in is NULL");
    if ((buffers->x != nullptr) == (buffers->out != nullptr)) return invalid("exactly one of x and out is wanted");
    if (buffers->x) {
        if (!std::isfinite(hp->lr) || hp->lr <= 0) return invalid("lr must be finite and > 0");
        if (!std::isfinite(hp->weight_decay) || hp->weight_decay < 0)
            return invalid("weight_decay must be finite and >= 0");
    }
    // The momentum is stored before the last read of `in`, and read after it.
    if (buffers->m && (buffers->m == buffers->in || buffers->m == buffers->out || buffers->m == buffers->x))
        return invalid("m is in, out or x");
    if (!aligned(buffers->in, 4) || !aligned(buffers->out, 4) || !aligned(buffers->m, 4) || !aligned(buffers->x, 4))
        return invalid("in, out, m or x is not aligned to its elements");
    return run_ortho(problem, buffers, hp, it);
}

}  // extern "C"
