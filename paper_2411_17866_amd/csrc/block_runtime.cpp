// Host runtime of the operators that a model's blocks and their gradients take
// (include/dsm.h): argument checks, plans and launches.  The runtime owns no memory of
// any kind; nothing here throws.
#include <algorithm>
#include <cmath>

#include "block_internal.h"
#include "dsm.h"
#include "runtime_checks.h"

namespace {

using dsm::aligned;
using dsm::bad;
using dsm::check_device;
using dsm::check_workspace;
using dsm::invalid;
using dsm::launched;
using dsm::round_up;

constexpr int64_t kMaxTokens = int64_t(1) << 20, kMaxSide = 1 << 16;
// Tiles' 32-bit offsets reach over rows that are at most this many elements apart.
constexpr int64_t kMaxStride = int64_t(1) << 22;

bool known_dtype(int32_t dtype) { return dtype == DSM_F32 || dtype == DSM_BF16; }

// ---- Linear layer ----

int64_t tiles(int64_t n, int64_t of) { return (n + of - 1) / of; }

// How products are cut is decided by estimated microseconds, of a turn of the CUs over
// tiles of 64 and 128 (two on a CU) and of 256 (one).  Measured over 14 shapes from 64 x 1600 x 6400
// to 8192 x 1600 x 6400 and every combination of tile and parts, the rules' choices take the least time
// or within 5% of it (fp32 4096 x 1600 x 6400).
constexpr int kTiles[3] = {64, 128, 256};
constexpr double kSlots[3] = {512, 512, 256};
constexpr int kMaxSplits = 16;

// A step of 64 of k for a turn that fills the CUs and for tiles that have one each, and what a turn takes
// besides: forward (bf16; both operands k-contiguous), and the gradients' products.
struct Turn {
    double full[3], alone[3], end[3], f32;
};
constexpr Turn kSingle = {{1.7, 0.0, 0.0}, {0.95, 0.0, 0.0}, {2.5, 0.0, 0.0}, 1.0};
constexpr Turn kForward = {{0.43, 0.97, 1.45}, {0.28, 0.55, 1.45}, {2.2, 5.0, 8.0}, 2.0};
constexpr Turn kBackward = {{0.50, 1.04, 1.66}, {0.58, 0.88, 1.26}, {3.0, 5.0, 10.0}, 2.42};
// Joining `parts` parts of n numbers: a launch, and what is moved.
double join_time(int parts, int64_t n, double each) {
    return parts > 1 ? 4.4 + each * 2e-6 * static_cast<double>(n * parts) : 0.0;
}

// fp32 products as they are up to this many tokens; microseconds as they are, and as halves.  Forward, 128 tokens:
// 4096 -> 4800 60 and 67, 1600 -> 6400 38.4 and 39.5, 768 -> 2304 13.5 and 18.5; 129, a third row of tiles: 90 and 75, 53
// and 43, 15.5 and 18.2; 192: 90 and 76, 63 and 44, 20 and 19.  Gradients, 33 tokens: 6400 -> 4800 124 and 137, 6400 -> 1600 58
// and 56, 768 -> 2304 21 and 26; 64: 126 and 152, 60 and 58, 21 and 27 (6400 -> 6400 173, library products 133).  More
// than 64 have no kernel of their own: 65 as halves 154, 59 and 30.
constexpr int64_t kSingleForward = 128, kSingleBackward = 64;
// bf16 gradients without tiles up to this many tokens: 1600 -> 6400 of 17 tokens 20.3 us and 25.4 by tiles, of 33
// 24.7 and 26.4, of 64 25.5 and 20.9; 768 -> 2304 of 32 10.1 and 13.8, of 64 12.3 and 11.4.
constexpr int64_t kFewBackward = 32;

// Tile columns: the last of 256 takes half as long where 128 columns of it lie past the end.
double columns(int64_t n, int of) {
    const int64_t all = tiles(n, of);
    return static_cast<double>(all) - (of == 256 && n <= (all - 1) * 256 + 128 ? 0.45 : 0.0);
}

// Forward: tiles, parts of k, and for tiles of 256 without parts how many of its columns
// they take (a tile of 128 that follows them has a CU for itself).  8192 x 1600 x 6400 in bf16: 159 us
// by 24 columns of 256 and 128 tiles of 128; 176 by 256 or 128 alone.
void cut_forward(dsm::LinearPlan* q) {
    const int64_t T = q->tokens, D = q->dim, N = q->wide, steps = tiles(D, 64);
    const bool single = q->form == dsm::kLinearSingle;
    const Turn& of = single ? kSingle : kForward;
    const double f32 = q->f32 ? of.f32 : 1.0;
    double best = 0.0;
    const auto take = [&](double cost, int tile, int splits, int64_t front) {
        if (best != 0.0 && cost >= best) return;
        best = cost;
        q->tile = tile;
        q->splits = splits;
        q->front = static_cast<int32_t>(front);
    };
    // Turns of n tiles of `i`, the last of which may leave CUs half filled.
    const auto turns = [&](int64_t n, int i, int64_t k) {
        const int64_t slots = static_cast<int64_t>(kSlots[i]), whole = n / slots, rest = n % slots;
        const double full = static_cast<double>(k) * of.full[i] * f32 + of.end[i];
        const double last = rest == 0 ? 0.0 : rest <= 256 ? static_cast<double>(k) * of.alone[i] * f32 + of.end[i] : full;
        return static_cast<double>(whole) * full + last;
    };
    for (int i = 0; i < (single ? 1 : 3); ++i) {
        const int64_t rows = tiles(T, kTiles[i]), all = tiles(N, kTiles[i]);
        for (int s = 1; s <= kMaxSplits && (s == 1 || s * 4 <= steps); ++s) {
            take(turns(rows * all * s, i, tiles(steps, s)) + join_time(s, T * N, 1.0), kTiles[i], s, all);
            if (kTiles[i] != 256 || s > 1) continue;
            const double turn = turns(1, 2, steps), alone = turns(1, 1, steps);
            for (int64_t front = all - 1; front >= std::max<int64_t>(all - 32, 1); --front) {
                // CUs that the last turn of 256 leaves idle take the first of the others.
                const int64_t last = rows * front % 256, idle = last > 0 ? 256 - last : 0;
                const int64_t rest = tiles(T, 128) * tiles(N - front * 256, 128) - idle * static_cast<int64_t>(turn / alone);
                take(turns(rows * front, 2, steps) + static_cast<double>(tiles(std::max<int64_t>(rest, 0), 256)) * alone, 256, 1, front);
            }
        }
    }
}

// Few tokens: parts of k, where few rows of w leave CUs idle.  A work-group reads its rows of
// w and x at some 75 GB/s, and joining the parts takes a launch.  One token of 6400 -> 256 in fp32: 15.2 us
// in one part, 8.7 in 4; 24 tokens of 6400 -> 1600 in bf16: 9.6, and 9.4 in 2.  In fp32 up to 32 tokens two
// work-groups a CU still gain: 1 token of 6400 -> 1600 17.1 us in 2 parts, 13.3 in 5; 55 tokens of 4096 -> 4096 28.1 and 37.1.
int few_splits(const dsm::LinearPlan& q) {
    const int64_t groups = tiles(q.wide, 16), size = q.f32 ? 4 : 2, rows = 16 + round_up(q.tokens, 16);
    const int64_t most = q.f32 && q.tokens <= 32 ? 512 : 256;
    const double whole = static_cast<double>(q.dim * size * rows) / 75e3;
    int best = 1;
    double least = whole - 1.5;
    for (int s = 2; s <= kMaxSplits && groups * s <= most && s * 1024 <= q.dim * size; ++s) {
        const double cost = whole / s + 3.4 + 0.5 * s;
        if (cost < least) {
            least = cost;
            best = s;
        }
    }
    return best;
}

// The gradients: dx and dw run side by side.  The work over the CUs, and a part of the longest tile
// for the uneven end.
// (Rows of one product by tiles of 128 behind tiles of 256, as forward, gained at most 2%: 4093 x 1600 x 6400.)
void cut_backward(dsm::LinearPlan* q) {
    const int64_t T = q->tokens, D = q->dim, N = q->wide;
    const double f32 = q->f32 ? kBackward.f32 : 1.0;
    double best = 0.0;
    if (q->back_few) {
        // dx by slabs of 64 columns, some 512 work-groups; parts of 256 rows of w at least.  (Past 32 tokens the CUs hold
        // no more at once: 64 of 6400 -> 6400 in fp32 dx 86 us by 500, 126 by 600; of 8 tokens 47 and 46.)
        const int64_t slabs = tiles(D, 64), parts = T > 32 ? 512 / slabs : tiles(512, slabs);
        q->dx_splits = static_cast<int32_t>(std::max<int64_t>(1, std::min<int64_t>({kMaxSplits, parts, N / 256})));
        return;
    }
    for (int i = 0; i < 3; ++i) {
        const int of = kTiles[i];
        const double dx = static_cast<double>(tiles(T, of)) * columns(D, of), dw = static_cast<double>(tiles(N, of)) * columns(D, of);
        const auto time = [&](int64_t k, const double* step) { return static_cast<double>(k) * step[i] * f32 + kBackward.end[i]; };
        const auto cost_of = [&](int sx, int sw) {
            const int64_t kx = tiles(tiles(N, 64), sx), kw = tiles(tiles(T, 64), sw) * (q->dz_halves ? 2 : 1);
            const double work = (dx * sx * time(kx, kBackward.full) + dw * sw * time(kw, kBackward.full)) / kSlots[i];
            const double longest = time(std::max(kx, kw), kBackward.alone);
            const double joins = join_time(sx, T * D, 0.25) + join_time(sw, N * D, 0.25) - (sx > 1 && sw > 1 ? 4.4 : 0.0);
            return std::max(work + 0.40 * longest, longest) + joins;
        };
        for (int sx = 1; sx <= kMaxSplits && (sx == 1 || sx * 256 <= N); ++sx)
            for (int sw = 1; sw <= kMaxSplits && (sw == 1 || sw * 256 <= T); ++sw) {
                const double cost = cost_of(sx, sw);
                if (best == 0.0 || cost < best) {
                    best = cost;
                    q->back_tile = of;
                    q->dx_splits = sx;
                    q->dw_splits = sw;
                }
            }
    }
}

dsm_status check_linear(const dsm_linear_problem* p) {
    if (!p) return invalid("problem is NULL");
    if (p->tokens < 0 || p->tokens > kMaxTokens) return invalid("tokens outside [0, 2^20]");
    if (p->dim < 1 || p->dim > kMaxSide) return invalid("dim outside [1, 2^16]");
    if (p->wide < 1 || p->wide > kMaxSide) return invalid("wide outside [1, 2^16]");
    if (!known_dtype(p->dtype)) return bad(DSM_ERR_INVALID_ARG, "unknown dtype %d", p->dtype);
    if (p->act < DSM_ACT_NONE || p->act > DSM_ACT_SILU) return bad(DSM_ERR_INVALID_ARG, "unknown act %d", p->act);
    if (p->dw_dtype != p->dtype && p->dw_dtype != DSM_F32) return invalid("dw_dtype is neither dtype nor fp32");
    if (p->grads != 0 && p->grads != 1) return invalid("grads must be 0 or 1");
    return DSM_OK;
}

dsm::LinearPlan make_linear_plan(const dsm_linear_problem* p) {
    dsm::LinearPlan q{};
    const int64_t T = p->tokens, D = p->dim, N = p->wide;
    q.tokens = static_cast<int32_t>(T);
    q.dim = static_cast<int32_t>(D);
    q.wide = static_cast<int32_t>(N);
    q.act = p->act;
    q.f32 = p->dtype == DSM_F32;
    q.dw_f32 = p->dw_dtype == DSM_F32;
    q.dz_halves = !q.f32 && q.dw_f32 && p->act != DSM_ACT_NONE;
    // fp32: halves take a pass over w that reads and writes it, fp32 products six times as long.
    q.form = !q.f32 ? dsm::kLinearBf16 : T <= kSingleForward ? dsm::kLinearSingle : dsm::kLinearHalves;
    q.back_form = !q.f32 ? dsm::kLinearBf16 : T <= kSingleBackward ? dsm::kLinearSingle : dsm::kLinearHalves;
    q.few = T <= dsm::kLinearFew;
    q.back_few = T <= (q.f32 ? kSingleBackward : kFewBackward);
    q.splits = q.dx_splits = q.dw_splits = 1;
    const int64_t width = q.f32 ? 2 : 1;  // 16-bit elements of a number
    q.ld_dim = round_up(D, 64) * width;
    q.ld_wide = round_up(N, 64) * width;
    q.pad_tokens = round_up(T, dsm::kDzRows);
    q.ld_y = round_up(N, 8);
    q.ld_dx = round_up(D, 8);
    int64_t at = 0;
    auto take = [&](int64_t bytes) {
        const int64_t here = at;
        at = round_up(at + bytes, 256);
        return here;
    };
    // Few tokens are read where they lie; of more, x and w may lie so that the tiles cannot.
    if (!q.few || (p->grads && !q.back_few)) {
        q.x = take((p->grads && q.dz_halves ? 2 * q.pad_tokens : T) * q.ld_dim * 2);
        q.w = take(N * q.ld_dim * 2);
    }
    const int64_t copies = at;
    const auto powers = [&] {
        q.x_exp = take(T * 4);
        q.w_exp = take(N * 4);
    };
    if (q.few) {
        at = 0;
        q.splits = few_splits(q);
    } else {
        cut_forward(&q);
    }
    if (q.form == dsm::kLinearHalves) powers();
    q.y_parts = take(q.splits > 1 ? q.splits * T * q.ld_y * 4 : 0);
    q.forward_bytes = at;
    if (!p->grads || T == 0) return q;
    at = q.back_few ? 0 : copies;
    cut_backward(&q);
    q.split_rows = T >= 1536 || N > 8192 ? 8 : 2;
    q.bias_parts = static_cast<int32_t>(q.back_form == dsm::kLinearHalves ? tiles(T, q.split_rows) : q.pad_tokens / dsm::kDzRows);
    if (q.back_form == dsm::kLinearHalves) {
        powers();
        q.z_exp = take(T * 4);
        q.w_tops = take(dsm::kLinearTopParts * 4);
        q.tops = take(q.pad_tokens / q.split_rows * 4);
    }
    // (Few tokens of bf16 without an activation: dz is dy, however it lies.)
    if (!q.back_few || q.f32 || p->act != DSM_ACT_NONE) q.dz = take(q.pad_tokens * q.ld_wide * (q.dz_halves ? 4 : 2));
    q.dx_parts = take(q.dx_splits > 1 ? q.dx_splits * T * q.ld_dx * 4 : 0);
    q.dw_parts = take(q.dw_splits > 1 ? q.dw_splits * N * q.ld_dx * 4 : 0);
    q.bias_sums = take(q.bias_parts * N * 4);
    q.backward_bytes = at;
    return q;
}

// A plan follows from the problem alone and takes some microseconds to weigh: each thread keeps
// the plans of the sizes that it asked for last.
const dsm::LinearPlan& plan_linear(const dsm_linear_problem* p) {
    constexpr int kKept = 16;
    static thread_local struct {
        dsm_linear_problem problem;
        dsm::LinearPlan plan;
        bool there;
    } kept[kKept];
    static thread_local int next = 0;
    const auto same = [&](const dsm_linear_problem& o) {
        return o.tokens == p->tokens && o.dim == p->dim && o.wide == p->wide && o.dtype == p->dtype && o.act == p->act &&
               o.dw_dtype == p->dw_dtype && o.grads == p->grads;
    };
    for (const auto& k : kept)
        if (k.there && same(k.problem)) return k.plan;
    auto& k = kept[next];
    next = (next + 1) % kKept;
    k.problem = *p;
    k.plan = make_linear_plan(p);
    k.there = true;
    return k.plan;
}

// Whether products can take a matrix's rows of `cols` elements where they lie: 16-byte
// loads of whole runs of `run` 16-bit elements.
bool direct(dsm::LinearForm form, const void* p, int64_t stride, int64_t cols, int64_t run) {
    if (form == dsm::kLinearHalves) return false;
    const int64_t size = form == dsm::kLinearSingle ? 4 : 2;
    return cols * size % (run * 2) == 0 && stride * size % 16 == 0 && stride * size < kMaxStride * 2 && aligned(p, 16);
}

dsm_status check_rows(const char* name, const void* p, int64_t rows, int64_t stride, int64_t cols, size_t elem, bool wanted) {
    if (!p) {
        if (wanted && rows > 0) return bad(DSM_ERR_INVALID_ARG, "%s is NULL", name);
        return DSM_OK;
    }
    if (rows > 1 && stride < cols) return bad(DSM_ERR_INVALID_ARG, "%s_stride < its columns", name);
    if (!aligned(p, elem)) return bad(DSM_ERR_INVALID_ARG, "%s is not aligned to its elements", name);
    return DSM_OK;
}

dsm::LinearCall linear_call(const dsm_linear_problem& p, const dsm_linear_buffers& b) {
    dsm::LinearCall c{};
    c.p = plan_linear(&p);
    c.x = b.x;
    c.w = b.w;
    c.x_stride = b.x_stride;
    c.w_stride = b.w_stride;
    c.z_stride = b.z_stride;
    c.workspace = static_cast<char*>(b.workspace);
    return c;
}

// ---- Norms ----

bool known_norm(int32_t kind) { return kind >= DSM_NORM_NONE && kind <= DSM_NORM_RMS; }

dsm_status check_norm(const dsm_norm_problem* p) {
    if (!p) return invalid("problem is NULL");
    if (p->tokens < 0 || p->tokens > (int64_t(1) << 30)) return invalid("tokens outside [0, 2^30]");
    if (p->dim < 1 || p->dim > dsm::kNormMaxDim) return invalid("dim outside [1, 8192]");
    if (!known_dtype(p->dtype)) return bad(DSM_ERR_INVALID_ARG, "unknown dtype %d", p->dtype);
    if (!known_norm(p->norm) || !known_norm(p->post)) return invalid("unknown norm or post");
    if (p->grads != 0 && p->grads != 1) return invalid("grads must be 0 or 1");
    if (!std::isfinite(p->eps) || p->eps < 0 || !std::isfinite(p->post_eps) || p->post_eps < 0)
        return invalid("eps and post_eps must be finite and >= 0");
    if (!std::isfinite(p->scale)) return invalid("scale is not finite");
    return DSM_OK;
}

int64_t norm_bytes(const dsm_norm_problem* p) {
    if (!p->grads) return 0;
    return round_up(static_cast<int64_t>(dsm::kNormSums) * dsm::norm_groups(p->tokens, p->dim) * p->dim * 4, 256);
}

dsm_status check_vectors(const dsm_norm_buffers& b) {
    const void* all[] = {b.weight, b.bias, b.gate, b.post_weight, b.post_bias, b.dweight, b.dbias, b.dgate, b.dpost_weight, b.dpost_bias};
    for (const void* v : all)
        if (!aligned(v, 4)) return invalid("a vector is not aligned to its elements");
    return DSM_OK;
}

dsm::NormCall norm_call(const dsm_norm_problem& p, const dsm_norm_buffers& b) {
    dsm::NormCall c{};
    c.tokens = static_cast<int32_t>(p.tokens);
    c.dim = static_cast<int32_t>(p.dim);
    c.f32 = p.dtype == DSM_F32;
    c.norm = p.norm;
    c.post = p.post;
    c.eps = p.eps;
    c.post_eps = p.post_eps;
    c.scale = p.scale;
    c.h = b.h;
    c.f = b.f;
    c.weight = b.weight;
    c.bias = b.bias;
    c.gate = b.gate;
    c.post_weight = b.post_weight;
    c.post_bias = b.post_bias;
    c.h_stride = b.h_stride;
    c.f_stride = b.f_stride;
    return c;
}

// ---- Clipping ----

dsm_status check_clip(const dsm_clip_tensor* t, int32_t n, int32_t groups, int64_t* chunks) {
    if (n < 0) return invalid("n_tensors < 0");
    if (n > 0 && !t) return invalid("tensors is NULL");
    if (groups < 1 || groups > dsm::kClipGroups) return invalid("n_groups outside [1, 256]");
    *chunks = 0;
    for (int i = 0; i < n; ++i) {
        if (t[i].first < 0 || t[i].numel < 0 || t[i].first > (int64_t(1) << 48) || t[i].numel > (int64_t(1) << 48))
            return bad(DSM_ERR_INVALID_ARG, "tensors[%d]: first or numel outside [0, 2^48]", i);
        if (t[i].block < 1 || t[i].stride < t[i].block)
            return bad(DSM_ERR_INVALID_ARG, "tensors[%d]: block < 1 or stride < block", i);
        if (!known_dtype(t[i].dtype)) return bad(DSM_ERR_INVALID_ARG, "tensors[%d]: unknown dtype %d", i, t[i].dtype);
        if (t[i].group < (i > 0 ? t[i - 1].group : 0) || t[i].group >= groups)
            return bad(DSM_ERR_INVALID_ARG, "tensors[%d]: group %d is out of order or range", i, t[i].group);
        *chunks += tiles(t[i].numel, dsm::kClipChunk);
        // (A launch's work-groups of 256 threads; 2^37 elements fill the memory.)
        if (*chunks > (int64_t(1) << 23)) return invalid("more elements than 2^37");
    }
    return DSM_OK;
}

int64_t clip_bytes(int64_t chunks) { return round_up(chunks * 8, 256) + dsm::kClipGroups * 8; }

bool contiguous(const dsm::ClipEntry& e) { return e.block >= e.first + e.numel; }

// Appends what follows entry e in memory, of its own kind, to it.
bool merged(dsm::ClipEntry* e, const dsm::ClipEntry& next) {
    if (e->group != next.group || e->bf16 != next.bf16) return false;
    const int64_t size = e->bf16 ? 2 : 4;
    if (contiguous(*e) && contiguous(next)) {
        if (static_cast<char*>(e->data) + (e->first + e->numel) * size != static_cast<char*>(next.data) + next.first * size)
            return false;
        e->numel += next.numel;
        e->block = e->stride = e->first + e->numel;
        return true;
    }
    if (e->data != next.data || e->block != next.block || e->stride != next.stride || e->first + e->numel != next.first) return false;
    e->numel += next.numel;
    return true;
}

// Fills the next launch's table from tensor *i on; tensors that follow each other in
// memory become one entry.  False where none is left.
bool next_table(const dsm_clip_tensor* tensors, int32_t n, int* i, dsm::ClipTable* table) {
    table->slot += table->chunks;
    table->count = table->chunks = 0;
    for (; *i < n; ++*i) {
        const dsm_clip_tensor& t = tensors[*i];
        if (t.numel == 0) continue;
        dsm::ClipEntry e{};
        e.data = t.data;
        e.first = t.first;
        e.numel = t.numel;
        e.block = t.block;
        e.stride = t.stride;
        e.group = static_cast<uint16_t>(t.group);
        e.bf16 = t.dtype == DSM_BF16;
        dsm::ClipEntry* last = table->count > 0 ? &table->e[table->count - 1] : nullptr;
        if (!last || !merged(last, e)) {
            if (table->count == dsm::kClipEntries) break;
            e.chunk = table->chunks;
            last = &table->e[table->count++];
            *last = e;
        }
        table->chunks = last->chunk + static_cast<int32_t>(tiles(last->numel, dsm::kClipChunk));
    }
    return table->count > 0;
}

}  // namespace

extern "C" {

dsm_status dsm_linear_workspace(const dsm_linear_problem* problem, int64_t* workspace_bytes) {
    if (dsm_status st = check_linear(problem)) return st;
    if (!workspace_bytes) return invalid("workspace_bytes is NULL");
    const dsm::LinearPlan& q = plan_linear(problem);
    *workspace_bytes = std::max(q.forward_bytes, q.backward_bytes);
    return DSM_OK;
}

dsm_status dsm_linear(const dsm_linear_problem* problem, const dsm_linear_buffers* buffers) {
    if (dsm_status st = check_linear(problem)) return st;
    if (!buffers) return invalid("buffers is NULL");
    const dsm_linear_problem& p = *problem;
    const dsm_linear_buffers& b = *buffers;
    const size_t elem = p.dtype == DSM_F32 ? 4 : 2;
    if (dsm_status st = check_rows("x", b.x, p.tokens, b.x_stride, p.dim, elem, true)) return st;
    if (dsm_status st = check_rows("w", b.w, p.wide, b.w_stride, p.dim, elem, true)) return st;
    if (dsm_status st = check_rows("residual", b.residual, p.tokens, b.residual_stride, p.wide, elem, false)) return st;
    if (dsm_status st = check_rows("y", b.y, p.tokens, b.y_stride, p.wide, elem, true)) return st;
    if (dsm_status st = check_rows("z", b.z, p.tokens, b.z_stride, p.wide, elem, false)) return st;
    if (!aligned(b.bias, 4)) return invalid("bias is not aligned to its elements");
    if (b.y && (b.y == b.x || b.y == b.w || b.y == b.z)) return invalid("y is x, w or z");
    if (b.z && (b.z == b.x || b.z == b.w || b.z == b.residual)) return invalid("z is x, w or residual");
    if (b.y && b.y == b.residual && p.tokens > 1 && b.y_stride != b.residual_stride)
        return invalid("y is the residual with another stride");
    if (p.tokens == 0) return DSM_OK;
    dsm::LinearCall c = linear_call(p, b);
    if (c.p.forward_bytes > 0)
        if (dsm_status st = check_workspace(b.workspace, b.workspace_bytes, c.p.forward_bytes)) return st;
    if (dsm_status st = check_device()) return st;
    c.residual = b.residual;
    c.residual_stride = b.residual_stride;
    c.bias = b.bias;
    c.y = b.y;
    c.y_stride = b.y_stride;
    c.z = b.z;
    c.x_direct = direct(c.p.form, b.x, b.x_stride, p.dim, 64);
    c.w_direct = direct(c.p.form, b.w, b.w_stride, p.dim, 64);
    return launched("launching the linear layer", dsm::launch_linear(c, static_cast<hipStream_t>(b.stream)));
}

dsm_status dsm_linear_backward(const dsm_linear_problem* problem, const dsm_linear_buffers* buffers) {
    if (dsm_status st = check_linear(problem)) return st;
    if (!problem->grads) return invalid("the problem is without gradients");
    if (!buffers) return invalid("buffers is NULL");
    const dsm_linear_problem& p = *problem;
    const dsm_linear_buffers& b = *buffers;
    const size_t elem = p.dtype == DSM_F32 ? 4 : 2, dw_elem = p.dw_dtype == DSM_F32 ? 4 : 2;
    const bool act = p.act != DSM_ACT_NONE;
    if (dsm_status st = check_rows("x", b.x, p.tokens, b.x_stride, p.dim, elem, b.dw != nullptr)) return st;
    if (dsm_status st = check_rows("w", b.w, p.wide, b.w_stride, p.dim, elem, b.dx != nullptr && p.tokens > 0)) return st;
    if (dsm_status st = check_rows("dy", b.dy, p.tokens, b.dy_stride, p.wide, elem, true)) return st;
    if (dsm_status st = check_rows("z", b.z, p.tokens, b.z_stride, p.wide, elem, act)) return st;
    if (dsm_status st = check_rows("dx", b.dx, p.tokens, b.dx_stride, p.dim, elem, false)) return st;
    if (dsm_status st = check_rows("dw", b.dw, p.wide, b.dw_stride, p.dim, dw_elem, false)) return st;
    if (!aligned(b.dbias, 4)) return invalid("dbias is not aligned to its elements");
    for (const void* out : {static_cast<const void*>(b.dx), static_cast<const void*>(b.dw)})
        if (out && (out == b.x || out == b.w || out == b.dy || out == b.z)) return invalid("dx or dw is x, w, dy or z");
    if (b.dx && b.dx == b.dw) return invalid("dx is dw");
    if (!b.dx && !b.dw && !b.dbias) return DSM_OK;
    dsm::LinearCall c = linear_call(p, b);
    if (c.p.backward_bytes > 0)
        if (dsm_status st = check_workspace(b.workspace, b.workspace_bytes, c.p.backward_bytes)) return st;
    if (dsm_status st = check_device()) return st;
    c.dy = b.dy;
    c.dy_stride = b.dy_stride;
    c.z_in = act ? b.z : nullptr;
    c.dx = b.dx;
    c.dx_stride = b.dx_stride;
    c.dw = b.dw;
    c.dw_stride = b.dw_stride;
    c.dbias = b.dbias;
    // k-strided operands: whole runs of 8.  dz is k-contiguous in dx, and its rows from
    // the last token on meet x's, so they have to be zeros.
    c.x_direct = !c.p.dz_halves && direct(c.p.back_form, b.x, b.x_stride, p.dim, 8);
    c.w_direct = direct(c.p.back_form, b.w, b.w_stride, p.dim, 8);
    // (Few tokens look for the ends of dz's rows themselves; in fp32 they take its copy.)
    c.dz_direct = !act && c.p.back_form == dsm::kLinearBf16 &&
                  (c.p.back_few || (direct(c.p.back_form, b.dy, b.dy_stride, p.wide, 64) && p.tokens % 64 == 0));
    return launched("launching the linear layer's gradients", dsm::launch_linear_backward(c, static_cast<hipStream_t>(b.stream)));
}

dsm_status dsm_norm_workspace(const dsm_norm_problem* problem, int64_t* workspace_bytes) {
    if (dsm_status st = check_norm(problem)) return st;
    if (!workspace_bytes) return invalid("workspace_bytes is NULL");
    *workspace_bytes = norm_bytes(problem);
    return DSM_OK;
}

dsm_status dsm_residual_norm(const dsm_norm_problem* problem, const dsm_norm_buffers* buffers) {
    if (dsm_status st = check_norm(problem)) return st;
    if (!buffers) return invalid("buffers is NULL");
    const dsm_norm_problem& p = *problem;
    const dsm_norm_buffers& b = *buffers;
    const size_t elem = p.dtype == DSM_F32 ? 4 : 2;
    if (dsm_status st = check_rows("h", b.h, p.tokens, b.h_stride, p.dim, elem, true)) return st;
    if (dsm_status st = check_rows("f", b.f, p.tokens, b.f_stride, p.dim, elem, p.post != DSM_NORM_NONE)) return st;
    if (dsm_status st = check_rows("s", b.s, p.tokens, b.s_stride, p.dim, elem, false)) return st;
    if (dsm_status st = check_rows("y", b.y, p.tokens, b.y_stride, p.dim, elem, p.norm != DSM_NORM_NONE)) return st;
    if (b.s && !b.f) return invalid("s without f is h");
    if (b.y && p.norm == DSM_NORM_NONE) return invalid("y without a norm");
    if (b.y && b.y == b.s) return invalid("y is s");
    if (dsm_status st = check_vectors(b)) return st;
    const struct { const void* out; int64_t stride; } outs[] = {{b.s, b.s_stride}, {b.y, b.y_stride}};
    for (const auto& o : outs)
        if (o.out && p.tokens > 1 && ((o.out == b.h && o.stride != b.h_stride) || (o.out == b.f && o.stride != b.f_stride)))
            return invalid("an output in place of an input has another stride");
    if (p.tokens == 0 || (!b.s && !b.y)) return DSM_OK;
    if (dsm_status st = check_device()) return st;
    dsm::NormCall c = norm_call(p, b);
    c.s = b.s;
    c.s_stride = b.s_stride;
    c.y = b.y;
    c.y_stride = b.y_stride;
    return launched("launching the norm", dsm::launch_norm(c, static_cast<hipStream_t>(b.stream)));
}

dsm_status dsm_residual_norm_backward(const dsm_norm_problem* problem, const dsm_norm_buffers* buffers) {
    if (dsm_status st = check_norm(problem)) return st;
    if (!problem->grads) return invalid("the problem is without gradients");
    if (!buffers) return invalid("buffers is NULL");
    const dsm_norm_problem& p = *problem;
    const dsm_norm_buffers& b = *buffers;
    const size_t elem = p.dtype == DSM_F32 ? 4 : 2;
    const bool normed = p.norm != DSM_NORM_NONE, posted = p.post != DSM_NORM_NONE;
    const bool needs_f = b.dgate || b.dpost_weight || b.dpost_bias || (posted && b.df);
    if (dsm_status st = check_rows("h", b.h, p.tokens, b.h_stride, p.dim, elem, normed)) return st;
    if (dsm_status st = check_rows("dy", b.dy, p.tokens, b.dy_stride, p.dim, elem, normed)) return st;
    if (dsm_status st = check_rows("ds", b.ds, p.tokens, b.ds_stride, p.dim, elem, !normed)) return st;
    if (dsm_status st = check_rows("f", b.f, p.tokens, b.f_stride, p.dim, elem, needs_f)) return st;
    if (dsm_status st = check_rows("dh", b.dh, p.tokens, b.dh_stride, p.dim, elem, false)) return st;
    if (dsm_status st = check_rows("df", b.df, p.tokens, b.df_stride, p.dim, elem, false)) return st;
    if (!normed && (b.dy || b.dweight || b.dbias)) return invalid("dy, dweight or dbias without a norm");
    if (!posted && (b.dpost_weight || b.dpost_bias)) return invalid("dpost_weight or dpost_bias without a post norm");
    if (b.dh && b.dh == b.df) return invalid("dh is df");
    if (b.dh && b.f && b.dh == b.f) return invalid("dh is f");
    if (dsm_status st = check_vectors(b)) return st;
    const struct { const void* out; int64_t stride; } outs[] = {{b.dh, b.dh_stride}, {b.df, b.df_stride}};
    const struct { const void* in; int64_t stride; } ins[] = {{b.h, b.h_stride}, {b.f, b.f_stride}, {b.dy, b.dy_stride}, {b.ds, b.ds_stride}};
    for (const auto& o : outs)
        for (const auto& i : ins)
            if (o.out && p.tokens > 1 && o.out == i.in && o.stride != i.stride)
                return invalid("an output in place of an input has another stride");
    float* const sums[dsm::kNormSums] = {b.dweight, b.dbias, b.dgate, b.dpost_weight, b.dpost_bias};
    bool any = false;
    for (int i = 0; i < dsm::kNormSums; ++i) {
        any = any || sums[i];
        for (int k = 0; k < i; ++k)
            if (sums[i] && sums[i] == sums[k]) return invalid("two vectors' gradients are one array");
    }
    if (!any && (p.tokens == 0 || (!b.dh && !b.df))) return DSM_OK;
    dsm::NormCall c = norm_call(p, b);
    if (any && norm_bytes(problem) > 0)
        if (dsm_status st = check_workspace(b.workspace, b.workspace_bytes, norm_bytes(problem))) return st;
    if (dsm_status st = check_device()) return st;
    // (f's own gradient without post, gate's gradients or post's needs no f.)
    if (!needs_f) c.f = nullptr;
    c.dy = b.dy;
    c.dy_stride = b.dy_stride;
    c.ds = b.ds;
    c.ds_stride = b.ds_stride;
    c.dh = b.dh;
    c.dh_stride = b.dh_stride;
    c.df = b.df;
    c.df_stride = b.df_stride;
    std::copy(sums, sums + dsm::kNormSums, c.sums);
    c.parts = static_cast<float*>(b.workspace);
    c.groups = dsm::norm_groups(p.tokens, p.dim);
    return launched("launching the norm's gradients", dsm::launch_norm_backward(c, static_cast<hipStream_t>(b.stream)));
}

dsm_status dsm_clip_workspace(const dsm_clip_tensor* tensors, int32_t n_tensors, int32_t n_groups, int64_t* workspace_bytes) {
    int64_t chunks = 0;
    if (dsm_status st = check_clip(tensors, n_tensors, n_groups, &chunks)) return st;
    if (!workspace_bytes) return invalid("workspace_bytes is NULL");
    *workspace_bytes = clip_bytes(chunks);
    return DSM_OK;
}

dsm_status dsm_grad_clip(const dsm_clip_tensor* tensors, int32_t n_tensors, int32_t n_groups, float max_norm, float eps,
                         float* norm, void* workspace, int64_t workspace_bytes, void* stream) {
    int64_t chunks = 0;
    if (dsm_status st = check_clip(tensors, n_tensors, n_groups, &chunks)) return st;
    if (!(max_norm >= 0)) return invalid("max_norm must be >= 0");
    if (!std::isfinite(eps) || eps < 0) return invalid("eps must be finite and >= 0");
    if (!norm) return invalid("norm is NULL");
    if (!aligned(norm, 4)) return invalid("norm is not aligned to its elements");
    for (int i = 0; i < n_tensors; ++i) {
        if (tensors[i].numel == 0) continue;
        if (!tensors[i].data) return bad(DSM_ERR_INVALID_ARG, "tensors[%d]: data is NULL", i);
        if (!aligned(tensors[i].data, tensors[i].dtype == DSM_F32 ? 4 : 2))
            return bad(DSM_ERR_INVALID_ARG, "tensors[%d]: data is not aligned to its elements", i);
    }
    if (dsm_status st = check_workspace(workspace, workspace_bytes, clip_bytes(chunks))) return st;
    if (dsm_status st = check_device()) return st;
    const auto s = static_cast<hipStream_t>(stream);
    double* parts = static_cast<double*>(workspace);
    double* factor = reinterpret_cast<double*>(static_cast<char*>(workspace) + round_up(chunks * 8, 256));
    dsm::ClipGroups groups;
    groups.count = n_groups;
    groups.max_norm = max_norm;
    groups.eps = eps;
    // Where the groups' chunks start, and the launches' tables once more for each pass.
    dsm::ClipTable table;
    const auto each = [&](auto use) {
        table.slot = table.chunks = 0;
        for (int i = 0; next_table(tensors, n_tensors, &i, &table);)
            if (const hipError_t e = use()) return e;
        return hipSuccess;
    };
    int64_t counts[dsm::kClipGroups] = {}, bytes = 0;
    int launches = 0;
    (void)each([&] {
        for (int k = 0; k < table.count; ++k) {
            counts[table.e[k].group] += tiles(table.e[k].numel, dsm::kClipChunk);
            bytes += table.e[k].numel * (table.e[k].bf16 ? 2 : 4);
        }
        ++launches;
        return hipSuccess;
    });
    groups.start[0] = 0;
    for (int g = 0; g < n_groups; ++g) groups.start[g + 1] = groups.start[g] + counts[g];
    if (const hipError_t e = each([&] { return dsm::launch_clip_squares(table, bytes, parts, s); })) return launched("launching the norms", e);
    const bool scales = max_norm < INFINITY;
    if (scales && launches == 1 && n_groups <= dsm::kClipFewGroups && groups.start[n_groups] <= dsm::kClipFewChunks) {
        dsm::ClipFew few;
        few.count = n_groups;
        few.max_norm = max_norm;
        few.eps = eps;
        for (int g = 0; g <= n_groups; ++g) few.start[g] = static_cast<int32_t>(groups.start[g]);
        return launched("launching the clipping", each([&] { return dsm::launch_clip_rest(table, few, parts, norm, s); }));
    }
    if (const hipError_t e = dsm::launch_clip_norms(groups, parts, norm, factor, s)) return launched("launching the norms", e);
    if (!scales) return DSM_OK;
    return launched("launching the clipping", each([&] { return dsm::launch_clip_scale(table, factor, s); }));
}

}  // extern "C"
