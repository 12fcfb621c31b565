// C ABI of the library: argument validation, workspace carving and the launch sequence of each
// entry point.  Host code only; every arithmetic step runs in the kernels of this directory.
#include <algorithm>
#include <cfloat>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <cstring>
#include <map>
#include <mutex>
#include <string>
#include <type_traits>
#include <vector>

#include "../../include/fvar.h"
#include "common.h"

using fvar::DType;

thread_local fvar::LaunchProbe *fvar::g_probe = nullptr;

// Scratch of fvar_score_select_static (the fp32 scores of one call): a fixed device array instead
// of caller workspace, so that the call needs no allocation anywhere.  Every GPU the library runs
// on holds its own copy; host code reaches it only through the per-device address below.
constexpr int kStaticScoreCap = 1 << 20;                       // floats: 4 MiB per device
static __device__ __align__(256) float scratch[kStaticScoreCap];
constexpr int kMaxDevices = 64;
static float *g_scratch_ptr[kMaxDevices];                      // resolved on a device's first call
static std::mutex g_scratch_mutex;

struct fvar_ctx {
    fvar_config cfg;
    std::vector<int32_t> scale_hw;
    float eps, scale;
    char err[256];
    bool debug_checks = false;
    // per-kernel timing
    bool profiling = false;
    struct Rec { std::string label; hipEvent_t a, b; };
    std::vector<Rec> recs;
    std::vector<hipEvent_t> pool;
};

namespace fvar {

// Whether two sets of rows have a byte in common: `rows` of them, `width` bytes of every `ld`, from a and b on.
bool rows_share_memory(size_t a, long width_a, long ld_a, long rows_a, size_t b, long width_b, long ld_b, long rows_b)
{
    if (a >= b + (size_t)((rows_b - 1) * ld_b + width_b) || b >= a + (size_t)((rows_a - 1) * ld_a + width_a)) return false;
    const long d = (long)(b - a);                            // row i of a is [i ld_a, + width_a), row j of b [d + j ld_b, + width_b)
    auto down = [](long x, long y) { return x >= 0 ? x / y : -((-x + y - 1) / y); };
    if (ld_a == ld_b) {
        // their distance is d + k ld, k = j - i, of which the largest below width_a counts, and the smaller ones that still reach the row
        const long last = std::min(down(width_a - 1 - d, ld_a), rows_b - 1);
        return last > -rows_a && d + last * ld_a > -width_b;
    }
    for (long i = std::max(0l, down(d - width_a, ld_a)); i < rows_a && i * ld_a < d + (rows_b - 1) * ld_b + width_b; ++i) {
        const long j = std::min(down(i * ld_a + width_a - 1 - d, ld_b), rows_b - 1);
        if (j >= 0 && d + j * ld_b + width_b > i * ld_a) return true;
    }
    return false;
}

}  // namespace fvar

namespace {

size_t align256(size_t v) { return (v + 255) & ~(size_t)255; }
size_t esize(const fvar_ctx *c) { return c->cfg.dtype == FVAR_BF16 ? 2 : 4; }
DType dtype(const fvar_ctx *c) { return c->cfg.dtype == FVAR_BF16 ? DType::BF16 : DType::F32; }
bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

fvar_status fail(fvar_ctx *c, fvar_status s, const char *fmt, ...)
{
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(c->err, sizeof(c->err), fmt, ap);
    va_end(ap);
    return s;
}

hipEvent_t get_event(fvar_ctx *c)
{
    if (!c->pool.empty()) {
        hipEvent_t e = c->pool.back();
        c->pool.pop_back();
        return e;
    }
    hipEvent_t e;
    (void)hipEventCreate(&e);
    return e;
}

// Runs `launch` (the kernels of one step) with their start/stop recorded in an event pair when
// profiling is on.
template <typename F>
void timed(fvar_ctx *c, hipStream_t st, const char *label, F &&launch)
{
    if (!c->profiling) { launch(); return; }
    fvar_ctx::Rec r{label, get_event(c), get_event(c)};
    fvar::LaunchProbe probe{r.a, r.b, false};
    fvar::g_probe = &probe;                   // the kernel launches inside record into it
    launch();
    fvar::g_probe = nullptr;
    (void)st;
    c->recs.push_back(r);
}

fvar_status launch_status(fvar_ctx *c, const char *what)
{
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return fail(c, FVAR_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
    c->err[0] = 0;
    return FVAR_OK;
}

constexpr size_t kCanaryBytes = 256;
constexpr unsigned char kCanaryByte = 0xA5;

// Debug checks: the index arrays are the caller's contract in normal operation; with the checks
// switched on they are brought to the host (which synchronises the stream) and verified:
// in range, strictly ascending per sample, and -- when both lists are given -- together exactly
// the set [0, M).
fvar_status validate_indices(fvar_ctx *c, hipStream_t st, const int32_t *idx_keep,
                             const int32_t *idx_drop, int B, int M, int k, const char *who)
{
    if (hipStreamSynchronize(st) != hipSuccess)
        return fail(c, FVAR_ERR_HIP, "%s: stream synchronisation failed in the index check", who);
    std::vector<int32_t> hk, hd;
    if (idx_keep && k > 0) {
        hk.resize((size_t)B * k);
        if (hipMemcpy(hk.data(), idx_keep, hk.size() * sizeof(int32_t), hipMemcpyDeviceToHost) != hipSuccess)
            return fail(c, FVAR_ERR_HIP, "%s: cannot read idx_keep", who);
    }
    if (idx_drop && k < M) {
        hd.resize((size_t)B * (M - k));
        if (hipMemcpy(hd.data(), idx_drop, hd.size() * sizeof(int32_t), hipMemcpyDeviceToHost) != hipSuccess)
            return fail(c, FVAR_ERR_HIP, "%s: cannot read idx_drop", who);
    }
    auto ascending = [&](const int32_t *v, int n, const char *name, int b) -> bool {
        for (int j = 0; j < n; ++j) {
            if (v[j] < 0 || v[j] >= M) {
                fail(c, FVAR_ERR_INVALID_ARG, "%s: %s[%d,%d] = %d is outside [0,%d)", who, name, b, j, v[j], M);
                return false;
            }
            if (j > 0 && v[j] <= v[j - 1]) {
                fail(c, FVAR_ERR_INVALID_ARG, "%s: %s[%d,:] is not strictly ascending at position %d", who,
                     name, b, j);
                return false;
            }
        }
        return true;
    };
    for (int b = 0; b < B; ++b) {
        const int32_t *kp = hk.empty() ? nullptr : hk.data() + (size_t)b * k;
        const int32_t *dp = hd.empty() ? nullptr : hd.data() + (size_t)b * (M - k);
        if (kp && !ascending(kp, k, "idx_keep", b)) return FVAR_ERR_INVALID_ARG;
        if (dp && !ascending(dp, M - k, "idx_drop", b)) return FVAR_ERR_INVALID_ARG;
        if (kp && dp) {
            // two ascending in-range lists of k and M-k entries partition [0,M) iff they share no entry
            int i = 0, j = 0;
            while (i < k && j < M - k) {
                if (kp[i] == dp[j])
                    return fail(c, FVAR_ERR_INVALID_ARG, "%s: token %d of sample %d is in idx_keep and idx_drop",
                                who, kp[i], b);
                if (kp[i] < dp[j]) ++i; else ++j;
            }
        }
    }
    return FVAR_OK;
}

struct BlockWs {
    char *x_keep, *u, *q, *att, *h1, *hid;
    char *k_new, *v_new;                      // new K / V rows on their way into a 4-bit or 8-bit cache
    float *part;                              // partial results of the attention and of each linear layer in turn
    fvar::GemmPlan qkv, o, fc1, fc2;          // how each linear layer runs at this row count
    size_t total;
};

// The cache that a block runs over, one of three kinds (the others are null); with 8 bits, what turns queries and keys (or null) and the rows'
// weights (or null).
struct BlockCache {
    const fvar_kv *kv = nullptr;
    const fvar_kvq *kvq = nullptr;
    const fvar_kvb *kvb = nullptr;
    const fvar_rope *rope = nullptr;
    const int32_t *pos = nullptr;
    float *weights = nullptr;
    int32_t add = 0;
};

BlockWs carve(const fvar_ctx *c, void *ws, int B, int rows, const BlockCache &q = {})
{
    const size_t es = esize(c), R = (size_t)B * rows, d = c->cfg.hidden, F = c->cfg.ffn_hidden;
    BlockWs w;
    char *p = static_cast<char *>(ws);
    size_t off = 0;
    auto take = [&](size_t bytes) { char *r = p ? p + off : nullptr; off += align256(bytes); return r; };
    w.x_keep = take(R * d * es);
    w.u = take(R * d * es);
    w.q = take(R * d * es);
    w.att = take(R * d * es);
    w.h1 = take(R * d * sizeof(float));       // intermediate residual stream, always fp32
    w.hid = take(R * F * es);
    const fvar::BlockPlan plan = fvar::block_plan(dtype(c), B, rows, c->cfg.hidden, c->cfg.heads, c->cfg.head_dim,
                                                  c->cfg.ffn_hidden);
    w.qkv = plan.layer[0]; w.o = plan.layer[1]; w.fc1 = plan.layer[2]; w.fc2 = plan.layer[3];
    size_t part = plan.floats;
    w.k_new = w.v_new = nullptr;
    if (q.kvq || q.kvb) {
        w.k_new = w.att;                      // both are read before their buffers are written
        w.v_new = w.h1;
        const size_t att = q.kvq ? fvar::kvq_attention_scratch_floats(dtype(c), B, rows, c->cfg.heads, q.kvq->kv_heads, c->cfg.head_dim,
                                                                      q.kvq->capacity)
                                 : fvar::kvb_attention_scratch_floats(dtype(c), B, rows, c->cfg.heads, q.kvb->kv_heads, c->cfg.head_dim,
                                                                      q.kvb->capacity, q.weights != nullptr);
        if (att > part) part = att;
    }
    w.part = part ? reinterpret_cast<float *>(take(part * sizeof(float))) : nullptr;
    w.total = off;
    return w;
}

// A 4-bit or 8-bit cache that a call with `rows` new rows per sample can work on (0: none are written).
template <typename Cache>
fvar_status check_cache(fvar_ctx *c, hipStream_t st, const Cache *kv, int B, int rows, const char *who)
{
    constexpr bool wide_scales = std::is_same<Cache, fvar_kvq>::value;   // read several at a time
    if (!kv) return fail(c, FVAR_ERR_INVALID_ARG, "%s: null cache", who);
    if (B < 1) return fail(c, FVAR_ERR_INVALID_ARG, "%s: need B>=1 (B=%d)", who, B);
    if (!kv->k || !kv->v || !kv->k_scale || !kv->v_scale)
        return fail(c, FVAR_ERR_INVALID_ARG, "%s: a pointer of the cache is NULL", who);
    if (!aligned16(kv->k) || !aligned16(kv->v) || (wide_scales && (!aligned16(kv->k_scale) || !aligned16(kv->v_scale))) ||
        (reinterpret_cast<uintptr_t>(kv->lens) & 3))
        return fail(c, FVAR_ERR_INVALID_ARG, "%s: pointer of the cache not aligned (16 bytes; lens 4)", who);
    if (kv->kv_heads < 1 || c->cfg.heads % kv->kv_heads)
        return fail(c, FVAR_ERR_INVALID_ARG, "%s: kv_heads=%d does not divide heads=%d", who, kv->kv_heads, c->cfg.heads);
    if (kv->capacity < 1) return fail(c, FVAR_ERR_INVALID_ARG, "%s: capacity=%d", who, kv->capacity);
    if (kv->capacity > (1 << 24) || (int64_t)B * kv->kv_heads > 65535)
        return fail(c, FVAR_ERR_UNSUPPORTED, "%s: capacity exceeds 2^24 or B*kv_heads 65535", who);
    if (!kv->lens && (kv->len < 0 || (int64_t)kv->len + rows > (int64_t)kv->capacity))
        return fail(c, FVAR_ERR_INVALID_ARG, "%s: cache too small (len=%d + rows=%d > capacity=%d)", who, kv->len, rows,
                    kv->capacity);
    if (!kv->lens || !c->debug_checks) return FVAR_OK;
    std::vector<int32_t> lens((size_t)B);
    if (hipStreamSynchronize(st) != hipSuccess ||
        hipMemcpy(lens.data(), kv->lens, lens.size() * sizeof(int32_t), hipMemcpyDeviceToHost) != hipSuccess)
        return fail(c, FVAR_ERR_HIP, "%s: cannot read lens", who);
    for (int b = 0; b < B; ++b)
        if (lens[b] < 0 || (int64_t)lens[b] + rows > (int64_t)kv->capacity)
            return fail(c, FVAR_ERR_INVALID_ARG, "%s: lens[%d] = %d with rows=%d is outside [0,%d]", who, b, lens[b], rows,
                        kv->capacity);
    return FVAR_OK;
}

fvar::KvbCache kvb_cache(const fvar_kvb *kv)
{
    return {(uint8_t *)kv->k, (uint8_t *)kv->v, (uint8_t *)kv->k_scale, (uint8_t *)kv->v_scale, kv->lens, kv->mask,
            kv->kv_heads, kv->capacity, kv->len};
}

fvar::KvqCache kvq_cache(const fvar_kvq *kv)
{
    return {(uint8_t *)kv->k, (uint8_t *)kv->v, (uint8_t *)kv->k_scale, (uint8_t *)kv->v_scale, kv->lens, kv->mask,
            kv->kv_heads, kv->capacity, kv->len};
}

// Elements from one row to the next: `ld`, or the row itself where it is 0; -1 where it is not one that can be read.
int row_pitch(const fvar_ctx *c, int ld, int row)
{
    const int chunk = c->cfg.dtype == FVAR_BF16 ? 8 : 4;
    if (ld == 0) return row;
    return ld < row || ld % chunk ? -1 : ld;
}

// Whether the sizes are some that workspace can be computed for: those that the calls accept.
template <typename Cache> bool cache_sizes(const fvar_ctx *c, const Cache *kv, int B, int n)
{
    return kv && B >= 1 && n >= 1 && kv->kv_heads >= 1 && c->cfg.heads % kv->kv_heads == 0 && kv->capacity >= 1 &&
           kv->capacity <= 1 << 24 && (int64_t)B * kv->kv_heads <= 65535 && (int64_t)B * n <= (1 << 25) / c->cfg.heads;
}

size_t kvq_attention_ws(const fvar_ctx *c, const fvar_kvq *kv, int B, int n)
{
    return align256(fvar::kvq_attention_scratch_floats(dtype(c), B, n, c->cfg.heads, kv->kv_heads, c->cfg.head_dim,
                                                       kv->capacity) * sizeof(float));
}

size_t kvb_attention_ws(const fvar_ctx *c, const fvar_kvb *kv, int B, int n, bool weights)
{
    return align256(fvar::kvb_attention_scratch_floats(dtype(c), B, n, c->cfg.heads, kv->kv_heads, c->cfg.head_dim, kv->capacity,
                                                       weights) * sizeof(float));
}

// 0, or a normal number of fp32
bool rope_magnitude(double m) { return m == 0.0 || (std::fabs(m) >= FLT_MIN && std::fabs(m) <= FLT_MAX); }

// Settings and positions that rows can be turned by.
fvar_status check_rope(fvar_ctx *c, const fvar_rope *r, const int32_t *pos, const char *who)
{
    if (!r || !pos) return fail(c, FVAR_ERR_INVALID_ARG, "%s: rope or pos is NULL", who);
    if (r->axes < 1 || r->axes > 2 || r->dim < 1 || r->dim > c->cfg.head_dim || r->dim % (16 * r->axes))
        return fail(c, FVAR_ERR_INVALID_ARG, "%s: dim=%d with axes=%d: a multiple of 16*axes up to head_dim is wanted", who, r->dim, r->axes);
    if (reinterpret_cast<uintptr_t>(pos) & 3) return fail(c, FVAR_ERR_INVALID_ARG, "%s: pos is not 4-byte aligned", who);
    bool some = false, finite = true;
    for (int i = 0; i < r->dim / r->axes / 2; ++i) {
        some |= r->turns[i] != 0.0;
        finite &= std::isfinite(r->turns[i]);
    }
    if (!some || !finite || !rope_magnitude(r->magnitude))
        return fail(c, FVAR_ERR_INVALID_ARG, "%s: rope has no turns (see fvar_rope_init), some that are not finite, or magnitude=%g", who, r->magnitude);
    return FVAR_OK;
}

fvar::RopeTable rope_table(const fvar_rope *r)
{
    fvar::RopeTable t;
    t.dim = r->dim;
    t.axes = r->axes;
    t.interleaved = r->interleaved != 0;
    t.magnitude = r->magnitude == 0.0 ? 1.f : (float)r->magnitude;
    for (int i = 0; i < 64; ++i) t.turns[i] = r->turns[i] - std::rint(r->turns[i]);   // exact; a position is a whole number, and so are its whole turns
    return t;
}

bool overlap(const void *a, size_t na, const void *b, size_t nb)
{
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return a && b && x < y + nb && y < x + na;
}

// The block on `rows` rows per sample, over one of three kinds of cache.
// idx == nullptr: rows are x's own rows (rows == M).
fvar_status block_forward(fvar_ctx *c, hipStream_t st, const fvar_block_weights *w, const void *x,
                          int B, int M, const int32_t *idx, int rows, const BlockCache &cache, void *y,
                          void *ws, size_t ws_bytes, const char *who)
{
    const fvar_kv *kv = cache.kv;
    const bool held = cache.kvq || cache.kvb;                // in 4 or 8 bits
    if (!w || !x || (!kv && !held) || !y) return fail(c, FVAR_ERR_INVALID_ARG, "%s: null argument", who);
    if (B < 1 || M < 1 || rows < 1 || rows > M)
        return fail(c, FVAR_ERR_INVALID_ARG, "%s: need B>=1 and 1<=rows<=M (B=%d M=%d rows=%d)", who, B,
                    M, rows);
    if (!idx && rows != M)
        return fail(c, FVAR_ERR_INVALID_ARG, "%s: idx_keep may be NULL only when k == M", who);
    if (!w->w_qkv || !w->w_o || !w->w_fc1 || !w->w_fc2)
        return fail(c, FVAR_ERR_INVALID_ARG, "%s: weight matrix pointer is NULL", who);
    if (held) {
        const fvar_status ks = cache.kvq ? check_cache(c, st, cache.kvq, B, rows, who) : check_cache(c, st, cache.kvb, B, rows, who);
        if (ks != FVAR_OK) return ks;
        const int kv_heads = cache.kvq ? cache.kvq->kv_heads : cache.kvb->kv_heads;
        if (kv_heads != c->cfg.heads)
            return fail(c, FVAR_ERR_UNSUPPORTED, "%s: kv_heads=%d, and the block has %d heads of keys", who, kv_heads,
                        c->cfg.heads);
        if ((int64_t)B * rows * c->cfg.heads > (1 << 25))
            return fail(c, FVAR_ERR_UNSUPPORTED, "%s: B*rows*heads exceeds 2^25", who);
    } else if (!kv->k || !kv->v || kv->len < 0 || kv->capacity < 1 ||
        (int64_t)kv->len + rows > (int64_t)kv->capacity)
        return fail(c, FVAR_ERR_INVALID_ARG, "%s: KV cache too small (len=%d + rows=%d > capacity=%d)",
                    who, kv->len, rows, kv->capacity);
    if (cache.rope || cache.pos) {
        const fvar_status rs = check_rope(c, cache.rope, cache.pos, who);
        if (rs != FVAR_OK) return rs;
    }
    if (!aligned16(cache.weights)) return fail(c, FVAR_ERR_INVALID_ARG, "%s: pointer not 16-byte aligned", who);
    const void *ptrs[] = {x, y, kv ? kv->k : nullptr, kv ? kv->v : nullptr, w->w_qkv, w->w_o, w->w_fc1, w->w_fc2, w->ln1_g, w->ln1_b,
                          w->ln2_g, w->ln2_b, w->b_qkv, w->b_o, w->b_fc1, w->b_fc2, ws};
    for (const void *p : ptrs)
        if (!aligned16(p)) return fail(c, FVAR_ERR_INVALID_ARG, "%s: pointer not 16-byte aligned", who);
    if ((int64_t)B * rows > (1 << 24))
        return fail(c, FVAR_ERR_UNSUPPORTED, "%s: B*rows exceeds 2^24", who);
    {
        // the linear-layer kernels address their operand tiles with 32-bit byte offsets from the
        // matrix base, and the attention grid carries (sample, key range) in blockIdx.z
        const int64_t wide = c->cfg.hidden > c->cfg.ffn_hidden ? c->cfg.hidden : c->cfg.ffn_hidden;
        const int64_t es = (int64_t)esize(c);
        if ((int64_t)B * rows * wide * es >= ((int64_t)1 << 32) ||
            (int64_t)3 * c->cfg.hidden * c->cfg.hidden * es >= ((int64_t)1 << 32) ||
            (int64_t)c->cfg.ffn_hidden * c->cfg.hidden * es >= ((int64_t)1 << 32))
            return fail(c, FVAR_ERR_UNSUPPORTED,
                        "%s: an operand matrix of B*rows=%lld rows reaches 4 GiB (32-bit tile offsets)",
                        who, (long long)B * rows);
        if ((int64_t)B * 8 > 65535 || c->cfg.heads > 65535)
            return fail(c, FVAR_ERR_UNSUPPORTED, "%s: B or heads exceeds the launch grid limits", who);
    }
    BlockWs s = carve(c, ws, B, rows, cache);
    const size_t ws_need = s.total + (c->debug_checks ? kCanaryBytes : 0);
    if (!ws || ws_bytes < ws_need)
        return fail(c, FVAR_ERR_WORKSPACE, "%s: workspace of %zu bytes needed, %zu given", who, ws_need,
                    ws_bytes);
    if (c->debug_checks) {
        if (idx) {
            const fvar_status vs = validate_indices(c, st, idx, nullptr, B, M, rows, who);
            if (vs != FVAR_OK) return vs;
        }
        // canary behind the carved workspace, verified after the kernels have finished
        if (hipMemsetAsync(static_cast<char *>(ws) + s.total, kCanaryByte, kCanaryBytes, st) != hipSuccess)
            return fail(c, FVAR_ERR_HIP, "%s: cannot write the workspace canary", who);
    }

    const DType dt = dtype(c);
    const int d = c->cfg.hidden, H = c->cfg.heads, Dh = c->cfg.head_dim, F = c->cfg.ffn_hidden;
    const int R = B * rows;

    bool launched = true;

    // gather (identity in the dense case) + LayerNorm 1; the dense case reads the residual from x
    const void *resid = idx ? (const void *)s.x_keep : x;
    timed(c, st, "gather_ln1", [&] {
        fvar::launch_gather_ln(dt, x, idx, B, M, rows, d, w->ln1_g, w->ln1_b, c->eps,
                               idx ? s.x_keep : nullptr, s.u, st);
    });
    // QKV projection; K and V rows land in the cache behind the valid prefix, or in the workspace to be quantised
    timed(c, st, "gemm_qkv", [&] {
        fvar::GemmEpilogue e;
        e.bias = w->b_qkv; e.out0 = s.q; e.ld0 = d; e.split = d;
        e.kcache = held ? s.k_new : kv->k; e.vcache = held ? s.v_new : kv->v; e.hd = d;
        e.cap = held ? rows : kv->capacity; e.len = held ? 0 : kv->len;
        e.rows_per_sample = rows;
        launched &= fvar::launch_gemm(dt, s.u, w->w_qkv, R, 3 * d, d, e, s.qkv, s.part, st);
    });
    if (cache.kvq) {
        timed(c, st, "kvq_append", [&] {
            fvar::launch_kvq_append(dt, s.k_new, s.v_new, d, kvq_cache(cache.kvq), B, rows, Dh, st);
        });
        timed(c, st, "kvq_attention", [&] {
            fvar::launch_kvq_attention(dt, s.q, d, kvq_cache(cache.kvq), rows, B, rows, H, Dh, c->scale, s.att, s.part, st);
        });
    } else if (cache.kvb) {
        if (cache.rope) {
            timed(c, st, "rope", [&] {
                fvar::launch_rope(dt, rope_table(cache.rope), {s.q, s.q, H, d, d}, {s.k_new, s.k_new, H, d, d}, cache.pos, R, Dh, st);
            });
        }
        timed(c, st, "kvb_append", [&] {
            fvar::launch_kvb_append(dt, s.k_new, s.v_new, d, kvb_cache(cache.kvb), B, rows, Dh, st);
        });
        timed(c, st, "kvb_attention", [&] {
            fvar::launch_kvb_attention(dt, s.q, d, kvb_cache(cache.kvb), rows, B, rows, H, Dh, c->scale, s.att, cache.weights,
                                       cache.add != 0, s.part, st);
        });
    } else {
        timed(c, st, "attention", [&] {
            fvar::launch_attention(dt, s.q, kv->k, kv->v, B, rows, kv->len + rows, kv->capacity, H, Dh, c->scale, s.att,
                                   s.part, st);
        });
    }
    timed(c, st, "gemm_o", [&] {
        fvar::GemmEpilogue e;
        e.bias = w->b_o; e.residual = resid; e.out0 = s.h1; e.ld0 = d; e.split = d;
        e.out_f32 = 1;
        launched &= fvar::launch_gemm(dt, s.att, w->w_o, R, d, d, e, s.o, s.part, st);
    });
    timed(c, st, "ln2", [&] {
        if (dt == DType::BF16)
            fvar::launch_ln_f32_to_bf16((const float *)s.h1, R, d, w->ln2_g, w->ln2_b, c->eps, s.u, st);
        else
            fvar::launch_gather_ln(dt, s.h1, nullptr, 1, R, R, d, w->ln2_g, w->ln2_b, c->eps, nullptr,
                                   s.u, st);
    });
    timed(c, st, "gemm_fc1", [&] {
        fvar::GemmEpilogue e;
        e.bias = w->b_fc1; e.gelu = 1; e.out0 = s.hid; e.ld0 = F; e.split = F;
        launched &= fvar::launch_gemm(dt, s.u, w->w_fc1, R, F, d, e, s.fc1, s.part, st);
    });
    timed(c, st, "gemm_fc2", [&] {
        fvar::GemmEpilogue e;
        e.bias = w->b_fc2; e.residual = s.h1; e.res_f32 = 1; e.out0 = y; e.ld0 = d; e.split = d;
        launched &= fvar::launch_gemm(dt, s.hid, w->w_fc2, R, d, F, e, s.fc2, s.part, st);
    });
    if (!launched) return fail(c, FVAR_ERR_UNSUPPORTED, "%s: a linear layer has no plan that can be launched", who);
    const fvar_status ls = launch_status(c, who);
    if (ls != FVAR_OK || !c->debug_checks) return ls;
    unsigned char canary[kCanaryBytes];
    if (hipStreamSynchronize(st) != hipSuccess ||
        hipMemcpy(canary, static_cast<char *>(ws) + s.total, kCanaryBytes, hipMemcpyDeviceToHost) != hipSuccess)
        return fail(c, FVAR_ERR_HIP, "%s: kernels failed (seen at the debug-check synchronisation)", who);
    for (size_t i = 0; i < kCanaryBytes; ++i)
        if (canary[i] != kCanaryByte)
            return fail(c, FVAR_ERR_WORKSPACE, "%s: a kernel wrote past the end of its workspace (canary byte %zu)",
                        who, i);
    return FVAR_OK;
}

}  // namespace

extern "C" {

const char *fvar_status_string(fvar_status s)
{
    switch (s) {
    case FVAR_OK: return "ok";
    case FVAR_ERR_INVALID_ARG: return "invalid argument";
    case FVAR_ERR_UNSUPPORTED: return "unsupported";
    case FVAR_ERR_WORKSPACE: return "workspace too small";
    case FVAR_ERR_HIP: return "HIP error";
    }
    return "unknown";
}

fvar_status fvar_create(const fvar_config *cfg, fvar_ctx **out)
{
    if (!cfg || !out) return FVAR_ERR_INVALID_ARG;
    *out = nullptr;
    if (cfg->hidden < 1 || cfg->heads < 1 || cfg->head_dim < 1 || cfg->ffn_hidden < 1 ||
        (int64_t)cfg->heads * cfg->head_dim != cfg->hidden)
        return FVAR_ERR_INVALID_ARG;
    if (cfg->dtype != FVAR_F32 && cfg->dtype != FVAR_BF16) return FVAR_ERR_INVALID_ARG;
    if (cfg->num_scales < 0 || (cfg->num_scales > 0 && !cfg->scale_hw)) return FVAR_ERR_INVALID_ARG;
    if (cfg->head_dim != 64 && cfg->head_dim != 128) return FVAR_ERR_UNSUPPORTED;
    // k-tiles of 64 in the GEMMs; one wavefront holds a whole row in the row kernels
    if (cfg->hidden % 64 || cfg->ffn_hidden % 64) return FVAR_ERR_UNSUPPORTED;
    const int max_hidden = cfg->dtype == FVAR_BF16 ? 8192 : 4096;
    if (cfg->hidden > max_hidden) return FVAR_ERR_UNSUPPORTED;
    for (int i = 0; i < 2 * cfg->num_scales; ++i)
        if (cfg->scale_hw[i] < 1) return FVAR_ERR_INVALID_ARG;
    fvar_ctx *c = new fvar_ctx();
    c->cfg = *cfg;
    c->scale_hw.assign(cfg->scale_hw, cfg->scale_hw + 2 * (size_t)cfg->num_scales);
    c->cfg.scale_hw = c->scale_hw.data();
    c->eps = cfg->ln_eps > 0.f ? cfg->ln_eps : 1e-6f;
    c->scale = cfg->attn_scale > 0.f ? cfg->attn_scale : 1.0f / sqrtf((float)cfg->head_dim);
    c->err[0] = 0;
    *out = c;
    return FVAR_OK;
}

void fvar_destroy(fvar_ctx *c)
{
    if (!c) return;
    for (auto &r : c->recs) { (void)hipEventDestroy(r.a); (void)hipEventDestroy(r.b); }
    for (auto e : c->pool) (void)hipEventDestroy(e);
    delete c;
}

const char *fvar_last_error(const fvar_ctx *c) { return c ? c->err : "null context"; }

int32_t fvar_keep_count(int32_t M, int32_t num, int32_t den)
{
    if (M < 1 || den < 1 || num < 0) return -1;
    int64_t k = ((int64_t)M * num + den - 1) / den;
    if (k < 1) k = 1;
    if (k > M) k = M;
    return (int32_t)k;
}

int32_t fvar_scale_tokens(const fvar_ctx *c, int32_t i)
{
    if (!c || i < 0 || i >= c->cfg.num_scales) return -1;
    return c->scale_hw[2 * i] * c->scale_hw[2 * i + 1];
}

int32_t fvar_scale_prev_len(const fvar_ctx *c, int32_t i)
{
    if (!c || i < 0 || i >= c->cfg.num_scales) return -1;
    int64_t s = 0;
    for (int j = 0; j < i; ++j) s += (int64_t)c->scale_hw[2 * j] * c->scale_hw[2 * j + 1];
    return s > INT32_MAX ? -1 : (int32_t)s;
}

size_t fvar_select_workspace_bytes(const fvar_ctx *c, int32_t B, int32_t M)
{
    if (!c || B < 1 || M < 1) return 0;
    return align256((size_t)B * M * sizeof(float));
}

size_t fvar_block_workspace_bytes(const fvar_ctx *c, int32_t B, int32_t rows)
{
    if (!c || B < 1 || rows < 1) return 0;
    return carve(c, nullptr, B, rows).total + (c->debug_checks ? kCanaryBytes : 0);
}

fvar_status fvar_debug_checks(fvar_ctx *c, int32_t on)
{
    if (!c) return FVAR_ERR_INVALID_ARG;
    c->debug_checks = on != 0;
    return FVAR_OK;
}

fvar_status fvar_score_select(fvar_ctx *c, fvar_stream stream, const void *x, int32_t B, int32_t M,
                              int32_t k, const float *scores_in, float *scores_out,
                              int32_t *idx_keep, int32_t *idx_drop, void *ws, size_t ws_bytes)
{
    if (!c) return FVAR_ERR_INVALID_ARG;
    const char *who = "fvar_score_select";
    if (B < 1 || M < 1 || k < 1 || k > M)
        return fail(c, FVAR_ERR_INVALID_ARG, "%s: need B>=1 and 1<=k<=M (B=%d M=%d k=%d)", who, B, M, k);
    if (M > (1 << 20) || (int64_t)B * M > (int64_t)INT32_MAX / 2)
        return fail(c, FVAR_ERR_UNSUPPORTED, "%s: M or B*M too large", who);
    if (!idx_keep) return fail(c, FVAR_ERR_INVALID_ARG, "%s: idx_keep is NULL", who);
    if (!x && !scores_in) return fail(c, FVAR_ERR_INVALID_ARG, "%s: x and scores_in both NULL", who);
    if (!aligned16(x) || !aligned16(ws))
        return fail(c, FVAR_ERR_INVALID_ARG, "%s: pointer not 16-byte aligned", who);
    hipStream_t st = static_cast<hipStream_t>(stream);
    const float *scores = scores_in;
    if (!scores_in) {
        float *buf = scores_out;
        if (!buf) {
            if (!ws || ws_bytes < fvar_select_workspace_bytes(c, B, M))
                return fail(c, FVAR_ERR_WORKSPACE, "%s: workspace of %zu bytes needed, %zu given", who,
                            fvar_select_workspace_bytes(c, B, M), ws_bytes);
            buf = static_cast<float *>(ws);
        }
        timed(c, st, "score", [&] { fvar::launch_scores(dtype(c), x, B * M, c->cfg.hidden, buf, st); });
        scores = buf;
    } else if (scores_out && scores_out != scores_in) {
        hipError_t e = hipMemcpyAsync(scores_out, scores_in, (size_t)B * M * sizeof(float),
                                      hipMemcpyDeviceToDevice, st);
        if (e != hipSuccess) return fail(c, FVAR_ERR_HIP, "%s: %s", who, hipGetErrorString(e));
    }
    timed(c, st, "select", [&] { fvar::launch_select(scores, B, M, k, idx_keep, idx_drop, st); });
    return launch_status(c, who);
}

fvar_status fvar_score_select_static(fvar_ctx *c, fvar_stream stream, const void *x, int32_t B,
                                     int32_t M, int32_t k, int32_t *idx_keep, int32_t *idx_drop)
{
    if (!c) return FVAR_ERR_INVALID_ARG;
    const char *who = "fvar_score_select_static";
    if (B < 1 || M < 1 || k < 1 || k > M)
        return fail(c, FVAR_ERR_INVALID_ARG, "%s: need B>=1 and 1<=k<=M (B=%d M=%d k=%d)", who, B, M, k);
    if ((int64_t)B * M > kStaticScoreCap)
        return fail(c, FVAR_ERR_UNSUPPORTED, "%s: B*M = %lld exceeds the built-in scratch of %d scores; use "
                    "fvar_score_select with a workspace", who, (long long)B * M, kStaticScoreCap);
    if (!x || !idx_keep) return fail(c, FVAR_ERR_INVALID_ARG, "%s: x or idx_keep is NULL", who);
    if (!aligned16(x)) return fail(c, FVAR_ERR_INVALID_ARG, "%s: pointer not 16-byte aligned", who);
    int dev = -1;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= kMaxDevices)
        return fail(c, FVAR_ERR_HIP, "%s: no usable current device", who);
    float *buf;
    {
        std::lock_guard<std::mutex> lock(g_scratch_mutex);
        if (!g_scratch_ptr[dev]) {
            // the array's name is only a host-side handle; this is its address on the current device
            float *p = nullptr;
            const hipError_t e = hipGetSymbolAddress(reinterpret_cast<void **>(&p), HIP_SYMBOL(scratch));
            if (e != hipSuccess || !p)
                return fail(c, FVAR_ERR_HIP, "%s: hipGetSymbolAddress: %s", who, hipGetErrorString(e));
            g_scratch_ptr[dev] = p;
        }
        buf = g_scratch_ptr[dev];
    }
    hipStream_t st = static_cast<hipStream_t>(stream);
    // every score of [0, B*M) is rewritten before the selection reads it: nothing to clear
    timed(c, st, "score", [&] { fvar::launch_scores(dtype(c), x, B * M, c->cfg.hidden, buf, st); });
    timed(c, st, "select", [&] { fvar::launch_select(buf, B, M, k, idx_keep, idx_drop, st); });
    return launch_status(c, who);
}

fvar_status fvar_block_forward_dense(fvar_ctx *c, fvar_stream stream, const fvar_block_weights *w,
                                     const void *x, int32_t B, int32_t M, const fvar_kv *kv, void *y,
                                     void *ws, size_t ws_bytes)
{
    if (!c) return FVAR_ERR_INVALID_ARG;
    BlockCache cache;
    cache.kv = kv;
    return block_forward(c, static_cast<hipStream_t>(stream), w, x, B, M, nullptr, M, cache, y, ws,
                         ws_bytes, "fvar_block_forward_dense");
}

fvar_status fvar_block_forward_pruned(fvar_ctx *c, fvar_stream stream, const fvar_block_weights *w,
                                      const void *x, int32_t B, int32_t M, const int32_t *idx_keep,
                                      int32_t k, const fvar_kv *kv, void *y_keep, void *ws,
                                      size_t ws_bytes)
{
    if (!c) return FVAR_ERR_INVALID_ARG;
    BlockCache cache;
    cache.kv = kv;
    return block_forward(c, static_cast<hipStream_t>(stream), w, x, B, M, idx_keep, k, cache, y_keep,
                         ws, ws_bytes, "fvar_block_forward_pruned");
}

fvar_status fvar_block_forward_dense_kvq(fvar_ctx *c, fvar_stream stream, const fvar_block_weights *w, const void *x,
                                         int32_t B, int32_t M, const fvar_kvq *kv, void *y, void *ws, size_t ws_bytes)
{
    if (!c) return FVAR_ERR_INVALID_ARG;
    BlockCache cache;
    cache.kvq = kv;
    return block_forward(c, static_cast<hipStream_t>(stream), w, x, B, M, nullptr, M, cache, y, ws, ws_bytes,
                         "fvar_block_forward_dense_kvq");
}

fvar_status fvar_block_forward_pruned_kvq(fvar_ctx *c, fvar_stream stream, const fvar_block_weights *w, const void *x,
                                          int32_t B, int32_t M, const int32_t *idx_keep, int32_t k, const fvar_kvq *kv,
                                          void *y_keep, void *ws, size_t ws_bytes)
{
    if (!c) return FVAR_ERR_INVALID_ARG;
    BlockCache cache;
    cache.kvq = kv;
    return block_forward(c, static_cast<hipStream_t>(stream), w, x, B, M, idx_keep, k, cache, y_keep, ws, ws_bytes,
                         "fvar_block_forward_pruned_kvq");
}

size_t fvar_block_kvq_workspace_bytes(const fvar_ctx *c, const fvar_kvq *kv, int32_t B, int32_t rows)
{
    if (!c || !cache_sizes(c, kv, B, rows)) return 0;
    BlockCache cache;
    cache.kvq = kv;
    return carve(c, nullptr, B, rows, cache).total + (c->debug_checks ? kCanaryBytes : 0);
}

size_t fvar_block_kvb_workspace_bytes(const fvar_ctx *c, const fvar_kvb *kv, int32_t B, int32_t rows, int32_t weights)
{
    if (!c || !cache_sizes(c, kv, B, rows)) return 0;
    float some;
    BlockCache cache;
    cache.kvb = kv;
    cache.weights = weights ? &some : nullptr;               // (only whether there are any)
    return carve(c, nullptr, B, rows, cache).total + (c->debug_checks ? kCanaryBytes : 0);
}

fvar_status fvar_block_forward_dense_kvb(fvar_ctx *c, fvar_stream stream, const fvar_block_weights *w, const void *x, int32_t B, int32_t M,
                                         const fvar_kvb *kv, const fvar_rope *rope, const int32_t *pos, float *weights, int32_t add, void *y,
                                         void *ws, size_t ws_bytes)
{
    if (!c) return FVAR_ERR_INVALID_ARG;
    BlockCache cache;
    cache.kvb = kv; cache.rope = rope; cache.pos = pos; cache.weights = weights; cache.add = add;
    return block_forward(c, static_cast<hipStream_t>(stream), w, x, B, M, nullptr, M, cache, y, ws, ws_bytes,
                         "fvar_block_forward_dense_kvb");
}

fvar_status fvar_block_forward_pruned_kvb(fvar_ctx *c, fvar_stream stream, const fvar_block_weights *w, const void *x, int32_t B, int32_t M,
                                          const int32_t *idx_keep, int32_t k, const fvar_kvb *kv, const fvar_rope *rope, const int32_t *pos,
                                          float *weights, int32_t add, void *y_keep, void *ws, size_t ws_bytes)
{
    if (!c) return FVAR_ERR_INVALID_ARG;
    BlockCache cache;
    cache.kvb = kv; cache.rope = rope; cache.pos = pos; cache.weights = weights; cache.add = add;
    return block_forward(c, static_cast<hipStream_t>(stream), w, x, B, M, idx_keep, k, cache, y_keep, ws, ws_bytes,
                         "fvar_block_forward_pruned_kvb");
}

fvar_status fvar_kvq_append(fvar_ctx *c, fvar_stream stream, const fvar_kvq *kv, const void *k, const void *v, int32_t ld,
                            int32_t B, int32_t rows)
{
    if (!c) return FVAR_ERR_INVALID_ARG;
    const char *who = "fvar_kvq_append";
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (rows < 1) return fail(c, FVAR_ERR_INVALID_ARG, "%s: need rows>=1 (rows=%d)", who, rows);
    const fvar_status ks = check_cache(c, st, kv, B, rows, who);
    if (ks != FVAR_OK) return ks;
    if (!k || !v) return fail(c, FVAR_ERR_INVALID_ARG, "%s: k or v is NULL", who);
    if (!aligned16(k) || !aligned16(v)) return fail(c, FVAR_ERR_INVALID_ARG, "%s: pointer not 16-byte aligned", who);
    if (rows > kv->capacity) return fail(c, FVAR_ERR_INVALID_ARG, "%s: rows=%d > capacity=%d", who, rows, kv->capacity);
    const int pitch = row_pitch(c, ld, kv->kv_heads * c->cfg.head_dim);
    if (pitch < 0)
        return fail(c, FVAR_ERR_INVALID_ARG, "%s: ld=%d is shorter than a row or no multiple of 16 bytes", who, ld);
    timed(c, st, "kvq_append", [&] {
        fvar::launch_kvq_append(dtype(c), k, v, pitch, kvq_cache(kv), B, rows, c->cfg.head_dim, st);
    });
    return launch_status(c, who);
}

fvar_status fvar_kvq_read(fvar_ctx *c, fvar_stream stream, const fvar_kvq *kv, int32_t B, int32_t first, int32_t rows,
                          void *k, void *v)
{
    if (!c) return FVAR_ERR_INVALID_ARG;
    const char *who = "fvar_kvq_read";
    hipStream_t st = static_cast<hipStream_t>(stream);
    const fvar_status ks = check_cache(c, st, kv, B, 0, who);
    if (ks != FVAR_OK) return ks;
    if (!k && !v) return fail(c, FVAR_ERR_INVALID_ARG, "%s: k and v both NULL", who);
    if (!aligned16(k) || !aligned16(v)) return fail(c, FVAR_ERR_INVALID_ARG, "%s: pointer not 16-byte aligned", who);
    if (rows < 1 || rows > kv->capacity || first < -kv->capacity || (int64_t)first + (first < 0 ? 0 : rows) > kv->capacity)
        return fail(c, FVAR_ERR_INVALID_ARG, "%s: rows [%d,+%d) are outside the capacity of %d", who, first, rows,
                    kv->capacity);
    timed(c, st, "kvq_read", [&] {
        fvar::launch_kvq_read(dtype(c), kvq_cache(kv), B, first, rows, c->cfg.head_dim, k, v, st);
    });
    return launch_status(c, who);
}

size_t fvar_kvq_attention_workspace_bytes(const fvar_ctx *c, const fvar_kvq *kv, int32_t B, int32_t n)
{
    if (!c || !cache_sizes(c, kv, B, n)) return 0;
    return kvq_attention_ws(c, kv, B, n);
}

fvar_status fvar_kvq_attention(fvar_ctx *c, fvar_stream stream, const void *q, int32_t ld, const fvar_kvq *kv, int32_t B,
                               int32_t n, void *o, void *ws, size_t ws_bytes)
{
    if (!c) return FVAR_ERR_INVALID_ARG;
    const char *who = "fvar_kvq_attention";
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (n < 1) return fail(c, FVAR_ERR_INVALID_ARG, "%s: need n>=1 (n=%d)", who, n);
    const fvar_status ks = check_cache(c, st, kv, B, 0, who);
    if (ks != FVAR_OK) return ks;
    if (!q || !o) return fail(c, FVAR_ERR_INVALID_ARG, "%s: q or o is NULL", who);
    if (!aligned16(q) || !aligned16(o) || !aligned16(ws))
        return fail(c, FVAR_ERR_INVALID_ARG, "%s: pointer not 16-byte aligned", who);
    const int pitch = row_pitch(c, ld, c->cfg.hidden);
    if (pitch < 0)
        return fail(c, FVAR_ERR_INVALID_ARG, "%s: ld=%d is shorter than a row or no multiple of 16 bytes", who, ld);
    if ((int64_t)B * n * c->cfg.heads > (1 << 25))
        return fail(c, FVAR_ERR_UNSUPPORTED, "%s: B*n*heads exceeds 2^25", who);
    const size_t need = kvq_attention_ws(c, kv, B, n);
    if (need && (!ws || ws_bytes < need))
        return fail(c, FVAR_ERR_WORKSPACE, "%s: workspace of %zu bytes needed, %zu given", who, need, ws_bytes);
    timed(c, st, "kvq_attention", [&] {
        fvar::launch_kvq_attention(dtype(c), q, pitch, kvq_cache(kv), 0, B, n, c->cfg.heads, c->cfg.head_dim, c->scale, o,
                                   (float *)ws, st);
    });
    return launch_status(c, who);
}

fvar_status fvar_rope_init(fvar_rope *r)
{
    if (!r || r->axes < 1 || r->axes > 2 || r->dim < 1 || r->dim > 128 || r->dim % (16 * r->axes)) return FVAR_ERR_INVALID_ARG;
    if (r->scaling < FVAR_ROPE_NONE || r->scaling > FVAR_ROPE_YARN || !(r->base > 1.0) || !std::isfinite(r->base) ||
        !rope_magnitude(r->magnitude))
        return FVAR_ERR_INVALID_ARG;
    if (r->scaling != FVAR_ROPE_NONE && (!(r->factor >= 1.0) || !std::isfinite(r->factor))) return FVAR_ERR_INVALID_ARG;
    if (r->scaling == FVAR_ROPE_YARN && (!(r->original > 0.0) || !(r->low < r->high) || !std::isfinite(r->original) ||
                                         !std::isfinite(r->low) || !std::isfinite(r->high)))
        return FVAR_ERR_INVALID_ARG;
    const double two_pi = 6.283185307179586476925;
    const int P = r->dim / r->axes;
    const double base = r->scaling == FVAR_ROPE_NTK ? r->base * std::pow(r->factor, (double)P / (P - 2)) : r->base;
    if (r->magnitude == 0.0) r->magnitude = 1.0;
    for (int i = 0; i < 64; ++i) {
        double f = i < P / 2 ? std::pow(base, -2.0 * i / P) : 0.0;
        if (r->scaling == FVAR_ROPE_LINEAR) f /= r->factor;
        if (r->scaling == FVAR_ROPE_YARN) {
            double g = (r->original * f / two_pi - r->low) / (r->high - r->low);
            g = g < 0.0 ? 0.0 : g > 1.0 ? 1.0 : g;
            f *= g + (1.0 - g) / r->factor;
        }
        r->turns[i] = f / two_pi;
    }
    return FVAR_OK;
}

fvar_status fvar_rope_apply(fvar_ctx *c, fvar_stream stream, const fvar_rope *r, const int32_t *pos, int32_t B, int32_t n,
                            int32_t kv_heads, const void *q, int32_t ld_q, const void *k, int32_t ld_k, void *q_out, int32_t ld_q_out,
                            void *k_out, int32_t ld_k_out)
{
    if (!c) return FVAR_ERR_INVALID_ARG;
    const char *who = "fvar_rope_apply";
    const fvar_status rs = check_rope(c, r, pos, who);
    if (rs != FVAR_OK) return rs;
    if (B < 1 || n < 1) return fail(c, FVAR_ERR_INVALID_ARG, "%s: need B>=1 and n>=1 (B=%d n=%d)", who, B, n);
    if ((int64_t)B * n > (1 << 24)) return fail(c, FVAR_ERR_UNSUPPORTED, "%s: B*n exceeds 2^24", who);
    if (!q && !k) return fail(c, FVAR_ERR_INVALID_ARG, "%s: q and k both NULL", who);
    if (!q != !q_out || !k != !k_out) return fail(c, FVAR_ERR_INVALID_ARG, "%s: an input without its output, or the reverse", who);
    if (kv_heads < 1 || c->cfg.heads % kv_heads)
        return fail(c, FVAR_ERR_INVALID_ARG, "%s: kv_heads=%d does not divide heads=%d", who, kv_heads, c->cfg.heads);
    if (!aligned16(q) || !aligned16(k) || !aligned16(q_out) || !aligned16(k_out))
        return fail(c, FVAR_ERR_INVALID_ARG, "%s: pointer not 16-byte aligned", who);
    const int wq = c->cfg.hidden, wk = kv_heads * c->cfg.head_dim;
    const fvar::RopeRows rows[2] = {{q, q_out, q ? c->cfg.heads : 0, row_pitch(c, ld_q, wq), row_pitch(c, ld_q_out, wq)},
                                    {k, k_out, k ? kv_heads : 0, row_pitch(c, ld_k, wk), row_pitch(c, ld_k_out, wk)}};
    for (const fvar::RopeRows &x : rows)
        if (x.in && (x.ld_in < 0 || x.ld_out < 0 || (x.in == x.out && x.ld_in != x.ld_out)))
            return fail(c, FVAR_ERR_INVALID_ARG, "%s: a row pitch is shorter than a row, no multiple of 16 bytes, or in place not the same", who);
    const long es = (long)esize(c), count = (long)B * n;
    auto meet = [&](const void *out, const fvar::RopeRows &x, const void *other, long width, long ld, long n_other) {
        return out && other && fvar::rows_share_memory((size_t)out, x.heads * c->cfg.head_dim * es, x.ld_out * es, count, (size_t)other, width, ld, n_other);
    };
    for (int i = 0; i < 2; ++i) {
        const fvar::RopeRows &x = rows[i], &y = rows[1 - i];
        const long wx = x.heads * c->cfg.head_dim * es, wy = y.heads * c->cfg.head_dim * es, wp = count * r->axes * (long)sizeof(int32_t);
        if ((x.out != x.in && meet(x.out, x, x.in, wx, x.ld_in * es, count)) || meet(x.out, x, y.in, wy, y.ld_in * es, count) ||
            meet(x.out, x, y.out, wy, y.ld_out * es, count) || meet(x.out, x, pos, wp, wp, 1))
            return fail(c, FVAR_ERR_INVALID_ARG, "%s: an output shares memory with another tensor", who);
    }
    hipStream_t st = static_cast<hipStream_t>(stream);
    timed(c, st, "rope", [&] { fvar::launch_rope(dtype(c), rope_table(r), rows[0], rows[1], pos, B * n, c->cfg.head_dim, st); });
    return launch_status(c, who);
}

fvar_status fvar_kvb_append(fvar_ctx *c, fvar_stream stream, const fvar_kvb *kv, const void *k, const void *v, int32_t ld,
                            int32_t B, int32_t rows)
{
    if (!c) return FVAR_ERR_INVALID_ARG;
    const char *who = "fvar_kvb_append";
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (rows < 1) return fail(c, FVAR_ERR_INVALID_ARG, "%s: need rows>=1 (rows=%d)", who, rows);
    const fvar_status ks = check_cache(c, st, kv, B, rows, who);
    if (ks != FVAR_OK) return ks;
    if (!k || !v) return fail(c, FVAR_ERR_INVALID_ARG, "%s: k or v is NULL", who);
    if (!aligned16(k) || !aligned16(v)) return fail(c, FVAR_ERR_INVALID_ARG, "%s: pointer not 16-byte aligned", who);
    if (rows > kv->capacity) return fail(c, FVAR_ERR_INVALID_ARG, "%s: rows=%d > capacity=%d", who, rows, kv->capacity);
    const int pitch = row_pitch(c, ld, kv->kv_heads * c->cfg.head_dim);
    if (pitch < 0)
        return fail(c, FVAR_ERR_INVALID_ARG, "%s: ld=%d is shorter than a row or no multiple of 16 bytes", who, ld);
    timed(c, st, "kvb_append", [&] {
        fvar::launch_kvb_append(dtype(c), k, v, pitch, kvb_cache(kv), B, rows, c->cfg.head_dim, st);
    });
    return launch_status(c, who);
}

fvar_status fvar_kvb_read(fvar_ctx *c, fvar_stream stream, const fvar_kvb *kv, int32_t B, int32_t first, int32_t rows,
                          void *k, void *v)
{
    if (!c) return FVAR_ERR_INVALID_ARG;
    const char *who = "fvar_kvb_read";
    hipStream_t st = static_cast<hipStream_t>(stream);
    const fvar_status ks = check_cache(c, st, kv, B, 0, who);
    if (ks != FVAR_OK) return ks;
    if (!k && !v) return fail(c, FVAR_ERR_INVALID_ARG, "%s: k and v both NULL", who);
    if (!aligned16(k) || !aligned16(v)) return fail(c, FVAR_ERR_INVALID_ARG, "%s: pointer not 16-byte aligned", who);
    if (rows < 1 || rows > kv->capacity || first < -kv->capacity || (int64_t)first + (first < 0 ? 0 : rows) > kv->capacity)
        return fail(c, FVAR_ERR_INVALID_ARG, "%s: rows [%d,+%d) are outside the capacity of %d", who, first, rows,
                    kv->capacity);
    timed(c, st, "kvb_read", [&] {
        fvar::launch_kvb_read(dtype(c), kvb_cache(kv), B, first, rows, c->cfg.head_dim, k, v, st);
    });
    return launch_status(c, who);
}

size_t fvar_kvb_attention_workspace_bytes(const fvar_ctx *c, const fvar_kvb *kv, int32_t B, int32_t n, int32_t weights)
{
    if (!c || !cache_sizes(c, kv, B, n)) return 0;
    return kvb_attention_ws(c, kv, B, n, weights != 0);
}

fvar_status fvar_kvb_attention(fvar_ctx *c, fvar_stream stream, const void *q, int32_t ld, const fvar_kvb *kv, int32_t B,
                               int32_t n, void *o, float *weights, int32_t add, void *ws, size_t ws_bytes)
{
    if (!c) return FVAR_ERR_INVALID_ARG;
    const char *who = "fvar_kvb_attention";
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (n < 1) return fail(c, FVAR_ERR_INVALID_ARG, "%s: need n>=1 (n=%d)", who, n);
    const fvar_status ks = check_cache(c, st, kv, B, 0, who);
    if (ks != FVAR_OK) return ks;
    if (!q || !o) return fail(c, FVAR_ERR_INVALID_ARG, "%s: q or o is NULL", who);
    if (!aligned16(q) || !aligned16(o) || !aligned16(weights) || !aligned16(ws))
        return fail(c, FVAR_ERR_INVALID_ARG, "%s: pointer not 16-byte aligned", who);
    const int pitch = row_pitch(c, ld, c->cfg.hidden);
    if (pitch < 0)
        return fail(c, FVAR_ERR_INVALID_ARG, "%s: ld=%d is shorter than a row or no multiple of 16 bytes", who, ld);
    if ((int64_t)B * n * c->cfg.heads > (1 << 25))
        return fail(c, FVAR_ERR_UNSUPPORTED, "%s: B*n*heads exceeds 2^25", who);
    const size_t need = kvb_attention_ws(c, kv, B, n, weights != nullptr);
    if (need && (!ws || ws_bytes < need))
        return fail(c, FVAR_ERR_WORKSPACE, "%s: workspace of %zu bytes needed, %zu given", who, need, ws_bytes);
    timed(c, st, "kvb_attention", [&] {
        fvar::launch_kvb_attention(dtype(c), q, pitch, kvb_cache(kv), 0, B, n, c->cfg.heads, c->cfg.head_dim, c->scale, o, weights,
                                   add != 0, (float *)ws, st);
    });
    return launch_status(c, who);
}

size_t fvar_kvb_evict_workspace_bytes(const fvar_ctx *c, const fvar_kvb *from, int32_t B, int32_t keep)
{
    if (!c || keep < 1 || keep > (1 << 24) || !cache_sizes(c, from, B, 1)) return 0;
    return align256((size_t)B * sizeof(int32_t)) + align256((size_t)B * from->kv_heads * keep * sizeof(int32_t));
}

fvar_status fvar_kvb_evict(fvar_ctx *c, fvar_stream stream, const fvar_kvb *from, const float *weights, int32_t B, int32_t keep,
                           int32_t recent, const fvar_kvb *to, float *to_weights, int32_t *to_lens, int32_t *idx, void *ws,
                           size_t ws_bytes)
{
    if (!c) return FVAR_ERR_INVALID_ARG;
    const char *who = "fvar_kvb_evict";
    hipStream_t st = static_cast<hipStream_t>(stream);
    const fvar_status ks = check_cache(c, st, from, B, 0, who);
    if (ks != FVAR_OK) return ks;
    if (!to || !to->k || !to->v || !to->k_scale || !to->v_scale || !weights || !to_weights)
        return fail(c, FVAR_ERR_INVALID_ARG, "%s: null argument", who);
    if (!aligned16(to->k) || !aligned16(to->v) || !aligned16(weights) || !aligned16(to_weights) || !aligned16(ws) ||
        (reinterpret_cast<uintptr_t>(to_lens) & 3) || (reinterpret_cast<uintptr_t>(idx) & 3))
        return fail(c, FVAR_ERR_INVALID_ARG, "%s: pointer not aligned (16 bytes; to_lens and idx 4)", who);
    if (to->kv_heads != from->kv_heads)
        return fail(c, FVAR_ERR_INVALID_ARG, "%s: caches of %d and %d kv heads", who, from->kv_heads, to->kv_heads);
    if (keep < 1 || recent < 0 || recent > keep || keep > to->capacity)
        return fail(c, FVAR_ERR_INVALID_ARG, "%s: need 0<=recent<=keep, 1<=keep<=capacity of the second cache (keep=%d recent=%d capacity=%d)",
                    who, keep, recent, to->capacity);
    if (to->capacity > (1 << 24)) return fail(c, FVAR_ERR_UNSUPPORTED, "%s: capacity exceeds 2^24", who);
    {
        const size_t heads = (size_t)B * from->kv_heads, Dh = c->cfg.head_dim;
        const bool here = from->k == to->k;
        const void *a[4] = {from->k, from->v, from->k_scale, from->v_scale}, *b[4] = {to->k, to->v, to->k_scale, to->v_scale};
        for (int i = 0; i < 4; ++i) {
            if (here && (a[i] != b[i] || from->capacity != to->capacity))
                return fail(c, FVAR_ERR_INVALID_ARG, "%s: the caches are one in part", who);
            for (int j = 0; j < 4 && !here; ++j) {
                const size_t na = heads * (i < 2 ? from->capacity * Dh : (from->capacity + 31) / 32);
                const size_t nb = heads * (j < 2 ? to->capacity * Dh : (to->capacity + 31) / 32);
                if (overlap(a[i], na, b[j], nb)) return fail(c, FVAR_ERR_INVALID_ARG, "%s: the caches share memory", who);
            }
        }
        if (!(here && weights == to_weights) &&
            overlap(weights, heads * from->capacity * sizeof(float), to_weights, heads * to->capacity * sizeof(float)))
            return fail(c, FVAR_ERR_INVALID_ARG, "%s: weights and to_weights share memory", who);
    }
    const size_t need = fvar_kvb_evict_workspace_bytes(c, from, B, keep);
    if (!ws || ws_bytes < need)
        return fail(c, FVAR_ERR_WORKSPACE, "%s: workspace of %zu bytes needed, %zu given", who, need, ws_bytes);
    int32_t *counts = static_cast<int32_t *>(ws);
    int32_t *rows = idx ? idx : reinterpret_cast<int32_t *>(static_cast<char *>(ws) + align256((size_t)B * sizeof(int32_t)));
    timed(c, st, "kvb_rank", [&] { fvar::launch_kvb_rank(kvb_cache(from), weights, B, keep, recent, rows, counts, st); });
    timed(c, st, "kvb_move", [&] {
        fvar::launch_kvb_move(kvb_cache(from), weights, kvb_cache(to), to_weights, to_lens, B, keep, c->cfg.head_dim, rows, counts, st);
    });
    return launch_status(c, who);
}

static fvar_status lowrank_fill(fvar_ctx *c, fvar_stream stream, const void *y_keep,
                                const int32_t *idx_keep, const int32_t *idx_drop, int32_t B, int32_t M,
                                int32_t k, int32_t r, const void *w_c, const void *g_c, void *y,
                                float *scores_out, void *ws, size_t ws_bytes, const char *who)
{
    if (B < 1 || M < 1 || k < 0 || k > M)
        return fail(c, FVAR_ERR_INVALID_ARG, "%s: need B>=1 and 0<=k<=M (B=%d M=%d k=%d)", who, B, M, k);
    if (!y || (k > 0 && !y_keep)) return fail(c, FVAR_ERR_INVALID_ARG, "%s: null output or y_keep", who);
    if (k < M) {
        if (!idx_keep && k > 0) return fail(c, FVAR_ERR_INVALID_ARG, "%s: idx_keep is NULL", who);
        if (!idx_drop || !w_c || !g_c)
            return fail(c, FVAR_ERR_INVALID_ARG, "%s: idx_drop, w_c and g_c are required when k < M", who);
        const int mult = c->cfg.dtype == FVAR_BF16 ? 8 : 4;
        if (r < 1 || r > 256 || r % mult)
            return fail(c, FVAR_ERR_INVALID_ARG, "%s: rank %d must be in [1,256] and a multiple of %d",
                        who, r, mult);
    }
    if (!aligned16(y) || !aligned16(y_keep) || !aligned16(w_c) || !aligned16(g_c) || !aligned16(ws))
        return fail(c, FVAR_ERR_INVALID_ARG, "%s: pointer not 16-byte aligned", who);
    if ((int64_t)B * M > (int64_t)INT32_MAX / 2)
        return fail(c, FVAR_ERR_UNSUPPORTED, "%s: B*M too large", who);
    double *parts = nullptr;
    if (scores_out) {
        const size_t need = fvar_fill_scored_workspace_bytes(c, B, M);
        if (!ws || ws_bytes < need)
            return fail(c, FVAR_ERR_WORKSPACE, "%s: workspace of %zu bytes needed, %zu given", who, need,
                        ws_bytes);
        parts = static_cast<double *>(ws);
    }
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (c->debug_checks && k < M) {
        const fvar_status vs = validate_indices(c, st, idx_keep, idx_drop, B, M, k, who);
        if (vs != FVAR_OK) return vs;
    }
    timed(c, st, "fill", [&] {
        fvar::launch_fill(dtype(c), y_keep, idx_keep, idx_drop, B, M, k, r, c->cfg.hidden, w_c, g_c, y,
                          parts, scores_out,
                          fvar::map_past_caches((size_t)B * M * c->cfg.hidden * esize(c), scores_out != nullptr), st);
    });
    return launch_status(c, who);
}

size_t fvar_fill_scored_workspace_bytes(const fvar_ctx *c, int32_t B, int32_t M)
{
    if (!c || B < 1 || M < 1) return 0;
    return align256((size_t)B * M * fvar::fill_score_parts(dtype(c), c->cfg.hidden) * sizeof(double));
}

fvar_status fvar_lowrank_fill(fvar_ctx *c, fvar_stream stream, const void *y_keep,
                              const int32_t *idx_keep, const int32_t *idx_drop, int32_t B, int32_t M,
                              int32_t k, int32_t r, const void *w_c, const void *g_c, void *y)
{
    if (!c) return FVAR_ERR_INVALID_ARG;
    return lowrank_fill(c, stream, y_keep, idx_keep, idx_drop, B, M, k, r, w_c, g_c, y, nullptr, nullptr,
                        0, "fvar_lowrank_fill");
}

fvar_status fvar_lowrank_fill_scored(fvar_ctx *c, fvar_stream stream, const void *y_keep,
                                     const int32_t *idx_keep, const int32_t *idx_drop, int32_t B,
                                     int32_t M, int32_t k, int32_t r, const void *w_c, const void *g_c,
                                     void *y, float *scores_out, void *ws, size_t ws_bytes)
{
    if (!c) return FVAR_ERR_INVALID_ARG;
    if (!scores_out)
        return fail(c, FVAR_ERR_INVALID_ARG, "fvar_lowrank_fill_scored: scores_out is NULL");
    return lowrank_fill(c, stream, y_keep, idx_keep, idx_drop, B, M, k, r, w_c, g_c, y, scores_out, ws,
                        ws_bytes, "fvar_lowrank_fill_scored");
}

fvar_status fvar_rp_project(fvar_ctx *c, fvar_stream stream, const void *qt, int32_t q_per_sample,
                            const void *x, int32_t B, int32_t M, int32_t rows, void *out)
{
    if (!c) return FVAR_ERR_INVALID_ARG;
    const char *who = "fvar_rp_project";
    if (B < 1 || M < 1 || rows < 1 || rows > M)
        return fail(c, FVAR_ERR_INVALID_ARG, "%s: need B>=1 and 1<=rows<=M (B=%d M=%d rows=%d)", who, B,
                    M, rows);
    if (!qt || !x || !out) return fail(c, FVAR_ERR_INVALID_ARG, "%s: null argument", who);
    if (!aligned16(qt) || !aligned16(x) || !aligned16(out))
        return fail(c, FVAR_ERR_INVALID_ARG, "%s: pointer not 16-byte aligned", who);
    const int mult = c->cfg.dtype == FVAR_BF16 ? 8 : 4;
    if (M % mult)
        return fail(c, FVAR_ERR_UNSUPPORTED, "%s: M=%d must be a multiple of %d", who, M, mult);
    if ((int64_t)B * M > (int64_t)INT32_MAX / 2 || B > 65535)
        return fail(c, FVAR_ERR_UNSUPPORTED, "%s: B or B*M too large", who);
    hipStream_t st = static_cast<hipStream_t>(stream);
    timed(c, st, "rp_project", [&] {
        fvar::launch_rp_project(dtype(c), qt, q_per_sample ? (size_t)rows * M : 0, x, B, M, rows,
                                c->cfg.hidden, out, st);
    });
    return launch_status(c, who);
}

fvar_status fvar_cache_fill(fvar_ctx *c, fvar_stream stream, const void *y_keep,
                            const int32_t *idx_keep, const int32_t *idx_drop, int32_t B, int32_t M,
                            int32_t k, const void *cache, void *y)
{
    if (!c) return FVAR_ERR_INVALID_ARG;
    const char *who = "fvar_cache_fill";
    if (B < 1 || M < 1 || k < 0 || k > M)
        return fail(c, FVAR_ERR_INVALID_ARG, "%s: need B>=1 and 0<=k<=M (B=%d M=%d k=%d)", who, B, M, k);
    if (!y || (k > 0 && (!y_keep || !idx_keep)))
        return fail(c, FVAR_ERR_INVALID_ARG, "%s: null output, y_keep or idx_keep", who);
    if (k < M && (!idx_drop || !cache))
        return fail(c, FVAR_ERR_INVALID_ARG, "%s: idx_drop and cache are required when k < M", who);
    if (!aligned16(y) || !aligned16(y_keep) || !aligned16(cache))
        return fail(c, FVAR_ERR_INVALID_ARG, "%s: pointer not 16-byte aligned", who);
    if ((int64_t)B * M > (int64_t)INT32_MAX / 2)
        return fail(c, FVAR_ERR_UNSUPPORTED, "%s: B*M too large", who);
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (c->debug_checks) {
        const fvar_status vs = validate_indices(c, st, idx_keep, idx_drop, B, M, k, who);
        if (vs != FVAR_OK) return vs;
    }
    timed(c, st, "cache_fill", [&] {
        fvar::launch_cache_fill(dtype(c), y_keep, idx_keep, idx_drop, B, M, k, c->cfg.hidden, cache, y,
                                st);
    });
    return launch_status(c, who);
}

size_t fvar_factors_workspace_bytes(const fvar_ctx *c, int32_t B, int32_t M, int32_t r)
{
    if (!c || B < 1 || M < 1 || r < 1) return 0;
    const size_t rr = (size_t)B * r * r * sizeof(double);
    return align256(fvar::factor_t_room(dtype(c), B, M, c->cfg.hidden) * r * sizeof(float)) +
           align256(rr * fvar::gram_room(dtype(c))) + align256(rr);
}

fvar_status fvar_cache_factors(fvar_ctx *c, fvar_stream stream, const void *cache, const void *qt,
                               int32_t q_per_sample, int32_t B, int32_t M, int32_t r, double ridge,
                               void *w_c, void *g_c, void *ws, size_t ws_bytes)
{
    if (!c) return FVAR_ERR_INVALID_ARG;
    const char *who = "fvar_cache_factors";
    const int mult = c->cfg.dtype == FVAR_BF16 ? 8 : 4;
    if (B < 1 || M < 1 || r < 1 || r > M)
        return fail(c, FVAR_ERR_INVALID_ARG, "%s: need B>=1 and 1<=r<=M (B=%d M=%d r=%d)", who, B, M, r);
    if (!cache || !qt || !w_c || !g_c) return fail(c, FVAR_ERR_INVALID_ARG, "%s: null argument", who);
    if (!(ridge >= 0.0)) return fail(c, FVAR_ERR_INVALID_ARG, "%s: ridge must be >= 0", who);
    if (r > 128 || r % mult)
        return fail(c, FVAR_ERR_UNSUPPORTED, "%s: rank %d must be <= 128 and a multiple of %d", who, r,
                    mult);
    if (M % mult)
        return fail(c, FVAR_ERR_UNSUPPORTED, "%s: M=%d must be a multiple of %d", who, M, mult);
    if ((int64_t)B * M > (int64_t)INT32_MAX / 2 || B > 65535)
        return fail(c, FVAR_ERR_UNSUPPORTED, "%s: B or B*M too large", who);
    if (!aligned16(cache) || !aligned16(qt) || !aligned16(w_c) || !aligned16(g_c) || !aligned16(ws))
        return fail(c, FVAR_ERR_INVALID_ARG, "%s: pointer not 16-byte aligned", who);
    const size_t need = fvar_factors_workspace_bytes(c, B, M, r);
    if (!ws || ws_bytes < need)
        return fail(c, FVAR_ERR_WORKSPACE, "%s: workspace of %zu bytes needed, %zu given", who, need,
                    ws_bytes);
    char *p = static_cast<char *>(ws);
    float *T = reinterpret_cast<float *>(p);
    p += align256(fvar::factor_t_room(dtype(c), B, M, c->cfg.hidden) * r * sizeof(float));
    double *S = reinterpret_cast<double *>(p);
    p += align256((size_t)B * r * r * sizeof(double) * fvar::gram_room(dtype(c)));
    double *Sinv = reinterpret_cast<double *>(p);
    hipStream_t st = static_cast<hipStream_t>(stream);
    const DType dt = dtype(c);
    const int d = c->cfg.hidden;
    timed(c, st, "factor_project", [&] {
        fvar::launch_rp_project(dt, qt, q_per_sample ? (size_t)r * M : 0, cache, B, M, r, d, g_c, st);
    });
    timed(c, st, "factor_gram", [&] { fvar::launch_factor_gram(dt, g_c, B, r, d, S, st); });
    if (dt == DType::BF16) {
        timed(c, st, "factor_t_inverse", [&] {
            fvar::launch_factor_t_inverse(cache, g_c, B, M, r, d, T, S, ridge, Sinv, st);
        });
    } else {
        timed(c, st, "factor_t", [&] { fvar::launch_factor_t_f32(cache, g_c, B, M, r, d, T, st); });
        timed(c, st, "factor_inverse", [&] { fvar::launch_factor_inverse(S, 1, B, r, ridge, Sinv, st); });
    }
    timed(c, st, "factor_w", [&] { fvar::launch_factor_w(dt, T, Sinv, B, M, r, d, w_c, st); });
    return launch_status(c, who);
}

fvar_status fvar_upsample_tokens(fvar_ctx *c, fvar_stream stream, const void *src, int32_t B,
                                 int32_t hs, int32_t ws, int32_t ch, int32_t hd, int32_t wd,
                                 void *dst)
{
    if (!c) return FVAR_ERR_INVALID_ARG;
    const char *who = "fvar_upsample_tokens";
    if (B < 1 || hs < 1 || ws < 1 || hd < 1 || wd < 1 || ch < 1)
        return fail(c, FVAR_ERR_INVALID_ARG, "%s: sizes must be >= 1", who);
    if (!src || !dst) return fail(c, FVAR_ERR_INVALID_ARG, "%s: null argument", who);
    if (!aligned16(src) || !aligned16(dst))
        return fail(c, FVAR_ERR_INVALID_ARG, "%s: pointer not 16-byte aligned", who);
    const int mult = c->cfg.dtype == FVAR_BF16 ? 8 : 4;
    if (ch % mult)
        return fail(c, FVAR_ERR_UNSUPPORTED, "%s: channel count %d must be a multiple of %d", who, ch,
                    mult);
    if ((int64_t)hs * ws > (1 << 24) || (int64_t)hd * wd > (1 << 24) ||
        (int64_t)B * hd * wd * (ch / mult) > ((int64_t)1 << 38))
        return fail(c, FVAR_ERR_UNSUPPORTED, "%s: grid too large", who);
    hipStream_t st = static_cast<hipStream_t>(stream);
    timed(c, st, "upsample", [&] {
        fvar::launch_upsample(dtype(c), src, B, hs, ws, hd, wd, ch, dst, st);
    });
    return launch_status(c, who);
}

fvar_status fvar_profile_enable(fvar_ctx *c, int32_t on)
{
    if (!c) return FVAR_ERR_INVALID_ARG;
    c->profiling = on != 0;
    return FVAR_OK;
}

int32_t fvar_profile_read(fvar_ctx *c, fvar_profile_entry *out, int32_t cap)
{
    if (!c) return 0;
    std::map<std::string, std::pair<int64_t, double>> acc;
    std::vector<std::string> order;
    for (auto &r : c->recs) {
        (void)hipEventSynchronize(r.b);
        float ms = 0.f;
        (void)hipEventElapsedTime(&ms, r.a, r.b);
        if (!acc.count(r.label)) order.push_back(r.label);
        auto &e = acc[r.label];
        e.first += 1;
        e.second += ms;
        c->pool.push_back(r.a);
        c->pool.push_back(r.b);
    }
    c->recs.clear();
    int32_t nlab = 0;
    for (auto &lab : order) {
        if (out && nlab < cap) {
            std::snprintf(out[nlab].label, sizeof(out[nlab].label), "%s", lab.c_str());
            out[nlab].launches = acc[lab].first;
            out[nlab].total_ms = acc[lab].second;
        }
        ++nlab;
    }
    return nlab;
}

}  // extern "C"
