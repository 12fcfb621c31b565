// Eviction from the 8-bit cache (format and layout: kvb.hip): which rows of a sample and kv head stay, and their way to the front.
//
// Of the rows that a sample holds and that its mask does not hide, `keep` stay: the last `recent` of all that it holds, and of the
// others those with the largest weights, equal ones from the lowest row on.
#include "kvb.h"
#include "select.h"

namespace fvar {

// Key of a row: hidden ones below all others, late ones above, a weight that is not a number above all numbers.
constexpr uint32_t kHidden = 0u, kNothing = 0x80000000u, kLate = 0xffffffffu, kNoNumber = 0xfffffffeu;   // kNothing: a weight of 0
__device__ __forceinline__ uint32_t row_key(float weight, bool seen, bool late)
{
    const uint32_t key = weight != weight ? kNoNumber : score_key(weight);
    return !seen ? kHidden : late ? kLate : key;
}

constexpr int kRankKeysMax = 20;                             // keys per thread that stay in registers

// One workgroup per sample and kv head, which its instructions and barriers bound: 7 us for 1000 rows, 13 for 10521, 23 for 16921 (26 with a
// mask).  KPT: keys per thread, 0: more than registers hold, read from memory in each pass.
// The kept rows, ascending, go to idx, -1 behind them; their number, the same for all heads, to counts.
template <int KPT>
__global__ __launch_bounds__(kSelThreads) void kvb_rank_kernel(KvbCache c, const float *__restrict__ weights, int keep, int recent,
                                                               int32_t *__restrict__ idx, int32_t *__restrict__ counts)
{
    __shared__ int late_here[kSelWaves], seen_here[kSelWaves], some_here[kSelWaves];
    const int tid = threadIdx.x, b = blockIdx.x / c.heads, len = kvb_length(c, b, 0);
    const int from = max(len - recent, 0);                   // the first late row
    const float *w = weights + (size_t)blockIdx.x * c.capacity;
    const uint8_t *mask = c.mask ? c.mask + (size_t)b * c.capacity : nullptr;
    int32_t *out = idx + (size_t)blockIdx.x * keep;
    auto key_at = [&](int i) { return row_key(w[i], !mask || mask[i] != 0, i >= from); };

    // Rows that have got nothing are many, and far from all others: the range in which the last row to stay is looked for is that of the
    // others, or, where those are too few, the rest.
    uint32_t key[KPT > 0 ? KPT : 1], lo = 0xffffffffu, hi = 0u, least = 0xffffffffu;
    int late = 0, seen = 0, some = 0;
    auto look = [&](uint32_t x) {
        late += x == kLate;
        seen += x != kHidden;
        if (x != kLate && x > kNothing) { ++some; lo = min(lo, x); hi = max(hi, x); }
        if (x != kHidden) least = min(least, x);
    };
    if constexpr (KPT > 0) {
        float weight[KPT];
        bool there[KPT];
#pragma unroll
        for (int j = 0; j < KPT; ++j) {                      // all loads ahead of their first use
            const int i = min(j * kSelThreads + tid, max(len - 1, 0));
            weight[j] = w[i];
            there[j] = !mask || mask[i] != 0;
        }
#pragma unroll
        for (int j = 0; j < KPT; ++j) {
            const int i = j * kSelThreads + tid;
            key[j] = row_key(weight[j], there[j] && i < len, i >= from);
            look(key[j]);
        }
    } else {
        for (int i = tid; i < len; i += kSelThreads) look(key_at(i));
    }
    late = (int)wave_total((uint32_t)late);
    seen = (int)wave_total((uint32_t)seen);
    some = (int)wave_total((uint32_t)some);
    if ((tid & 63) == 0) { late_here[tid >> 6] = late; seen_here[tid >> 6] = seen; some_here[tid >> 6] = some; }
    __syncthreads();
    late = seen = some = 0;
#pragma unroll
    for (int i = 0; i < kSelWaves; ++i) { late += late_here[i]; seen += seen_here[i]; some += some_here[i]; }
    const int count = min(keep, seen);
    for (int i = count + tid; i < keep; i += kSelThreads) out[i] = -1;
    if (blockIdx.x % c.heads == 0 && tid == 0) counts[b] = count;
    if (count == 0) return;
    auto emit = [&](int i, bool stays, int at) {
        if (stays) out[at] = i;
    };
    if constexpr (KPT > 0) {
        __shared__ SelectLds<KPT> sh;
        uint32_t T = kNoNumber;                              // late rows alone
        int need_eq = 0;
        int want = count - late;
        if (want > some) {                                   // (keys above hi are not counted)
            want -= some;
            lo = least;
            hi = kNothing;
        }
        if (want > 0) select_threshold<KPT>(key, len, want, lo, hi, sh, T, need_eq);
        select_sweep<KPT>(key, len, T, need_eq, sh, emit);
    } else {
        __shared__ SelectStreamLds sh;
        select_streamed(key_at, len, count, sh, emit);
    }
}

// Sixteen bytes of a row per lane, whole rows one after the other: a wavefront holds a block of 32 rows in DH / 32 registers of sixteen bytes.
template <int DH> struct MovedBlock {
    static constexpr int PER = DH / 16, ROWS = 64 / PER, N = kKvbBlock / ROWS;   // lanes of a row; rows of a load; loads
    uint4 w[N];
    uint32_t byte[N];
    uint32_t top;                                            // fp32 bits of the block's largest magnitude

    // rows idx[32 block ..] of a head's `codes`, those at `count` and beyond left out
    __device__ __forceinline__ void fetch(const uint8_t *codes, const uint8_t *scales, const int32_t *idx, int block, int count)
    {
        const int lane = threadIdx.x & 63;
        int row[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int at = block * kKvbBlock + i * ROWS + lane / PER;
            row[i] = at < count ? idx[at] : -1;
        }
#pragma unroll
        for (int i = 0; i < N; ++i) {
            w[i] = make_uint4(0, 0, 0, 0);
            byte[i] = 10;
            if (row[i] >= 0) {
                w[i] = *reinterpret_cast<const uint4 *>(codes + (size_t)row[i] * DH + lane % PER * 16);
                byte[i] = scales[row[i] / kKvbBlock];
            }
        }
    }
    // a code's magnitude grows with its lower 7 bits; 127 is not a number
    static __device__ __forceinline__ uint32_t largest(uint32_t x)
    {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t code = x >> (8 * i) & 127;
            m = max(m, code == 127 ? 0 : code);
        }
        return m;
    }
    __device__ __forceinline__ void measure()
    {
        top = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const uint32_t m = max(max(largest(w[i].x), largest(w[i].y)), max(largest(w[i].z), largest(w[i].w)));
            top = max(top, __float_as_uint(__builtin_amdgcn_cvt_scalef32_pk_f32_fp8(m, __uint_as_float(byte[i] << 23), false)[0]));
        }
        top = wave_largest(top);
    }
    __device__ __forceinline__ void put(uint8_t *codes, uint8_t *scales, int block, int count)
    {
        const int lane = threadIdx.x & 63;
        const uint32_t to = kvb_byte(top);
        const float size = __uint_as_float(to << 23);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int at = block * kKvbBlock + i * ROWS + lane / PER;
            if (at >= count) continue;
            if (byte[i] != to) {
                const float from = __uint_as_float(byte[i] << 23);
                w[i].x = kvb_again(w[i].x, from, size);
                w[i].y = kvb_again(w[i].y, from, size);
                w[i].z = kvb_again(w[i].z, from, size);
                w[i].w = kvb_again(w[i].w, from, size);
            }
            *reinterpret_cast<uint4 *>(codes + (size_t)at * DH + lane % PER * 16) = w[i];
        }
        if (lane == 0) scales[block] = (uint8_t)to;
    }
};

// A wavefront per block, four to a workgroup, into a cache that shares no memory with the first.  grid: (blocks / 4, B * heads, K or V).
// Memory-bound: 187 MB to where they go, 4 samples of up to 8461 rows, 32 heads of 128, 70 us (5.3 TB/s).
template <int DH>
__global__ __launch_bounds__(256) void kvb_move_kernel(KvbCache from, const float *__restrict__ weights, KvbCache to, float *__restrict__ to_weights,
                                                       int32_t *__restrict__ to_lens, int keep, const int32_t *__restrict__ idx,
                                                       const int32_t *__restrict__ counts)
{
    const int head = blockIdx.y, b = head / from.heads, count = counts[b];
    const int32_t *rows = idx + (size_t)head * keep;
    const int block = blockIdx.x * 4 + (threadIdx.x >> 6);
    if (blockIdx.z == 0) {
        const int per = 4 * kKvbBlock, at = blockIdx.x * per + threadIdx.x;
        if (threadIdx.x < per && at < to.capacity)
            to_weights[(size_t)head * to.capacity + at] = at < count ? weights[(size_t)head * from.capacity + rows[at]] : 0.f;
        if (to_lens && head % from.heads == 0 && blockIdx.x == 0 && threadIdx.x == 0) to_lens[b] = count;
    }
    if (block * kKvbBlock >= count) return;
    const size_t src = (size_t)head * from.capacity * DH, dst = (size_t)head * to.capacity * DH;
    MovedBlock<DH> x;
    x.fetch((blockIdx.z ? from.v : from.k) + src, (blockIdx.z ? from.v_scale : from.k_scale) + (size_t)head * from.blocks(), rows, block, count);
    x.measure();
    x.put((blockIdx.z ? to.v : to.k) + dst, (blockIdx.z ? to.v_scale : to.k_scale) + (size_t)head * to.blocks(), block, count);
}

// The same within one cache: a workgroup per sample, head and K or V takes sixteen blocks at a time, in order.  A kept row comes from its own
// place or one further on, so what a step writes over is what this and earlier steps have fetched: all of a step is in registers before any
// of it is written, and the next step's rows, which are fetched meanwhile, lie behind all that this one writes.  Where there are heads enough it
// is as fast as into another cache (4 x 32 heads of 128, 8461 of 16921 rows, 108 us, 106); of few heads each goes its way alone (16 heads, 4209 of 10521
// rows, 30 us, 8; the places of rows looked up two steps ahead take the registers that the steps need, 42).
template <int DH>
__global__ __launch_bounds__(1024) void kvb_move_here_kernel(KvbCache c, const float *weights, float *to_weights, int32_t *to_lens, int keep,
                                                             const int32_t *__restrict__ idx, const int32_t *__restrict__ counts)
{
    constexpr int STEP = 16;                                 // blocks
    const int head = blockIdx.x, b = head / c.heads, count = counts[b], wave = threadIdx.x >> 6;
    const int32_t *rows = idx + (size_t)head * keep;
    uint8_t *codes = (blockIdx.y ? c.v : c.k) + (size_t)head * c.capacity * DH;
    uint8_t *scales = (blockIdx.y ? c.v_scale : c.k_scale) + (size_t)head * c.blocks();
    const float *w = weights + (size_t)head * c.capacity;
    float *to_w = to_weights + (size_t)head * c.capacity;
    const int blocks = (count + kKvbBlock - 1) / kKvbBlock;
    const bool weigh = blockIdx.y == 0 && threadIdx.x < STEP * kKvbBlock;
    if (to_lens && blockIdx.y == 0 && head % c.heads == 0 && threadIdx.x == 0) to_lens[b] = count;

    struct Step { MovedBlock<DH> x; float weight; };
    auto fetch = [&](int block0, Step &s) {
        s.x.fetch(codes, scales, rows, block0 + wave, count);
        const int at = block0 * kKvbBlock + threadIdx.x;
        s.weight = weigh && at < count ? w[rows[at]] : 0.f;
    };
    auto step = [&](int block0, Step &now, Step &next) {
        if (block0 + STEP < blocks) fetch(block0 + STEP, next);
        now.x.measure();
        asm volatile("" : "+v"(now.weight));
        __syncthreads();                                     // everything of this step has been fetched
        if (block0 + wave < blocks) now.x.put(codes, scales, block0 + wave, count);
        const int at = block0 * kKvbBlock + threadIdx.x;
        if (weigh && at < count) to_w[at] = now.weight;
    };
    Step one, two;
    fetch(0, one);
    for (int block0 = 0; block0 < blocks; block0 += 2 * STEP) {
        step(block0, one, two);
        if (block0 + STEP < blocks) step(block0 + STEP, two, one);
    }
    __syncthreads();
    if (blockIdx.y == 0)
        for (int at = count + threadIdx.x; at < c.capacity; at += 1024) to_w[at] = 0.f;
}

void launch_kvb_rank(const KvbCache &c, const float *weights, int B, int keep, int recent, int32_t *idx, int32_t *counts, hipStream_t st)
{
    const int longest = c.lens ? c.capacity : c.len, kpt = (longest + kSelThreads - 1) / kSelThreads;
#define FVAR_RANK(KPT) launch(kvb_rank_kernel<KPT>, dim3((unsigned)(B * c.heads)), dim3(kSelThreads), 0, st, c, weights, keep, recent, idx, counts)
    if (kpt <= 1) FVAR_RANK(1);
    else if (kpt <= 2) FVAR_RANK(2);
    else if (kpt <= 4) FVAR_RANK(4);
    else if (kpt <= 8) FVAR_RANK(8);
    else if (kpt <= 12) FVAR_RANK(12);
    else if (kpt <= kRankKeysMax) FVAR_RANK(kRankKeysMax);
    else FVAR_RANK(0);
#undef FVAR_RANK
}

void launch_kvb_move(const KvbCache &from, const float *weights, const KvbCache &to, float *to_weights, int32_t *to_lens, int B, int keep, int Dh,
                     const int32_t *idx, const int32_t *counts, hipStream_t st)
{
    const unsigned heads = (unsigned)(B * from.heads);
    if (from.k == to.k) {
#define FVAR_HERE(DH) launch(kvb_move_here_kernel<DH>, dim3(heads, 2), dim3(1024), 0, st, from, weights, to_weights, to_lens, keep, idx, counts)
        if (Dh == 64) FVAR_HERE(64);
        else FVAR_HERE(128);
#undef FVAR_HERE
        return;
    }
    const dim3 grid((unsigned)((to.blocks() + 3) / 4), heads, 2);
#define FVAR_MOVE(DH) launch(kvb_move_kernel<DH>, grid, dim3(256), 0, st, from, weights, to, to_weights, to_lens, keep, idx, counts)
    if (Dh == 64) FVAR_MOVE(64);
    else FVAR_MOVE(128);
#undef FVAR_MOVE
}

}  // namespace fvar
