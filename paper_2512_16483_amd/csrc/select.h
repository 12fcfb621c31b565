// Selection of the k largest of M keys by one workgroup of 1024 threads, ties to the lowest index, with the kept ones in ascending
// order: for the token selection (score_select.hip) and the eviction from a cache (kvb_evict.hip).
#pragma once
#include "common.h"

namespace fvar {

// Order-preserving map float -> uint32 (larger float <=> larger key); -0 and +0 share a key.
__device__ __forceinline__ uint32_t score_key(float s)
{
    uint32_t b = __float_as_uint(s);
    if (b == 0x80000000u) b = 0u;
    return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}

// Over a wavefront, in registers (a shuffle is a trip through LDS): sum and largest in every lane, running sum.
template <typename Op> __device__ __forceinline__ uint32_t wave_fold(uint32_t v, Op op)
{
    v = op(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0xb1, 0xf, 0xf, true));             // quad_perm 1,0,3,2
    v = op(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x4e, 0xf, 0xf, true));             // quad_perm 2,3,0,1
    v = op(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x141, 0xf, 0xf, true));            // row_half_mirror
    v = op(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x140, 0xf, 0xf, true));            // row_mirror
    const auto a = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    v = op(a[0], a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return op(b[0], b[1]);
}
__device__ __forceinline__ uint32_t wave_total(uint32_t v) { return wave_fold(v, [](uint32_t x, uint32_t y) { return x + y; }); }
__device__ __forceinline__ uint32_t wave_largest(uint32_t v) { return wave_fold(v, [](uint32_t x, uint32_t y) { return max(x, y); }); }
__device__ __forceinline__ int wave_running(int v)
{
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, true);                           // row_shr:1, 2, 4, 8
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, true);
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, true);
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, true);
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);                          // row_bcast:15 to rows 1 and 3
    v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);                          // row_bcast:31 to rows 2 and 3
    return v;
}

constexpr int kSelThreads = 1024;
constexpr int kSelWaves = kSelThreads / 64;
constexpr int kSelBins = 4096;               // four per thread

template <int KPT> struct SelectLds {
    int hist[kSelBins];
    uint32_t wave_min[kSelWaves], wave_max[kSelWaves], few[64];
    int totals[kSelWaves], counts[KPT * kSelWaves];
    int bin, remaining, count, found;
};

// T: the k-th largest key; need_eq: how many keys equal to T are kept (the lowest indices).  Thread tid holds the keys tid, tid + 1024,
// ... of M in registers; lo and hi: the smallest and the largest key of those that count, among the thread's own.  Keys above hi are
// not counted in k, and those below lo are not among the k.
// The first histogram spans the keys' own range, so that neighbouring scores (a few
// binades in all, which one 8-bit digit throws into a handful of bins whose LDS atomics then run one by one)
// spread over its 4096 bins; the bin that holds the k-th largest key is divided in the same way until at most
// 64 keys are left, all of the bin is kept, or its keys are equal.  Those few are ranked by each wavefront for
// itself.  The sweep that follows counts all its pieces at once, for one barrier in all.
// Latency alone counts here: one workgroup per sample, six barriers where four 8-bit digits from LDS and a
// barrier per 1024 tokens of the sweep took 12 and more.  8 x 4096 scores 11.3 -> 6.6 us, 2304 scores 9 -> 5.9,
// 8 x 576 scores 5.0 -> 5.1.
template <int KPT>
__device__ __forceinline__ void select_threshold(const uint32_t (&key)[KPT], int M, int k, uint32_t lo, uint32_t hi, SelectLds<KPT> &sh,
                                                 uint32_t &T, int &need_eq)
{
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    lo = ~wave_largest(~lo);
    hi = wave_largest(hi);
    if (lane == 0) { sh.wave_min[wave] = lo; sh.wave_max[wave] = hi; }
    reinterpret_cast<int4 *>(sh.hist)[tid] = make_int4(0, 0, 0, 0);
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kSelWaves; ++w) { lo = min(lo, sh.wave_min[w]); hi = max(hi, sh.wave_max[w]); }

    // `base` is the largest key of the range in question, `bins` its bins of 2^shift keys, largest first.
    uint32_t base = hi;
    int remaining = k;
    uint32_t bins = kSelBins;
    int shift = max(0, 20 - __clz((int)(hi - lo)));      // hi == lo: clz 32
    for (;;) {
#pragma unroll
        for (int j = 0; j < KPT; ++j) {
            const uint32_t bin = (base - key[j]) >> shift;
            // keys above the range wrap to a large difference, which at shift 0 and a base of few bits is the
            // only thing that tells them apart
            if (j * kSelThreads + tid < M && key[j] <= base && bin < bins) atomicAdd(&sh.hist[bin], 1);
        }
        if (tid == 0) sh.found = 0;
        __syncthreads();
        const int4 c = reinterpret_cast<const int4 *>(sh.hist)[tid];
        const int sum = c.x + c.y + c.z + c.w;
        const int incl = wave_running(sum);
        if (lane == 63) sh.totals[wave] = incl;
        __syncthreads();
        int run = incl - sum;                            // keys in larger bins
#pragma unroll
        for (int w = 0; w < kSelWaves; ++w) run += w < wave ? sh.totals[w] : 0;
        if (run < remaining && remaining <= run + sum) { // one thread
            int bin = 4 * tid, n = c.x;
            if (remaining > run + n) { run += n; ++bin; n = c.y; }
            if (remaining > run + n) { run += n; ++bin; n = c.z; }
            if (remaining > run + n) { run += n; ++bin; n = c.w; }
            sh.bin = bin; sh.remaining = remaining - run; sh.count = n;
        }
        __syncthreads();
        const uint32_t bin = (uint32_t)sh.bin;
        const int count = sh.count;
        remaining = sh.remaining;
        base -= bin << shift;                            // the bin's largest key
        if (count == remaining || shift == 0) {          // all of it, or equal keys
            const uint32_t width = (1u << shift) - 1u;
            T = width > base ? 0u : base - width;
            need_eq = count == remaining ? M : remaining;
            break;
        }
        if (count <= 64) {
#pragma unroll
            for (int j = 0; j < KPT; ++j)
                if (j * kSelThreads + tid < M && key[j] <= base && (base - key[j]) >> shift == 0)
                    sh.few[atomicAdd(&sh.found, 1)] = key[j];
            __syncthreads();
            const uint32_t mine = sh.few[min(lane, count - 1)];
            const uint32_t one = (uint32_t)__builtin_amdgcn_readfirstlane((int)mine);
            if (__ballot(mine == one) == ~0ull) {        // equal scores: 48 of them ranked one by one take 3 us
                T = one;
                need_eq = remaining;
                break;
            }
            int above = 0, equal = 0;
            for (int i = 0; i < count; ++i) {
                const uint32_t other = (uint32_t)__builtin_amdgcn_readlane((int)mine, i);
                above += other > mine;
                equal += other == mine;
            }
            // every lane with the wanted key agrees; take the first
            const int src = __ffsll(__ballot(above < remaining && remaining <= above + equal)) - 1;
            T = (uint32_t)__builtin_amdgcn_readlane((int)mine, src);
            need_eq = remaining - __builtin_amdgcn_readlane(above, src);
            break;
        }
        // divide the bin; its counts were read before the last barrier
        const int next = max(0, shift - 12);
        bins = 1u << (shift - next);
        shift = next;
        reinterpret_cast<int4 *>(sh.hist)[tid] = make_int4(0, 0, 0, 0);
        __syncthreads();
    }
}

template <int KPT, typename Emit>
__device__ __forceinline__ void select_sweep(const uint32_t (&key)[KPT], int M, uint32_t T, int need_eq, SelectLds<KPT> &sh, Emit &&emit)
{
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    // ---- ordered sweep: stable compaction of kept and pruned indices.  Keys above T and keys equal to T are
    // counted together (low and high half): the kept keys before index i are those above T plus the first
    // need_eq of those equal to it.
    const unsigned long long below = (1ull << lane) - 1ull;
    unsigned long long mg[KPT], me[KPT];
#pragma unroll
    for (int j = 0; j < KPT; ++j) {
        const bool valid = j * kSelThreads + tid < M;
        mg[j] = __ballot(valid && key[j] > T);
        me[j] = __ballot(valid && key[j] == T);
        if (lane == 0) sh.counts[j * kSelWaves + wave] = __popcll(mg[j]) | __popcll(me[j]) << 16;
    }
    __syncthreads();
    int carry = 0;
#pragma unroll
    for (int j0 = 0; j0 < KPT; j0 += 4) {                // 64 pieces of 64 tokens at a time
        const int mine = j0 * kSelWaves + lane < KPT * kSelWaves ? sh.counts[j0 * kSelWaves + lane] : 0;
        const int incl = wave_running(mine);
        const int before = incl - mine + carry;
        carry += __builtin_amdgcn_readlane(incl, 63);
#pragma unroll
        for (int j = j0; j < min(j0 + 4, KPT); ++j) {
            const int i = j * kSelThreads + tid;
            const int piece = __builtin_amdgcn_readlane(before, (j - j0) * kSelWaves + wave);
            const int gt_before = (piece & 0xffff) + __popcll(mg[j] & below);
            const int eq_before = (piece >> 16) + __popcll(me[j] & below);
            const bool keep = (mg[j] >> lane & 1) || ((me[j] >> lane & 1) && eq_before < need_eq);
            const int keep_pos = gt_before + min(eq_before, need_eq);
            if (i < M) emit(i, keep, keep_pos);
        }
    }
}

struct SelectStreamLds {
    int hist[256];
    int2 wave_tot[2][kSelWaves];
    uint32_t prefix;
    int remaining;
};

// More scores than registers hold: MSB-first radix select in four passes of 8 bits, the keys read from
// memory in each.
template <typename Key, typename Emit>
__device__ __forceinline__ void select_streamed(Key &&key_at, int M, int k, SelectStreamLds &sh, Emit &&emit)
{
    const int tid = threadIdx.x;
    if (tid == 0) { sh.prefix = 0u; sh.remaining = k; }

    // ---- radix select of the k-th largest key
    for (int pass = 0; pass < 4; ++pass) {
        const int shift = 24 - 8 * pass;
        if (tid < 256) sh.hist[tid] = 0;
        __syncthreads();
        const uint32_t prefix = sh.prefix;
        const int remaining = sh.remaining;
        // keys whose already-fixed high bits equal the prefix
        const uint32_t himask = (pass == 0) ? 0u : (0xffffffffu << (shift + 8));
        for (int i = tid; i < M; i += kSelThreads) {
            uint32_t key = key_at(i);
            if ((key & himask) == prefix) atomicAdd(&sh.hist[(key >> shift) & 0xffu], 1);
        }
        __syncthreads();
        if (tid < 64) {
            // lane l owns bins 255-4l .. 252-4l (descending); `above` = keys in higher bins
            int c[4], sum = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) { c[j] = sh.hist[255 - 4 * tid - j]; sum += c[j]; }
            int incl = sum;
#pragma unroll
            for (int o = 1; o < 64; o <<= 1) {
                int t = __shfl_up(incl, o);
                if (tid >= o) incl += t;
            }
            int run = incl - sum;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (run < remaining && remaining <= run + c[j]) {
                    sh.prefix = prefix | ((uint32_t)(255 - 4 * tid - j) << shift);
                    sh.remaining = remaining - run;
                }
                run += c[j];
            }
        }
        __syncthreads();
    }
    const uint32_t T = sh.prefix;      // k-th largest key
    const int need_eq = sh.remaining;  // how many keys == T are kept (the lowest indices)

    // ---- ordered sweep: stable compaction of kept and pruned indices.  Keys above T and keys equal to
    // T are counted together: the kept keys before index i are those above T plus the first need_eq of
    // those equal to it.  The wavefronts' counts alternate between two buffers, so a sweep takes one
    // barrier (four with a scan for each flag: 12.1 -> 11.3 us for 8 x 4096 scores, 5.4 -> 5.0 for 8 x 576).
    const int lane = tid & 63, wave = tid >> 6;
    int run_gt = 0, run_eq = 0;
    for (int base = 0, it = 0; base < M; base += kSelThreads, ++it) {
        const int i = base + tid;
        const bool valid = i < M;
        const uint32_t key = valid ? key_at(i) : 0u;
        const bool eq = valid && key == T, gt = valid && key > T;
        const unsigned long long me = __ballot(eq), mg = __ballot(gt), below = (1ull << lane) - 1ull;
        if (lane == 0) sh.wave_tot[it & 1][wave] = make_int2(__popcll(mg), __popcll(me));
        __syncthreads();
        int gt_before = run_gt + __popcll(mg & below), eq_before = run_eq + __popcll(me & below);
#pragma unroll
        for (int w = 0; w < kSelWaves; ++w) {
            const int2 t = sh.wave_tot[it & 1][w];
            if (w < wave) { gt_before += t.x; eq_before += t.y; }
            run_gt += t.x;
            run_eq += t.y;
        }
        const bool keep = gt || (eq && eq_before < need_eq);
        const int keep_pos = gt_before + min(eq_before, need_eq);
        if (valid) emit(i, keep, keep_pos);
    }
}

}  // namespace fvar
