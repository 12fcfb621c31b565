// Attention over a key/value cache held in 8 bits (format and layout: kvb.hip).
//   o[b,i,h,:] = sum_t p_t V[b,t,h',:],  p = softmax over the visible t of scale * q[b,i,h,:] . K[b,t,h',:],
//   h' = h / (H / heads); t is visible when t < length of sample b and mask[b][t] != 0; o = 0 where nothing is visible.
//   weights[b,h',t] = the sum of p_t over the queries i and the query heads h of h'.
//
// The query heads of one kv head are further rows of the same problem: row r of a (sample, kv head) is query r / G of
// query head h' * G + r % G, G = H / heads.
#include <type_traits>

#include "kvb.h"

namespace fvar {

typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));
typedef short shortx4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) shortx4_t lds_shortx4_t;

// Values as fp16 operands: a value goes in as value * 2^(kTop - E), E the largest exponent of a tile seen so far and kRoom more (sums are
// rescaled when a tile's exceeds E, which is seldom).  A value is at most 448, and fp16 numbers reach down to 2^-24, so tiles are exact
// down to 2^-19 of the largest one's size, and 0 below 2^-37.  Weights go in as p * 2^kShift, with a reference that may be up to 2^kLag below the true
// maximum.  Next to bf16 operands the weights keep 11 bits, so that the output's own rounding is the only one of note.
// fp32 takes values as they are in bf16, exact, up to tiles of 2^64, and at 2^64 over E from there on: a sum of weights up to 2^7 each stays finite.
constexpr int kTop = 6, kRoom = 2, kLarge = 64;
constexpr float kShift = 8.f, kLag = 7.f;

__device__ __forceinline__ uint4 half_eight(uint32_t a, uint32_t b, float s)
{
    return make_uint4(kvb_f16<0>(a, s), kvb_f16<1>(a, s), kvb_f16<0>(b, s), kvb_f16<1>(b, s));
}
__device__ __forceinline__ uint4 bf16_eight(uint32_t a, uint32_t b, float s)
{
    return make_uint4(kvb_bf16<0>(a, s), kvb_bf16<1>(a, s), kvb_bf16<0>(b, s), kvb_bf16<1>(b, s));
}
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((uint32_t)min(max(e + 127, 0), 254) << 23); }

// the same value in the lanes of a column group: 16 and 32 lanes apart
__device__ __forceinline__ float column_max(float v)
{
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float column_sum(float v)
{
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}
// What is taken off scores whose largest is m: m, or 0 where nothing finite has been seen and all scores are -inf
__device__ __forceinline__ float reference(float m) { return m == -INFINITY ? 0.f : m; }

// Three bf16 numbers that add up to an fp32 one: its bits from the top (no rounding, so no overflow either).
__device__ __forceinline__ void three_pieces(const float *x, bf16x8_t *out)
{
    uint32_t w[3][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float a = x[2 * i], b = x[2 * i + 1];
#pragma unroll
        for (int p = 0; p < 3; ++p) {
            const uint32_t ha = __float_as_uint(a) & 0xffff0000u, hb = __float_as_uint(b) & 0xffff0000u;
            w[p][i] = (ha >> 16) | hb;
            a -= __uint_as_float(ha);
            b -= __uint_as_float(hb);
        }
    }
#pragma unroll
    for (int p = 0; p < 3; ++p) out[p] = __builtin_bit_cast(bf16x8_t, make_uint4(w[p][0], w[p][1], w[p][2], w[p][3]));
}

template <typename T> struct Quad;                           // four consecutive results
template <> struct Quad<uint16_t> {
    __device__ static __forceinline__ void store(uint16_t *p, float4 v)
    {
        *reinterpret_cast<uint2 *>(p) = make_uint2(pack_bf16x2(v.x, v.y), pack_bf16x2(v.z, v.w));
    }
};
template <> struct Quad<float> {
    __device__ static __forceinline__ void store(float *p, float4 v) { *reinterpret_cast<float4 *>(p) = v; }
};

// Workgroup `id` -> one of `groups` groups of `size`: the workgroups of a group on one XCD (id % 8), whose L2 they share, and neighbouring
// groups on different ones, so that long samples next to each other do not meet on one.
__device__ __forceinline__ int xcd_grouped(int id, int groups, int size)
{
    const int even = groups & ~7;                            // the last few groups stay as they are numbered
    if (id >= even * size) return id;
    const int pos = id >> 3;
    return (pos / size * 8 + (id & 7)) * size + pos % size;
}

// Sixteen rows per workgroup, whose wavefronts take every NW-th tile of 32 keys, a block of the cache, of the workgroup's share [t0, t1) of the
// key axis, each with a softmax of its own, and meet in LDS at the end.  For the rows of one query or a few, where the
// cache's way from memory is what counts (each wavefront fetches a tile ahead, no barrier in the loop), and for fp32.
//   S^T = K Q^T by 16x16x32 MFMAs: a lane holds a quarter of one key as it lies in memory, converts it to bf16 (exact) and
//     multiplies eight elements at a time; Q follows that order.
//   O^T = V^T P^T: a lane takes pieces of sixteen values as they lie in memory, converts them and leaves them in LDS row by
//     row, from where the transposing load brings eight keys of one head-dim element; P is in that order already.
// fp32: Q and P go in as three bf16 numbers each, K and V are exact in one.
// stats: null, or for every row what its weights were taken against: reference and sum.
template <typename T, int DH, int NW, bool MASKED>
__global__ __launch_bounds__(64 * NW, 2) void kvb_attn_rows_kernel(const T *__restrict__ q, int ld, KvbCache c, int extra,
                                                                int n, int H, float c_log2, T *__restrict__ o,
                                                                int nrb, int splits, float *__restrict__ part_o,
                                                                float *__restrict__ part_ml, float2 *__restrict__ stats)
{
    constexpr bool F32 = sizeof(T) == 4;
    constexpr int NP = F32 ? 3 : 1;
    constexpr int KS = DH / 32, DB = DH / 16;                // steps of S, 16-row blocks of O^T
    constexpr int KW = DH / 64;                              // sixteen bytes of a key per lane
    constexpr int VL = DH / 32, VP = DH / 16;                // pieces of values per lane, and of a row
    __shared__ uint4 vlds[NW][32 * DH / 8];                  // a tile of values; at the end the partial results
    __shared__ float2 ml[NW][16];

    const int tid = threadIdx.x, lane = tid & 63, c16 = lane & 15, g4 = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int unit = xcd_grouped(blockIdx.x, (int)(gridDim.x / nrb), nrb);
    const int rb = unit % nrb;
    unit /= nrb;
    const int split = unit % splits;
    unit /= splits;
    const int hk = unit % c.heads, b = unit / c.heads;
    const int G = H / c.heads, R = n * G;
    const int len = kvb_length(c, b, extra);
    const int tiles = (len + 31) / 32;
    // (products below 2^30: at most 2^19 tiles and 1024 shares)
    const int t0 = tiles * split / splits, t1 = tiles * (split + 1) / splits;
    const int last = max(tiles - 1, 0), last_row = max(len - 1, 0);

    // ---- Q: lane = row, the elements of the lane's part of a key
    const int row = min(rb * 16 + c16, R - 1);
    const T *qsrc = q + (size_t)(b * (long)n + row / G) * ld + (size_t)(hk * G + row % G) * DH + g4 * (DH / 4);
    bf16x8_t qf[KS][NP];
#pragma unroll
    for (int s = 0; s < KS; ++s) {
        if constexpr (F32) {
            float x[8];
            *reinterpret_cast<float4 *>(x) = *reinterpret_cast<const float4 *>(qsrc + 8 * s);
            *reinterpret_cast<float4 *>(x + 4) = *reinterpret_cast<const float4 *>(qsrc + 8 * s + 4);
            three_pieces(x, qf[s]);
        } else {
            qf[s][0] = *reinterpret_cast<const bf16x8_t *>(qsrc + 8 * s);
        }
    }

    const size_t head = (size_t)(b * c.heads + hk);
    const uint8_t *Kc = c.k + head * c.capacity * DH, *Vc = c.v + head * c.capacity * DH;
    const uint8_t *Ks = c.k_scale + head * c.blocks(), *Vs = c.v_scale + head * c.blocks();
    const uint8_t *mask = MASKED ? c.mask + (size_t)b * c.capacity : nullptr;

    struct Tile {
        uint4 k[2][KW], v[VL];
        uint32_t ks, vs, vis;                                // vis: with a mask, the keys that are seen; otherwise whether the lane's is
    };
    // Mask bytes come a tile before the rows that they let pass: instead of a hidden row, the first of the tile that is seen is fetched
    // again.
    uint32_t ahead = 0;
    auto fetch_mask = [&](int t) {
        if constexpr (MASKED) ahead = mask[min(min(t, last) * 32 + (lane & 31), last_row)];
    };
    auto fetch = [&](int t, Tile &x) {
        const int at = min(t, last), base = at * 32;
        if constexpr (MASKED) x.vis = (uint32_t)__ballot(base + (lane & 31) < len && ahead != 0);
        const int first = MASKED && x.vis ? __builtin_ctz(x.vis) : 0;
        auto place = [&](int i) { return (uint32_t)min(base + (!MASKED || (x.vis >> i & 1) ? i : first), last_row); };
        fetch_mask(t + NW);
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const uint32_t key = place(16 * u + c16);
#pragma unroll
            for (int w = 0; w < KW; ++w) x.k[u][w] = *reinterpret_cast<const uint4 *>(Kc + key * DH + g4 * (DH / 4) + 16 * w);
        }
#pragma unroll
        for (int j = 0; j < VL; ++j)
            x.v[j] = *reinterpret_cast<const uint4 *>(Vc + place((64 * j + lane) / VP) * DH + lane % VP * 16);
        x.ks = Ks[at];
        x.vs = Vs[at];
        if constexpr (!MASKED) x.vis = base + (lane & 31) < len;
    };

    // ---- LDS: 32-byte pieces of a row are turned by its number, so that eight rows' pieces of one column lie in different banks
    uint16_t *vl = reinterpret_cast<uint16_t *>(vlds[wave]);
    auto turn = [](int key) { return DH == 128 ? key & 7 : (key >> 1) & 3; };
    const int rrow = 4 * g4 + ((lane >> 2) & 3);             // transposing load: the lane's row and four elements of it
    const int rturn = turn(rrow), rbase = rrow * DH + (lane & 3) * 4;

    floatx4_t acc[DB];
#pragma unroll
    for (int i = 0; i < DB; ++i) acc[i] = floatx4_t{0};
    float m_ref = -INFINITY, l_run = 0.f;
    const float lag = fminf(kLag / c_log2, 3e38f);           // (finite: any score is more than that above none)
    constexpr int TOP = F32 ? kLarge : kTop, NONE = F32 ? kLarge : -200;
    int E = NONE, acc_E = NONE;                              // of the values, of the sums

    // A tile's keys and values are converted first; the next one's are then fetched into the same registers, under the softmax and the
    // products.  A wavefront without a tile looks at one in which it sees nothing.
    Tile x;
    int t = t0 + wave;
    fetch_mask(t);
    fetch(t, x);
    do {
        const uint32_t vis = MASKED ? (t < t1 ? x.vis : 0) : (uint32_t)__ballot(x.vis != 0 && t < t1);
        // A tile without a visible key is passed over.
        const bool any = vis != 0;
        floatx4_t s[2];
        if (any) {
            // ---- S^T: lane (c16, g4) gets the keys 4 g4 .. + 3 and 16 more of row c16
            const float ksize = __uint_as_float(x.ks << 23);
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                s[u] = floatx4_t{0};
#pragma unroll
                for (int i = 0; i < KS; ++i) {
                    const uint4 w = x.k[u][i / 2];
                    const bf16x8_t kf = __builtin_bit_cast(bf16x8_t, i & 1 ? bf16_eight(w.z, w.w, ksize) : bf16_eight(w.x, w.y, ksize));
#pragma unroll
                    for (int p = NP - 1; p >= 0; --p)
                        s[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[i][p], s[u], 0, 0, 0);
                }
            }
            // ---- values to LDS
            const int ve = (int)__builtin_amdgcn_readfirstlane((int)x.vs) - 127;
            if (__builtin_expect(ve > E, 0)) E = ve + kRoom;
            const float vsize = power_of_two(ve - E + TOP);
#pragma unroll
            for (int j = 0; j < VL; ++j) {
                const int key = (64 * j + lane) / VP, piece = (lane % VP) ^ turn(key);
                uint4 w = x.v[j];
                if (__builtin_expect(vis != ~0u, 0) && !(vis >> key & 1)) w = make_uint4(0, 0, 0, 0);
                uint4 *dst = reinterpret_cast<uint4 *>(vl + key * DH + piece * 16);
                dst[0] = F32 ? bf16_eight(w.x, w.y, vsize) : half_eight(w.x, w.y, vsize);
                dst[1] = F32 ? bf16_eight(w.z, w.w, vsize) : half_eight(w.z, w.w, vsize);
            }
        }
        t += NW;
        fetch(t, x);
        if (any) {
            // ---- softmax
            if (__builtin_expect(vis != ~0u, 0)) {
                const uint32_t mine = vis >> (4 * g4);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (!(mine >> i & 1)) s[0][i] = -INFINITY;
                    if (!(mine >> (16 + i) & 1)) s[1][i] = -INFINITY;
                }
            }
            const float mx = fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])), fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3])));
            const bool lags = __builtin_amdgcn_ballot_w64(mx - m_ref > lag) != 0 || E != acc_E;
            if (__builtin_expect(lags, 0)) {
                const float now = column_max(fmaxf(m_ref, mx));
                const float alpha = __builtin_amdgcn_exp2f((m_ref - reference(now)) * c_log2);
                const float down = __builtin_amdgcn_ldexpf(alpha, max(acc_E - E, -200));
                m_ref = now;
                acc_E = E;
                l_run *= alpha;
#pragma unroll
                for (int i = 0; i < DB; ++i) {
                    acc[i] *= down;
                    asm volatile("" : "+v"(acc[i]));
                }
            }
            const float fin = reference(m_ref);
            float p[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                // the difference first: exact near the reference, however large the scores
                const float y = s[i >> 2][i & 3] - fin;
                p[i] = __builtin_amdgcn_exp2f(F32 ? y * c_log2 : fmaf(y, c_log2, kShift));
                l_run += p[i];
            }
            // ---- O^T += V^T P^T
            bf16x8_t pf[NP];
            f16x8_t ph;
            if constexpr (F32) {
                three_pieces(p, pf);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) ph[i] = (_Float16)p[i];
            }
            asm volatile("" ::: "memory");
            shortx4_t v[DB][2];
#pragma unroll
            for (int i = 0; i < DB; ++i) {
                const uint16_t *src = vl + rbase + ((i ^ rturn) << 4);
                v[i][0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4_t *)src);
                v[i][1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4_t *)(src + 16 * DH));
            }
#pragma unroll
            for (int i = 0; i < DB; ++i) {
                const auto both = __builtin_shufflevector(v[i][0], v[i][1], 0, 1, 2, 3, 4, 5, 6, 7);
                if constexpr (F32) {
#pragma unroll
                    for (int k = NP - 1; k >= 0; --k)
                        acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, both), pf[k], acc[i], 0, 0, 0);
                } else {
                    acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8_t, both), ph, acc[i], 0, 0, 0);
                }
            }
            asm volatile("" ::: "memory");
        }
    } while (t < t1);

    // ---- the wavefronts' results: each as the mean of the values it saw, with its weight l at the reference m
    l_run = column_sum(l_run);
    const float inv = l_run == 0.f ? 0.f : 1.0f / l_run;
    float4 *slots = reinterpret_cast<float4 *>(vlds[wave]);
#pragma unroll
    for (int i = 0; i < DB; ++i) {
        float4 v = make_float4(acc[i][0] * inv, acc[i][1] * inv, acc[i][2] * inv, acc[i][3] * inv);
        // back to its size, which may be any
        v.x = __builtin_amdgcn_ldexpf(v.x, acc_E - TOP); v.y = __builtin_amdgcn_ldexpf(v.y, acc_E - TOP);
        v.z = __builtin_amdgcn_ldexpf(v.z, acc_E - TOP); v.w = __builtin_amdgcn_ldexpf(v.w, acc_E - TOP);
        slots[i * 64 + lane] = v;
    }
    if (g4 == 0) ml[wave][c16] = make_float2(m_ref, l_run);
    __syncthreads();
    float m = ml[0][c16].x;
#pragma unroll
    for (int w = 1; w < NW; ++w) m = fmaxf(m, ml[w][c16].x);
    const float fin = reference(m);
    float wgt[NW], sum = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
        wgt[w] = ml[w][c16].y * __builtin_amdgcn_exp2f((ml[w][c16].x - fin) * c_log2);
        sum += wgt[w];
    }
    const float each = sum == 0.f ? 0.f : 1.0f / sum;
    if (rb * 16 + c16 >= R) return;
    const size_t prow = (((size_t)head * nrb + rb) * splits + split) * 16 + c16;
    T *dst = o + (size_t)(b * (long)n + row / G) * H * DH + (size_t)(hk * G + row % G) * DH;
    for (int i = wave; i < DB; i += NW) {
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            const float4 x = reinterpret_cast<const float4 *>(vlds[w])[i * 64 + lane];
            const float k = wgt[w] * each;
            v.x = fmaf(x.x, k, v.x); v.y = fmaf(x.y, k, v.y); v.z = fmaf(x.z, k, v.z); v.w = fmaf(x.w, k, v.w);
        }
        if (splits > 1) *reinterpret_cast<float4 *>(part_o + prow * DH + 16 * i + 4 * g4) = v;
        else Quad<T>::store(dst + 16 * i + 4 * g4, v);
    }
    if (wave == 0 && g4 == 0) {
        if (splits > 1) *reinterpret_cast<float2 *>(part_ml + prow * 2) = make_float2(m, sum);
        else if (stats) stats[head * R + row] = make_float2(m, F32 ? sum : sum * 0.00390625f);   // (without 2^kShift)
    }
}

// The shares of rows joined: each is a mean and its weight.  A unit is a block of BR rows of one (sample, kv head); the shares
// of unit first + u lie at [u][share][row].  GROUPS groups of DH/4 threads per row, four head-dim elements a thread: a group takes every
// GROUPS-th share, four at a time, with a running reference and mean (not the sum: a mean times its weight need not be a number that fp32
// holds), and the groups meet in LDS.  One group where the shares are few and the
// rows many; more where a few rows have many shares, whose loads would wait for each other (64 shares of 16 rows: 24 us by one, 3 by 8).
template <typename T, int DH, int GROUPS>
__global__ __launch_bounds__(256) void kvb_attn_merge_kernel(const float *__restrict__ part_o, const float *__restrict__ part_ml,
                                                             int n, int H, int heads, int nrb, int BR, int first, int shares,
                                                             float c_log2, int total, T *__restrict__ o, float2 *__restrict__ stats)
{
    constexpr int W = DH / 4, ROWS = 256 / (W * GROUPS);     // threads of a group, rows of a workgroup
    __shared__ float4 lo[GROUPS > 1 ? 256 : 1];
    __shared__ float2 lm[GROUPS > 1 ? 256 / W : 1];
    const int d = threadIdx.x % W * 4, group = threadIdx.x / W % GROUPS, in_wg = threadIdx.x / (W * GROUPS);
    const int idx = blockIdx.x * ROWS + in_wg;               // row among those of the divided units
    const int r = idx % BR, u = idx / BR, unit = first + u;
    const int G = H / heads, row = unit % nrb * BR + r, hk = unit / nrb % heads;
    const long b = unit / nrb / heads;
    const bool mine = idx < total && row < n * G;
    const size_t prow = (size_t)u * shares * BR + r;
    auto weight = [&](float2 ml, float m) { return ml.y * __builtin_amdgcn_exp2f((ml.x - reference(m)) * c_log2); };
    float m = -INFINITY, sum = 0.f;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    auto add = [&](float4 v, float w) {
        acc.x = fmaf(v.x, w, acc.x); acc.y = fmaf(v.y, w, acc.y); acc.z = fmaf(v.z, w, acc.z); acc.w = fmaf(v.w, w, acc.w);
    };
    if (mine) {
        for (int s = group; s < shares; s += 4 * GROUPS) {
            float2 ml[4];
            float4 v[4];
            float now = m, w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const bool there = s + i * GROUPS < shares;  // (instead of one that is not, the first with a weight of 0)
                const size_t at = prow + (size_t)(there ? s + i * GROUPS : s) * BR;
                ml[i] = *reinterpret_cast<const float2 *>(part_ml + at * 2);
                v[i] = *reinterpret_cast<const float4 *>(part_o + at * DH + d);
                if (!there) ml[i].y = 0.f;
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) now = fmaxf(now, ml[i].x);
            const float before = weight(make_float2(m, sum), now);
            sum = before;
#pragma unroll
            for (int i = 0; i < 4; ++i) sum += w[i] = weight(ml[i], now);
            const float each = sum == 0.f ? 0.f : 1.0f / sum, keep = before * each;
            acc.x *= keep; acc.y *= keep; acc.z *= keep; acc.w *= keep;
#pragma unroll
            for (int i = 0; i < 4; ++i) add(v[i], w[i] * each);
            m = now;
        }
    }
    if constexpr (GROUPS > 1) {
        lo[threadIdx.x] = acc;
        if (d == 0) lm[threadIdx.x / W] = make_float2(m, sum);
        __syncthreads();
        if (group) return;
#pragma unroll
        for (int k = 1; k < GROUPS; ++k) m = fmaxf(m, lm[threadIdx.x / W + k].x);
        sum = 0.f;
#pragma unroll
        for (int k = 0; k < GROUPS; ++k) sum += weight(lm[threadIdx.x / W + k], m);
        const float each = sum == 0.f ? 0.f : 1.0f / sum;
        acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int k = 0; k < GROUPS; ++k) add(lo[threadIdx.x + k * W], weight(lm[threadIdx.x / W + k], m) * each);
    }
    if (mine) {
        Quad<T>::store(o + (size_t)(b * n + row / G) * H * DH + (size_t)(hk * G + row % G) * DH + d, acc);
        if (stats && d == 0) stats[(size_t)(unit / nrb) * n * G + row] = make_float2(m, sizeof(T) == 4 ? sum : sum * 0.00390625f);
    }
}

// Weights of the rows: every wavefront holds 64 keys as bf16 operands, takes the scores of all rows of queries against them once more, and
// adds up exp2((s - reference) * c - log2(sum)) over the rows, each key's in its own registers: no atomics, one order.  32 rows at a time come
// through LDS for the four wavefronts, the next ones on their way.  A row whose weights are not numbers adds nothing.
//   grid: (blocks of 256 keys, B * heads, shares of the rows); shares: as partial sums [share][B * heads][256 * gridDim.x].
template <typename T, int DH>
__global__ __launch_bounds__(256, 2) void kvb_weights_kernel(const T *__restrict__ q, int ld, KvbCache c, int extra, int n, int H, float c_log2,
                                                             const float2 *__restrict__ stats, float *__restrict__ weights, int add,
                                                             float *__restrict__ part)
{
    constexpr bool F32 = sizeof(T) == 4;
    constexpr int NP = F32 ? 3 : 1, KS = DH / 16, CH = DH / 8, PER = 32 * CH / 256;   // PER: chunks of eight elements per thread
    __shared__ uint4 ql[2][NP][32 * CH];
    const int tid = threadIdx.x, lane = tid & 63, rl = lane & 31, g = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int head = blockIdx.y, b = head / c.heads, hk = head % c.heads;
    const int G = H / c.heads, R = n * G, len = kvb_length(c, b, extra);
    const int key0 = blockIdx.x * 256 + wave * 64;
    if ((int)blockIdx.x * 256 >= len) return;                // (of the whole workgroup)
    const int tiles = (R + 31) / 32, t0 = (int)((long)tiles * blockIdx.z / gridDim.z), t1 = (int)((long)tiles * (blockIdx.z + 1) / gridDim.z);

    // ---- keys: lane = key, half a row
    bf16x8_t kf[2][KS];
    const uint8_t *Kc = c.k + (size_t)head * c.capacity * DH, *Ks = c.k_scale + (size_t)head * c.blocks();
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const int key = min(key0 + 32 * u + rl, len - 1);
        const float size = __uint_as_float((uint32_t)Ks[min(key0 + 32 * u, len - 1) / kKvbBlock] << 23);
#pragma unroll
        for (int s = 0; s < KS; s += 2) {
            const uint4 w = *reinterpret_cast<const uint4 *>(Kc + (size_t)key * DH + g * (DH / 2) + 8 * s);
            kf[u][s] = __builtin_bit_cast(bf16x8_t, bf16_eight(w.x, w.y, size));
            kf[u][s + 1] = __builtin_bit_cast(bf16x8_t, bf16_eight(w.z, w.w, size));
        }
    }

    // ---- rows of queries: chunks are turned by the row's number, so that the rows of sixteen lanes that read one chunk lie in all banks
    auto place = [](int row, int chunk) { return row * CH + (chunk ^ (DH == 128 ? row & 15 : (row >> 1) & 7)); };
    uint4 next[PER][F32 ? 2 : 1];
    float2 next_stat;
    auto fetch = [&](int t) {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int at = i * 256 + tid, row = min(t * 32 + at / CH, R - 1);
            const T *src = q + (size_t)(b * (long)n + row / G) * ld + (size_t)(hk * G + row % G) * DH + at % CH * 8;
            next[i][0] = *reinterpret_cast<const uint4 *>(src);
            if constexpr (F32) next[i][1] = *reinterpret_cast<const uint4 *>(src + 4);
        }
        next_stat = stats[(size_t)head * R + min(t * 32 + rl, R - 1)];
    };
    auto put = [&](int buffer) {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int at = i * 256 + tid, to = place(at / CH, at % CH);
            if constexpr (F32) {
                float x[8];
                bf16x8_t pieces[3];
                Elem<float>::unpack(next[i][0], x);
                Elem<float>::unpack(next[i][1], x + 4);
                three_pieces(x, pieces);
#pragma unroll
                for (int p = 0; p < 3; ++p) ql[buffer][p][to] = __builtin_bit_cast(uint4, pieces[p]);
            } else {
                ql[buffer][0][to] = next[i][0];
            }
        }
    };

    floatx16_t acc[2] = {floatx16_t{0}, floatx16_t{0}};
    if (t0 < t1) {
        fetch(t0);
        put(0);
    }
    for (int t = t0; t < t1; ++t) {
        const float2 stat = next_stat;
        const int buffer = (t - t0) & 1;
        __syncthreads();                                     // this tile's rows are there, the other buffer has been read
        if (t + 1 < t1) fetch(t + 1);
        floatx16_t s[2] = {floatx16_t{0}, floatx16_t{0}};
#pragma unroll
        for (int i = 0; i < KS; ++i) {
#pragma unroll
            for (int p = NP - 1; p >= 0; --p) {
                const bf16x8_t qf = __builtin_bit_cast(bf16x8_t, ql[buffer][p][place(rl, g * KS + i)]);
#pragma unroll
                for (int u = 0; u < 2; ++u) s[u] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[u][i], qf, s[u], 0, 0, 0);
            }
        }
        const bool counts = t * 32 + rl < R && stat.y > 0.f;
        const float m = counts ? reference(stat.x) : 0.f, off = counts ? -__builtin_amdgcn_logf(stat.y) : -INFINITY;
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const float x = fmaf(s[u][i] - m, c_log2, off);
                // (at most 1: scores of 2^20 and more differ by more than that between two ways to add their products up)
                acc[u][i] += __builtin_amdgcn_fmed3f(__builtin_amdgcn_exp2f(x), 0.f, 1.f);
            }
        if (t + 1 < t1) put(buffer ^ 1);
    }

    // ---- sums over the rows of a tile: 32 lanes; the lane then takes one key
    float mine = 0.f;
    const int mu = rl >> 4, mi = rl & 15;
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            float v = acc[u][i];
            v += __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(v), 0xb1, 0xf, 0xf, true));    // quad_perm 1,0,3,2
            v += __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(v), 0x4e, 0xf, 0xf, true));    // quad_perm 2,3,0,1
            v += __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(v), 0x141, 0xf, 0xf, true));   // row_half_mirror
            v += __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(v), 0x140, 0xf, 0xf, true));   // row_mirror
            const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
            v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
            if (mu == u && mi == i) mine = v;
        }
    const int key = key0 + 32 * mu + 8 * (mi >> 2) + 4 * g + (mi & 3);
    if (key >= len) return;
    if (c.mask && c.mask[(size_t)b * c.capacity + key] == 0) mine = 0.f;
    if (gridDim.z > 1) {
        part[((size_t)blockIdx.z * gridDim.y + head) * (256 * gridDim.x) + key] = mine;
        return;
    }
    float *to = weights + (size_t)head * c.capacity + key;
    *to = add ? *to + mine : mine;
}

__global__ __launch_bounds__(256) void kvb_weights_join_kernel(KvbCache c, int extra, const float *__restrict__ part, int pitch, int shares,
                                                               float *__restrict__ weights, int add)
{
    const int key = blockIdx.x * 256 + threadIdx.x, head = blockIdx.y;
    if (key >= kvb_length(c, head / c.heads, extra)) return;
    float sum = 0.f;
    for (int i = 0; i < shares; ++i) sum += part[((size_t)i * gridDim.y + head) * pitch + key];
    float *to = weights + (size_t)head * c.capacity + key;
    *to = add ? *to + sum : sum;
}

// nrb blocks per (sample, kv head), units in all, of which the first `full` take all keys and each other one is divided into `shares`.
// `ragged`: samples of lengths of their own, which only the GPU knows.  waves: wavefronts of a workgroup.
struct KvbRun { int block, nrb, units, full, shares, waves; };
static KvbRun kvb_run(int block, int B, int n, int H, int heads, int length, bool ragged)
{
    KvbRun run;
    run.block = block;
    run.nrb = (n * (H / heads) + block - 1) / block;
    run.units = B * heads * run.nrb;
    run.waves = 4;
    const int tiles = (length + 31) / 32;
    const int places = ragged ? 1024 : 512, least = run.units < 256 ? 2 : 8;
    const int want = (places + run.units - 1) / run.units, most = tiles / (least * 4);
    run.shares = want < most ? want : most > 0 ? most : 1;
    run.full = run.shares > 1 ? 0 : run.units;
    return run;
}

// Shares of the rows of queries for the weights: where the keys alone do not fill the chip.
constexpr int kWeightPlaces = 512;
static int weight_shares(int B, int heads, int length, int rows)
{
    const long wgs = (long)B * heads * ((length + 255) / 256);
    long shares = wgs > 0 ? kWeightPlaces / wgs : 1;
    if (shares > (rows + 31) / 32) shares = (rows + 31) / 32;
    return (int)(shares > 8 ? 8 : shares < 1 ? 1 : shares);
}

size_t kvb_attention_scratch_floats(DType dt, int B, int n, int H, int heads, int Dh, int capacity, bool weights)
{
    const KvbRun run = kvb_run(16, B, n, H, heads, capacity, true);
    size_t floats = (size_t)(run.units - run.full) * run.shares * run.block * (Dh + 2);
    // every row's reference and sum; partial sums of at most kWeightPlaces workgroups of 256 keys
    if (weights) floats += 2 * (size_t)B * n * H + 256 * kWeightPlaces;
    return floats;
}

template <typename T, int DH>
static void launch_kvb(const void *q, int ld, const KvbCache &c, int extra, int B, int n, int H, float c_log2, void *o, float *weights, bool add,
                       float *part, hipStream_t st)
{
    const int length = c.lens ? c.capacity : c.len + extra;
    const KvbRun run = kvb_run(16, B, n, H, c.heads, length, c.lens != nullptr);
    const int divided = run.units - run.full;
    float2 *stats = nullptr;
    float *sums = part;
    if (weights) {
        stats = reinterpret_cast<float2 *>(part);
        sums = part + 2 * (size_t)B * n * H;
        part = sums + 256 * kWeightPlaces;
    }
    float *part_ml = part + (size_t)divided * run.shares * run.block * DH;
    const unsigned wgs = (unsigned)(run.full + divided * run.shares);
#define FVAR_ROWS(NW, MASKED)                                                                                            \
    launch(kvb_attn_rows_kernel<T, DH, NW, MASKED>, dim3(wgs), dim3(64 * NW), 0, st, (const T *)q, ld, c, extra, n, H,    \
           c_log2, (T *)o, run.nrb, run.shares, part, part_ml, stats)
    if (c.mask) FVAR_ROWS(4, true);
    else FVAR_ROWS(4, false);
#undef FVAR_ROWS
    if (divided) {
        const int total = divided * run.block, per = 256 / (DH / 4);
        if (run.shares > 8)
            launch(kvb_attn_merge_kernel<T, DH, 8>, dim3((unsigned)((total + per / 8 - 1) / (per / 8))), dim3(256), 0, st, (const float *)part,
                   (const float *)part_ml, n, H, c.heads, run.nrb, run.block, run.full, run.shares, c_log2, total, (T *)o, stats);
        else
            launch(kvb_attn_merge_kernel<T, DH, 1>, dim3((unsigned)((total + per - 1) / per)), dim3(256), 0, st, (const float *)part,
                   (const float *)part_ml, n, H, c.heads, run.nrb, run.block, run.full, run.shares, c_log2, total, (T *)o, stats);
    }
    if (weights && length > 0) {
        const int blocks = (length + 255) / 256, shares = weight_shares(B, c.heads, length, n * (H / c.heads));
        launch(kvb_weights_kernel<T, DH>, dim3((unsigned)blocks, (unsigned)(B * c.heads), (unsigned)shares), dim3(256), 0, st, (const T *)q, ld, c,
               extra, n, H, c_log2, (const float2 *)stats, weights, add ? 1 : 0, sums);
        if (shares > 1)
            launch(kvb_weights_join_kernel, dim3((unsigned)blocks, (unsigned)(B * c.heads)), dim3(256), 0, st, c, extra, (const float *)sums,
                   256 * blocks, shares, weights, add ? 1 : 0);
    }
}

void launch_kvb_attention(DType dt, const void *q, int ld, const KvbCache &c, int extra, int B, int n, int H, int Dh,
                          float scale, void *o, float *weights, bool add, float *part, hipStream_t st)
{
    const float c_log2 = scale * 1.4426950408889634f;
    if (dt == DType::BF16) {
        if (Dh == 64) launch_kvb<uint16_t, 64>(q, ld, c, extra, B, n, H, c_log2, o, weights, add, part, st);
        else launch_kvb<uint16_t, 128>(q, ld, c, extra, B, n, H, c_log2, o, weights, add, part, st);
    } else {
        if (Dh == 64) launch_kvb<float, 64>(q, ld, c, extra, B, n, H, c_log2, o, weights, add, part, st);
        else launch_kvb<float, 128>(q, ld, c, extra, B, n, H, c_log2, o, weights, add, part, st);
    }
}

}  // namespace fvar
