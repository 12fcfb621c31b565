// Attention over a key/value cache held in 4 bits (format and layout: kvq.hip).
//   o[b,i,h,:] = sum_t p_t V[b,t,h',:],  p = softmax over the visible t of scale * q[b,i,h,:] . K[b,t,h',:],
//   h' = h / (H / heads); t is visible when t < length of sample b and mask[b][t] != 0; o = 0 where nothing is visible.
//
// The query heads of one kv head are further rows of the same problem: row r of a (sample, kv head) is query r / G of
// query head h' * G + r % G, G = H / heads.
#include <type_traits>

#include "common.h"

namespace fvar {

typedef _Float16 f16x2_t __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));
typedef short shortx4_t __attribute__((ext_vector_type(4)));
typedef int intx8_t __attribute__((ext_vector_type(8)));
typedef unsigned uintx4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) const uintx4_t lds_uintx4_t;
typedef unsigned uintx6_t __attribute__((ext_vector_type(6)));
typedef float floatx32_t __attribute__((ext_vector_type(32)));
typedef __attribute__((address_space(3))) shortx4_t lds_shortx4_t;
typedef __attribute__((address_space(3))) uint8_t lds_byte_t;

// Values as fp16 operands.  An fp16 number holds an element of the format times 2^-25 to 2^13, so a value goes in as
// value * 2^(kTop - E), E the largest scale byte seen so far and two more: sums are rescaled when a byte exceeds E, which is
// seldom, and blocks 2^-35 and less of the largest may vanish.  Weights go in as p * 2^8, with a reference that may be up to
// 2^7 below the true maximum.  Next to bf16 operands (any exponent, 8 bits) the weights keep 11 bits, so that the
// output's own rounding is the only one of note: 1.7e-3 against 2.4e-3 of the result.
// fp32 takes them as they are in bf16 up to blocks of 2^64, and at 2^64 over E from there on: a sum of weights up to 2^7 each stays finite.
constexpr int kTop = 13, kRoom = 2, kLarge = 127 + 64;
constexpr float kShift = 8.f, kLag = 7.f, kMost = 32768.f;

// The scale with which a block of scale byte `byte` is converted: E's goes in as 2^(top - 127).
__device__ __forceinline__ float value_scale(uint32_t byte, int E, int top, bool seen)
{
    const int e = (int)byte - E + top;
    return seen ? __uint_as_float(byte == 255 ? 0x7f800000u : (uint32_t)max(e, 0) << 23) : 0.f;
}

template <int W> __device__ __forceinline__ uint32_t half_pair(uint32_t word, float scale)
{
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(word, scale, W));
}
template <int W> __device__ __forceinline__ uint32_t bf16_pair(uint32_t word, float scale)
{
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale, W));
}
__device__ __forceinline__ uint4 half_eight(uint32_t w, float s)
{
    return make_uint4(half_pair<0>(w, s), half_pair<1>(w, s), half_pair<2>(w, s), half_pair<3>(w, s));
}
__device__ __forceinline__ uint4 bf16_eight(uint32_t w, float s)
{
    return make_uint4(bf16_pair<0>(w, s), bf16_pair<1>(w, s), bf16_pair<2>(w, s), bf16_pair<3>(w, s));
}

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
// the smaller of two 16-bit numbers each; of 32 lanes' numbers, in each of them
__device__ __forceinline__ uint32_t pair_min(uint32_t a, uint32_t b)
{
    typedef uint16_t uint16x2_t __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_min(__builtin_bit_cast(uint16x2_t, a), __builtin_bit_cast(uint16x2_t, b)));
}
__device__ __forceinline__ uint32_t half_min(uint32_t v)
{
    v = pair_min(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0xb1, 0xf, 0xf, true));       // quad_perm 1,0,3,2
    v = pair_min(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x4e, 0xf, 0xf, true));       // quad_perm 2,3,0,1
    v = pair_min(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x141, 0xf, 0xf, true));      // row_half_mirror
    v = pair_min(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x140, 0xf, 0xf, true));      // row_mirror
    const auto a = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    return pair_min(a[0], a[1]);
}
// What is taken off scores whose largest is m: m, or 0 where nothing finite has been seen and all scores are -inf
__device__ __forceinline__ float reference(float m) { return m == -INFINITY ? 0.f : m; }

__device__ __forceinline__ uint32_t wave_max(uint32_t v)
{
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, d));
    return __builtin_amdgcn_readfirstlane(v);
}

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
// groups on different ones, so that long samples next to each other do not meet on one.  (Contiguous shares of the numbering for
// each XCD: 79 us instead of 60 for 32 samples of 1 to 16921 keys.)
__device__ __forceinline__ int xcd_grouped(int id, int groups, int size)
{
    const int even = groups & ~7;                            // the last few groups stay as they are numbered
    if (id >= even * size) return id;
    const int pos = id >> 3;
    return (pos / size * 8 + (id & 7)) * size + pos % size;
}

// Sixteen rows per workgroup, whose wavefronts take every NW-th tile of 32 keys of the workgroup's share [t0, t1) of the
// key axis, each with a softmax of its own, and meet in LDS at the end.  For the rows of one query or a few, where the
// cache's way from memory is what counts (each wavefront fetches a tile ahead, no barrier in the loop), and for fp32, where the
// three products that make up one of 24 bits are.
//   S^T = K Q^T by 16x16x32 MFMAs: a lane holds 32 (16) elements of one key as they lie in memory, a block or half of one,
//     converts them to bf16 (exact) and multiplies them eight at a time; Q follows that order.
//   O^T = V^T P^T: a lane takes whole blocks of values as they lie in memory, converts them and leaves them in LDS row by
//     row, from where the transposing load brings eight keys of one head-dim element; P is in that order already.
// fp32: Q and P go in as three bf16 numbers each, K and V are exact in one.
template <typename T, int DH, int NW, bool MASKED>
__global__ __launch_bounds__(64 * NW, sizeof(T) == 4 ? 2 : 3) void kvq_attn_rows_kernel(const T *__restrict__ q, int ld, KvqCache c, int extra,
                                                                int n, int H, float c_log2, T *__restrict__ o,
                                                                int nrb, int splits, float *__restrict__ part_o,
                                                                float *__restrict__ part_ml)
{
    constexpr bool F32 = sizeof(T) == 4;
    constexpr int NP = F32 ? 3 : 1;
    constexpr int KS = DH / 32, DB = DH / 16, NB = DH / 32;  // steps of S, 16-row blocks of O^T, scale blocks of a row
    constexpr int KW = DH / 32;                              // words of a key per lane
    constexpr int VL = DH / 64;                              // blocks of values per lane
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
    const int len = kvq_length(c, b, extra);
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

    const size_t head = (size_t)(b * c.heads + hk) * c.capacity;
    const uint8_t *Kc = c.k + head * (DH / 2), *Vc = c.v + head * (DH / 2), *Ks = c.k_scale + head * NB, *Vs = c.v_scale + head * NB;
    const uint8_t *mask = MASKED ? c.mask + (size_t)b * c.capacity : nullptr;

    struct Tile {
        uint32_t k[2][KW];
        uint4 v[VL];
        uint32_t ks[2], vs[VL], vis;                         // vis: with a mask, the keys that are seen; otherwise whether the lane's is
    };
    // Mask bytes come a tile before the rows that they let pass: instead of a hidden row, the first of the tile that is seen is fetched
    // again (32 x 8461 rows, 8 kv heads of 128, 0.3 of them hidden: 54 us, 65 with all rows; without a mask, where the same code
    // would cost 56, 54).
    uint32_t ahead = 0;
    auto fetch_mask = [&](int t) {
        if constexpr (MASKED) ahead = mask[min(min(t, last) * 32 + (lane & 31), last_row)];
    };
    auto fetch = [&](int t, Tile &x) {
        const int base = min(t, last) * 32;
        if constexpr (MASKED) x.vis = (uint32_t)__ballot(base + (lane & 31) < len && ahead != 0);
        const int first = MASKED && x.vis ? __builtin_ctz(x.vis) : 0;
        auto place = [&](int i) { return (uint32_t)min(base + (!MASKED || (x.vis >> i & 1) ? i : first), last_row); };
        fetch_mask(t + NW);
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const uint32_t key = place(16 * u + c16);
            if constexpr (KW == 4) {
                const uint4 w = *reinterpret_cast<const uint4 *>(Kc + key * (DH / 2) + g4 * 16);
                x.k[u][0] = w.x; x.k[u][1] = w.y; x.k[u][2] = w.z; x.k[u][3] = w.w;
            } else {
                const uint2 w = *reinterpret_cast<const uint2 *>(Kc + key * (DH / 2) + g4 * 8);
                x.k[u][0] = w.x; x.k[u][1] = w.y;
            }
            x.ks[u] = Ks[key * NB + g4 * NB / 4];
        }
#pragma unroll
        for (int j = 0; j < VL; ++j) {
            const uint32_t key = place((64 * j + lane) / NB), blk = lane % NB;
            x.v[j] = *reinterpret_cast<const uint4 *>(Vc + key * (DH / 2) + blk * 16);
            x.vs[j] = Vs[key * NB + blk];
        }
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
    constexpr int TOP = F32 ? kLarge : kTop + 127;
    int E = F32 ? kLarge : 0, acc_E = E;                     // of the values, of the sums

    // A tile's keys and values are converted first; the next one's are then fetched into the same registers, under the softmax and the
    // products.  A wavefront without a tile looks at one in which it sees nothing.
    Tile x;
    int t = t0 + wave;
    fetch_mask(t);
    fetch(t, x);
    do {
        const uint32_t vis = MASKED ? (t < t1 ? x.vis : 0) : (uint32_t)__ballot(x.vis != 0 && t < t1);
        // A tile without a visible key is passed over (32 x 8461 rows of 8 kv heads, seven tenths of them hidden in one stretch: 32 us,
        // 45 with its products; where a third of all rows is hidden, here and there, 54.5, 53).
        const bool any = !MASKED || vis != 0;
        floatx4_t s[2];
        if (any) {
            // ---- S^T: lane (c16, g4) gets the keys 4 g4 .. + 3 and 16 more of row c16
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                s[u] = floatx4_t{0};
                const float scale = __uint_as_float(x.ks[u] << 23);
#pragma unroll
                for (int i = 0; i < KS; ++i) {
                    const bf16x8_t kf = __builtin_bit_cast(bf16x8_t, bf16_eight(x.k[u][i], scale));
#pragma unroll
                    for (int p = NP - 1; p >= 0; --p)
                        s[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[i][p], s[u], 0, 0, 0);
                }
            }
            // ---- values to LDS
            uint32_t top = 0;
#pragma unroll
            for (int j = 0; j < VL; ++j) {
                const bool seen = (vis >> ((64 * j + lane) / NB)) & 1;
                if (seen && x.vs[j] != 255) top = max(top, x.vs[j]);
            }
            if (__builtin_expect(__builtin_amdgcn_ballot_w64((int)top > E) != 0, 0)) E = (int)wave_max(top) + kRoom;
#pragma unroll
            for (int j = 0; j < VL; ++j) {
                const int key = (64 * j + lane) / NB, blk = lane % NB;
                const bool seen = (vis >> key) & 1;
                const uint32_t w[4] = {x.v[j].x, x.v[j].y, x.v[j].z, x.v[j].w};
                const float scale = value_scale(x.vs[j], E, TOP, seen);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int piece = (2 * blk + (i >> 1)) ^ turn(key);
                    *reinterpret_cast<uint4 *>(vl + key * DH + piece * 16 + (i & 1) * 8) = F32 ? bf16_eight(w[i], scale) : half_eight(w[i], scale);
                }
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
                const float x = s[i >> 2][i & 3] - fin;
                p[i] = __builtin_amdgcn_exp2f(F32 ? x * c_log2 : fmaf(x, c_log2, kShift));
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
    const size_t prow = ((size_t)((b * c.heads + hk) * nrb + rb) * splits + split) * 16 + c16;
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
    if (splits > 1 && wave == 0 && g4 == 0) *reinterpret_cast<float2 *>(part_ml + prow * 2) = make_float2(m, sum);
}

// 16 bytes per lane global -> LDS; the wavefront fills 1 KiB starting at `lds_addr` in lane order.  The compiler does not see the
// load: it is waited for by hand before a barrier.
__device__ __forceinline__ void tile_dma_b128(const void *base, uint32_t byte_off, uint32_t lds_addr)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
                 :: "s"(lds_addr), "v"(byte_off), "s"(base) : "memory", "m0");
}

// 128 rows per workgroup, 32 per wavefront, over tiles of 64 keys; bf16.  For the rows of a whole scale, where the matrix cores and the
// softmax bound the time.
//   S^T = K Q^T by the 32x32x64 block-scaled MFMA: it takes keys in 4 bits with their scale bytes as they lie in memory, so K is
//     not converted, and at four times the rate of bf16 where the other operand has 6 bits.  Q, scaled so that scores come in units of
//     log2, goes in as three E2M3 numbers per element (sign, 2 bits of exponent, 3 of mantissa, a shared 2^e, 2^(e-4), 2^(e-9) per 32),
//     each for what the one before leaves.  That is at most 2^-2 of its unit, then 2^-3, which the next one's units hold whole
//     (2^-5 after the first would be 8, past the largest, 7.5); what the last leaves is at most 2^(e-12).
//     What is left is the same for an element of any size, so it is held against the keys: a block of 32 adds at most 6 * 2^k (a key's
//     largest value) times the sum of what is left to a score's error.  While that is below 2^-5 over a row for all rows of a wavefront and
//     the keys of a tile, the pieces serve (queries and keys of normal numbers: 2^-7.5 at most, 2^-14 rms).  From the first tile on for
//     which it is not (scores of 15 and more, or a few elements far larger than the others), a wavefront takes its queries as they came, in bf16, and
//     converts the keys: exact, four products of 16 elements for three of 64 and 32 conversions per half a tile more, 10 to 24 % slower (4 x 1600
//     x 12121, 32 heads of 128: 1280 us, 1075 with pieces; 8 x 231 x 871, 30 of 64, 27.0, 23.3; 16 x 410 x 1281, 116, 106; 4 x 300 x 2500, 16
//     of 128, 49.6, 40.0).
//   O^T = V^T P^T by the 32x32x16 fp16 MFMA: the workgroup converts a tile of values once, into LDS.
// In the 32x32 accumulator layout a lane owns a query column, so the sum is lane-local, and P is in the order in which the second
// product takes it, as in attention.hip.
// Tiles come by DMA two ahead, into one of three stages of LDS that hold a tile's codes, scales and converted values.
// The loop goes by halves of a tile: beside the softmax of one stand the scores of the next and the products of the one before, in turn.
// Matrix cores and vector unit overlap only for instructions that do not wait for each other and stand next to each other, and a
// product that adds to the one right before it waits (a pair of weights 38 cycles, a product 40, both 58, 66 where they add on).
// KG = 2: two groups of four wavefronts on the same rows, each with half of the keys and stages of its own, which meet in LDS at the end:
// as full a CU as two workgroups make, without partial results in memory.
// WAVES, of a SIMD: 3 with 64-wide rows where there are more than two workgroups for every CU (30 heads, 8 x 410 x 1281 keys 65 us, 67 with
// 2, 16 x 410 x 1281 106, 115); with 2 there are registers for products that start from the reference, an addition less per weight (32 x 480 x
// 3001, 16 heads of 128, 373 to 365 us; 30 of 64, 8 x 231 x 871, 24.3 to 23.0).
template <int DH, int KG, int WAVES>
__global__ __launch_bounds__(256 * KG, WAVES) void kvq_attn_tiles_kernel(const uint16_t *__restrict__ q, int ld, KvqCache c, int extra,
                                                                int n, int H, float c_log2, uint16_t *__restrict__ o, int nrb,
                                                                int full_units, int shares, float *__restrict__ part_o,
                                                                float *__restrict__ part_ml)
{
    constexpr int KS = DH / 64, DB = DH / 32, NB = DH / 32;  // k64 steps of S, 32-row blocks of O^T, scale blocks of a row
    constexpr int VW = DH / 32;                              // words of values per thread
    constexpr int RAW = 64 * DH / 2;                         // bytes of a tile's codes
    constexpr int KOFF = 64 * DH * 2, VOFF = KOFF + RAW, SOFF = VOFF + RAW, STAGE = SOFF + 2 * 64 * NB;
    __shared__ uint4 lds[KG * 3 * STAGE / 16];               // [group][stage][values fp16 | codes of K | of V | scales of K | of V]

    const int tid = threadIdx.x & 255, lane = tid & 63, rl = lane & 31, g = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int kg = KG > 1 ? __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 8) : 0;
    int unit = blockIdx.x, share = 0, ranges = 1;
    if (unit < full_units) {
        unit = xcd_grouped(unit, full_units / nrb, nrb);
    } else {
        const int t = unit - full_units;
        unit = full_units + t / shares;
        share = t % shares;
        ranges = shares;
    }
    const int rb = unit % nrb, hk = unit / nrb % c.heads, b = unit / (nrb * c.heads);
    const int G = H / c.heads, R = n * G;
    const int len = kvq_length(c, b, extra);
    const int tiles = (len + 63) / 64;
    // the group's tiles [t0, t1], one at least and as many as the other's: where there is none, one in which nothing is seen
    const int first_tile = tiles * share / ranges, end = tiles * (share + 1) / ranges;   // (at most 2^18 tiles and 16 shares)
    const int trips = max((end - first_tile + KG - 1) / KG, 1), t0 = first_tile + kg * trips, t1 = t0 + trips - 1;
    const int seen_end = min(len, min(end, t1 + 1) * 64), last_row = max(len - 1, 0);
    const int r0 = rb * 128 + wave * 32, row = min(r0 + rl, R - 1);
    const bool active = __builtin_amdgcn_readfirstlane(r0 < R ? 1 : 0) != 0;

    const size_t head = (size_t)(b * c.heads + hk) * c.capacity;
    const uint8_t *Kc = c.k + head * (DH / 2), *Vc = c.v + head * (DH / 2), *Ks = c.k_scale + head * NB, *Vs = c.v_scale + head * NB;
    const uint8_t *mask = c.mask ? c.mask + (size_t)b * c.capacity : nullptr;
    uint8_t *lds8 = reinterpret_cast<uint8_t *>(lds) + kg * 3 * STAGE;
    const uint32_t lds_base = (uint32_t)(uintptr_t)lds + kg * 3 * STAGE;

    // ---- A tile by DMA.  K: 16-byte chunks of a row are turned by its number, so that the rows of sixteen lanes that read one chunk
    // lie in all banks.  V: the order in which the threads convert it: a quarter of a row each, neighbouring quads four rows apart
    // (128-wide rows) so that their writes lie in different banks.  A row past the last is the last again.
    const int vkey = DH == 128 ? wave * 16 + ((lane >> 4) & 3) + (lane >> 2 & 3) * 4 : tid >> 2, vpart = tid & 3;
    const int dwave = DH == 128 ? wave : wave & 1;           // 64-wide rows: two wavefronts fetch V, two K
    const int krow = DH == 128 ? dwave * 16 + (lane >> 2) : dwave * 32 + (lane >> 1);
    const int kchunk = DH == 128 ? (lane & 3) ^ ((krow >> 2) & 3) : (lane & 1) ^ ((krow >> 3) & 1);
    const int vrow_d = DH == 128 ? vkey : krow, vchunk = DH == 128 ? vpart : lane & 1;
    struct Next { uint32_t scale, seen; };                   // scales of the tile on their way to LDS (wavefront 0: K, 1: V); mask bytes
    auto fetch = [&](int t, int stage, Next &x) {
        const int first = t * 64;
        uint32_t kr = (uint32_t)(first + krow), vr = (uint32_t)(first + vrow_d), sr = (uint32_t)(first + lane);
        if (first + 64 > len) {                              // uniform: the last tile
            kr = min(kr, (uint32_t)last_row);
            vr = min(vr, (uint32_t)last_row);
            sr = min(sr, (uint32_t)last_row);
        }
        const uint32_t at = lds_base + stage * STAGE + dwave * 1024;
        if (DH == 128 || wave >= 2) tile_dma_b128(Kc, kr * (DH / 2) + kchunk * 16, at + KOFF);
        if (DH == 128 || wave < 2) tile_dma_b128(Vc, vr * (DH / 2) + vchunk * 16, at + VOFF);
        if (wave < 2) {
            const uint8_t *src = wave ? Vs : Ks;
            x.scale = NB == 4 ? *reinterpret_cast<const uint32_t *>(src + sr * NB) : *reinterpret_cast<const uint16_t *>(src + sr * NB);
        }
        if (mask) x.seen = mask[sr];
    };
    auto put_scales = [&](int stage, const Next &x) {
        if (wave < 2) {
            uint8_t *dst = lds8 + stage * STAGE + SOFF + wave * (64 * NB) + lane * NB;
            if (NB == 4) *reinterpret_cast<uint32_t *>(dst) = x.scale;
            else *reinterpret_cast<uint16_t *>(dst) = (uint16_t)x.scale;
        }
    };
    Next next, later;
    fetch(t0, 0, next);                                      // on their way under what follows
    fetch(min(t0 + 1, t1), 1, later);

    // ---- Q in three pieces of 6 bits: lane = row, block 2 s + g of its elements
    intx8_t qf[KS][3];
    int qs[KS];                                              // scale bytes of the pieces, in byte 0, 1, 2
    uint32_t limit = 0;                                      // largest scale bytes of keys for them, of block g in the low half, 2 + g above
    {
        const uint16_t *src = q + (size_t)(b * (long)n + row / G) * ld + (size_t)(hk * G + row % G) * DH + g * 32;
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            uint32_t w[16];
#pragma unroll
            for (int i = 0; i < 4; ++i) *reinterpret_cast<uint4 *>(w + 4 * i) = *reinterpret_cast<const uint4 *>(src + 64 * s + 8 * i);
            uint32_t top = 0;
            floatx16_t even, odd;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                even[i] = bf16_lo(w[i]) * c_log2;
                odd[i] = bf16_hi(w[i]) * c_log2;
                top = max(top, max(__float_as_uint(even[i]) & 0x7fffffffu, __float_as_uint(odd[i]) & 0x7fffffffu));
            }
            // the smallest 2^e with all elements below 7.75 * 2^e, which round to at most 7.5
            const int e = min(max((int)((top + (1u << 19)) >> 23) - 2, 13), 252);
#pragma unroll
            for (int p = 0; p < 3; ++p) {
                const float size = __uint_as_float((uint32_t)(p ? e + 1 - 5 * p : e) << 23);
                const uintx6_t x = __builtin_amdgcn_cvt_scalef32_2xpk16_fp6_f32(even, odd, size);
                const floatx32_t back = __builtin_amdgcn_cvt_scalef32_pk32_f32_fp6(x, size);
#pragma unroll
                for (int i = 0; i < 16; ++i) { even[i] -= back[2 * i]; odd[i] -= back[2 * i + 1]; }
                qf[s][p] = intx8_t{(int)x[0], (int)x[1], (int)x[2], (int)x[3], (int)x[4], (int)x[5], 0, 0};
            }
            qs[s] = e | (e - 4) << 8 | (e - 9) << 16;
            // A block of a key adds at most 6 * 2^k * rest to a score's error: the largest k for which that is below 2^-5 / NB; none for
            // what is not finite.
            float rest = 0.f;
#pragma unroll
            for (int i = 0; i < 16; ++i) rest += fabsf(even[i]) + fabsf(odd[i]);
            const int most_k = 127 - 6 - (DH == 128) - ((int)(__float_as_uint(6.f * rest) >> 23) - 126);
            limit |= (uint32_t)(top >= 0x7f800000u ? 0 : rest == 0.f ? 254 : min(max(most_k, 0), 254)) << (16 * s);
        }
    }
    limit = half_min(limit);                                 // of the wavefront's rows: blocks 0 and 2, 1 and 3
    const uint32_t limit_even = __builtin_amdgcn_readlane(limit, 0) + 0x1000100, limit_odd = __builtin_amdgcn_readlane(limit, 32) + 0x1000100;

    // everything on its way to LDS is there, for all wavefronts
    auto meet = [&]() {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
    };

    // ---- values: chunks of a row are turned so that four rows' 64-byte quarters lie in different banks when they are read
    // (transposing load, as in attention.hip), and the chunks of neighbouring quads of lanes when they are written
    auto turn = [](int key) { return DH == 128 ? ((key & 3) << 2) | ((key >> 2) & 3) : ((key >> 1) & 1) << 2; };
    const int tG = lane >> 4, tj = (lane >> 2) & 3, ta = lane & 3;
    const int vrow = 4 * (tG >> 1) + tj;
    // chunk 4 db + 2 (tG & 1) + (ta >> 1) of row vrow + 8 step8, in bytes
    auto chunk_at = [&](int db, int step8) {
        const int key = vrow + 8 * step8;
        return (key * DH + (((4 * db + 2 * (tG & 1) + (ta >> 1)) ^ turn(key)) << 3) + (ta & 1) * 4) * 2;
    };

    floatx16_t acc[DB];
#pragma unroll
    for (int i = 0; i < DB; ++i) acc[i] = floatx16_t{0};
    float l_run = 0.f, most = -1.f;                          // most: the sum of weights from which on a reference is looked for; < 0: no reference yet
    // Queries in pieces: - reference + kShift, in units of log2 as the scores; where registers allow, the products that make scores start
    // from it.
    constexpr bool FROM = WAVES == 2;
    float base = kShift;
    floatx16_t bases;
    auto set_base = [&](float x) {
        base = x;
#pragma unroll
        for (int i = 0; i < 16; ++i) bases[i] = FROM ? x : 0.f;
        if constexpr (FROM) asm volatile("" : "+v"(bases));
    };
    set_base(kShift);
    auto with_base = [&](float score) { return FROM ? score : score + base; };
    // Queries as they came: the reference, in units of the scores (which are not yet those of log2).
    float m_ref = -INFINITY;
    auto from_ref = [&](float score) { return fmaf(score - reference(m_ref), c_log2, kShift); };
    int E = 0, E_now = 0, acc_E = 0;                         // of the values converted last, of the tile at work, of the sums

    // A thread's values as they came, and their scale byte; all scale bytes of the lane's row, of values and of keys.  The rows that can be
    // seen, and the size of the values: E is the same in all wavefronts, each of which sees all bytes.
    struct Raw { uint32_t v[VW], vs, all, keys; };
    auto read_raw = [&](int stage, Raw &x) {
        const uint8_t *src = lds8 + stage * STAGE;
        if constexpr (VW == 4) {
            const uint4 w = *reinterpret_cast<const uint4 *>(src + VOFF + tid * 16);
            x.v[0] = w.x; x.v[1] = w.y; x.v[2] = w.z; x.v[3] = w.w;
        } else {
            const uint2 w = *reinterpret_cast<const uint2 *>(src + VOFF + tid * 8);
            x.v[0] = w.x; x.v[1] = w.y;
        }
        const uint8_t *sc = src + SOFF + 64 * NB;
        x.vs = sc[vkey * NB + vpart * NB / 4];
        x.all = NB == 4 ? *reinterpret_cast<const uint32_t *>(sc + lane * NB) : *reinterpret_cast<const uint16_t *>(sc + lane * NB);
        sc = src + SOFF;
        x.keys = NB == 4 ? *reinterpret_cast<const uint32_t *>(sc + lane * NB) : *reinterpret_cast<const uint16_t *>(sc + lane * NB);
    };
    float scale;
    bool far = false;                                        // whether a key that is seen is too large for queries in pieces
    auto look = [&](int t, const Raw &x, const Next &f, auto as_came) -> unsigned long long {
        constexpr bool WHOLE = decltype(as_came)::value;     // (queries as they came: any key will do)
        const bool seen = t * 64 + lane < seen_end && (!mask || f.seen);
        const unsigned long long vis = __ballot(seen);
        // bit 8 of 256 + limit - byte, for two bytes at a time: at most the limit
        constexpr uint32_t LOW = 0xff00ff, BIT = 0x1000100;
        const uint32_t size = (uint32_t)E * 0x10001 + BIT;
        const uint32_t keys = (limit_even - (x.keys & LOW)) & (limit_odd - (x.keys >> 8 & LOW)) & BIT;
        const uint32_t fits = (size - (x.all & LOW)) & (size - (x.all >> 8 & LOW)) & (WHOLE ? BIT : keys);
        if constexpr (!WHOLE) far = false;
        if (__builtin_expect((__builtin_amdgcn_ballot_w64(fits != BIT) & vis) != 0, 0)) {
            uint32_t top = 0;
            if (seen) {
#pragma unroll
                for (int i = 0; i < NB; ++i) {
                    const uint32_t byte = x.all >> (8 * i) & 255;
                    if (byte != 255) top = max(top, byte);
                }
            }
            if (__builtin_amdgcn_ballot_w64((int)top > E) != 0) E = (int)wave_max(top) + kRoom;
            if constexpr (!WHOLE) far = (__builtin_amdgcn_ballot_w64(keys != BIT) & vis) != 0;
        }
        scale = value_scale(x.vs, E, kTop + 127, (vis >> vkey) & 1);
        return vis;
    };
    int vdst[VW];                                            // where the thread's words go, in bytes
#pragma unroll
    for (int i = 0; i < VW; ++i) vdst[i] = (vkey * DH + (((vpart * VW + i) ^ turn(vkey)) << 3)) * 2;
    auto convert = [&](int stage, const Raw &x, int i) {
        *reinterpret_cast<uint4 *>(lds8 + stage * STAGE + vdst[i]) = half_eight(x.v[i], scale);
    };

    Raw raw;
    put_scales(0, next);
    put_scales(1, later);
    meet();
    read_raw(0, raw);
    unsigned long long vis = look(t0, raw, next, std::false_type{}), vis_next;
#pragma unroll
    for (int i = 0; i < VW; ++i) convert(0, raw, i);
    next = later;
    __syncthreads();
    int stage = 0;                                           // of the tile at work
    auto after = [](int s) { return s == 2 ? 0 : s + 1; };
    if (!active) {                                           // rows past the end: only helps with the tiles
        for (int t = t0; t <= t1; ++t) {
            const int s1 = after(stage);
            fetch(min(t + 2, t1), after(s1), later);
            read_raw(s1, raw);
            look(min(t + 1, t1), raw, next, std::true_type{});
#pragma unroll
            for (int i = 0; i < VW; ++i) convert(s1, raw, i);
            put_scales(after(s1), later);
            next = later;
            stage = s1;
            meet();
        }
        if (KG > 1) {                                        // (the meeting of the groups)
            __syncthreads();
            __syncthreads();
        }
        return;
    }

    // Where the lane reads values of the first 16 keys of a tile, and the first 32 keys; further on by constants.
    lds_byte_t *vp[DB][2], *kp[KS], *sp;
#pragma unroll
    for (int i = 0; i < DB; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h) vp[i][h] = (lds_byte_t *)(lds8 + chunk_at(i, h));
#pragma unroll
    for (int s = 0; s < KS; ++s)
        kp[s] = (lds_byte_t *)(lds8 + KOFF + rl * (DH / 2) + ((2 * s + g) ^ (DH == 128 ? (rl >> 2) & 3 : (rl >> 3) & 1)) * 16);
    sp = (lds_byte_t *)(lds8 + SOFF + rl * NB);

    floatx16_t s[2];                                         // scores of the two halves of a tile
    f16x8_t pf[2][2];                                        // their weights, by steps of 16 keys
    float sum;
    pf[1][0] = pf[1][1] = f16x8_t{0};
    auto load_keys = [&](int half, uintx4_t *k) -> int {
#pragma unroll
        for (int x = 0; x < KS; ++x) k[x] = *(lds_uintx4_t *)(kp[x] + half * (RAW / 2));
        const uint32_t w = NB == 4 ? *(__attribute__((address_space(3))) const uint32_t *)(sp + half * 32 * NB)
                                   : *(__attribute__((address_space(3))) const uint16_t *)(sp + half * 32 * NB);
        return (int)(w >> (8 * g));
    };
#define FVAR_S(half, ks, p, on)                                                                                          \
    s[half] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(                                                           \
        intx8_t{(int)k[ks][0], (int)k[ks][1], (int)k[ks][2], (int)k[ks][3], 0, 0, 0, 0}, qf[ks][p], on, 4, 2, 2 * (ks), sc, p, qs[ks])
    // product number i of a half's scores: smallest pieces first
    auto score = [&](int half, int i, const uintx4_t *k, int sc) {
        if (i == 0) FVAR_S(half, 0, 2, bases);
        if (i == 1) FVAR_S(half, KS - 1, KS == 2 ? 2 : 1, s[half]);
        if (i == 2) FVAR_S(half, 0, KS == 2 ? 1 : 0, s[half]);
        if constexpr (KS == 2) {
            if (i == 3) FVAR_S(half, 1, 1, s[half]);
            if (i == 4) FVAR_S(half, 0, 0, s[half]);
            if (i == 5) FVAR_S(half, 1, 0, s[half]);
        }
    };
#undef FVAR_S
    // The same with queries as they came: eight elements of a key at a time as bf16.
    bf16x8_t whole[4 * KS];
    auto score_whole = [&](int half, int i, const uintx4_t *k, int sc) {
        const bf16x8_t kf = __builtin_bit_cast(bf16x8_t, bf16_eight(k[i / 4][i % 4], __uint_as_float((uint32_t)(sc >> (16 * (i / 4)) & 255) << 23)));
        const floatx16_t none = {0};
        s[half] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, whole[i], i ? s[half] : none, 0, 0, 0);
    };
    auto load_v = [&](int i, int rows) -> f16x8_t {
        const shortx4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4_t *)(vp[i][0] + rows * DH * 2));
        const shortx4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4_t *)(vp[i][1] + rows * DH * 2));
        return __builtin_bit_cast(f16x8_t, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    };
    // One half's softmax beside the scores of the other (of the next tile where that is the first) and the products of the other's
    // weights (of the tile before where that is the second).  A step: a product, the weights of a pair or two in three stages.
    auto region = [&](auto which, auto as_came, int s1) {
        constexpr int half = decltype(which)::value, other = 1 - half;
        constexpr bool WHOLE = decltype(as_came)::value;
        constexpr int NS = WHOLE ? 4 * KS : 3 * KS, NPV = 2 * DB, STEPS = NS + NPV, PP = DH == 128 ? 1 : 2;     // PP: pairs of weights per step
        uintx4_t k[KS];
        f16x8_t vf[DB];
        const int sc = load_keys(other, k);
#pragma unroll
        for (int i = 0; i < DB; ++i) vf[i] = load_v(i, other * 32);
        if constexpr (half == 0) read_raw(s1, raw);
        __builtin_amdgcn_sched_barrier(0);
        float x[16], a, bsum;
#pragma unroll
        for (int step = 0; step < STEPS; ++step) {
            const int before = min((step + 1) / 2, NS);      // scores' products up to here, this one included if it is one
            if ((step & 1) && step / 2 < NS) {
                if constexpr (WHOLE) score_whole(other, step / 2, k, sc);
                else score(other, step / 2, k, sc);
            } else {
                const int i = step - before;
                acc[i % DB] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vf[i % DB], pf[other][i / DB], acc[i % DB], 0, 0, 0);
                if (i < DB) vf[i] = load_v(i, other * 32 + 16);
            }
#pragma unroll
            for (int w = 0; w < PP; ++w) {
                const int p2 = (step - 2) * PP + w, p1 = (step - 1) * PP + w, p0 = step * PP + w;
                if (p1 >= 0 && p1 < 8) {
                    x[2 * p1] = __builtin_amdgcn_exp2f(x[2 * p1]);
                    x[2 * p1 + 1] = __builtin_amdgcn_exp2f(x[2 * p1 + 1]);
                }
                if (p0 < 8) {
                    x[2 * p0] = WHOLE ? from_ref(s[half][2 * p0]) : with_base(s[half][2 * p0]);
                    x[2 * p0 + 1] = WHOLE ? from_ref(s[half][2 * p0 + 1]) : with_base(s[half][2 * p0 + 1]);
                }
                if (p2 >= 0 && p2 < 8) {
                    a = p2 ? a + x[2 * p2] : x[0];
                    bsum = p2 ? bsum + x[2 * p2 + 1] : x[1];
                    asm volatile("" : "+v"(a), "+v"(bsum));  // here, not after the region with all of x alive until then
                    const f16x2_t p = __builtin_convertvector((floatx2_t{x[2 * p2], x[2 * p2 + 1]}), f16x2_t);
                    pf[half][p2 >> 2][(2 * p2) & 7] = p[0];
                    pf[half][p2 >> 2][(2 * p2 + 1) & 7] = p[1];
                }
            }
            if constexpr (half == 1) {
                constexpr int from = DH == 128 ? 8 : 4;
                if (step >= from && step - from < VW) convert(s1, raw, step - from);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        sum = a + bsum;
        // the region's results are made in it
        asm volatile("" : "+v"(pf[half][0]), "+v"(pf[half][1]), "+v"(sum));
        asm volatile("" : "+v"(s[other]));
#pragma unroll
        for (int i = 0; i < DB; ++i) asm volatile("" : "+v"(acc[i]));
        __builtin_amdgcn_sched_barrier(0);
    };
    auto hide = [&](int half) {
        const uint32_t part = (uint32_t)(vis >> (32 * half));
        if (__builtin_expect(part != ~0u, 0)) {
            const uint32_t mine = part >> (4 * g);
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (!(mine >> (8 * (i >> 2) + (i & 3)) & 1)) s[half][i] = -INFINITY;
        }
    };
    auto settle = [&](int half, auto as_came) {
        constexpr bool WHOLE = decltype(as_came)::value;
        // The reference is not the running maximum but one that was it; the weights tell when it no longer serves.  A sum of NaN
        // does not ask for another: it stays NaN.
        const bool anew = (__builtin_amdgcn_ballot_w64(sum > most) != 0 && (uint32_t)(vis >> (32 * half)) != 0) || E_now != acc_E;
        if (__builtin_expect(anew, 0)) {
            float mx = s[half][0];
#pragma unroll
            for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[half][i]);
            const auto halves = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
            mx = fmaxf(__uint_as_float(halves[0]), __uint_as_float(halves[1]));
            const bool had = most >= 0.f, none = !had && mx == -INFINITY;
            float alpha = 1.f;
            if constexpr (WHOLE) {
                const float now = fmaxf(m_ref, mx);
                alpha = __builtin_amdgcn_exp2f((m_ref - reference(now)) * c_log2);
                m_ref = now;
            } else {
                // the largest score to kShift, or to 0 where its neighbours are too far apart for kShift to count
                const float before = base, over = FROM ? mx : mx + base;
                if (!none && (!had || over > kShift)) {
                    const float by = fabsf(mx) >= 0x1p24f ? mx : mx - kShift;
                    if constexpr (FROM) {
                        s[0] -= by;
                        s[1] -= by;
                    }
                    set_base(FROM ? base - by : -by);
                }
                alpha = __builtin_amdgcn_exp2f(base - before);
            }
            if (!had) alpha = 0.f;
            const float down = __builtin_amdgcn_ldexpf(alpha, max(acc_E - E_now, -200));
            most = none ? -1.f : kMost;
            acc_E = E_now;
            l_run *= alpha;
#pragma unroll
            for (int i = 0; i < DB; ++i) {
                acc[i] *= down;
                asm volatile("" : "+v"(acc[i]));
            }
            sum = 0.f;
#pragma unroll
            for (int i = 0; i < 16; i += 2) {
                const float x = __builtin_amdgcn_exp2f(WHOLE ? from_ref(s[half][i]) : with_base(s[half][i]));
                const float y = __builtin_amdgcn_exp2f(WHOLE ? from_ref(s[half][i + 1]) : with_base(s[half][i + 1]));
                sum += x + y;
                const f16x2_t p = __builtin_convertvector((floatx2_t{x, y}), f16x2_t);
                pf[half][i >> 3][i & 7] = p[0];
                pf[half][i >> 3][(i & 7) + 1] = p[1];
            }
        }
        l_run += sum;
    };

    E_now = E;
    int t = t0;
    auto tile = [&](auto as_came) {
        const int s1 = after(stage), s2 = after(s1);
        fetch(min(t + 2, t1), s2, later);
        hide(0);
        region(std::integral_constant<int, 0>{}, as_came, s1);
        settle(0, as_came);
        {
            // values go on to this tile's stage, keys to the next's
            const int by = (stage == 0 ? -2 : 1) * STAGE, k_by = (s1 == 0 ? -2 : 1) * STAGE, v_by = t == t0 ? 0 : by;
#pragma unroll
            for (int i = 0; i < DB; ++i) { vp[i][0] += v_by; vp[i][1] += v_by; }
#pragma unroll
            for (int i = 0; i < KS; ++i) kp[i] += k_by;
            sp += k_by;
        }
        hide(1);
        vis_next = look(min(t + 1, t1), raw, next, as_came);
        region(std::integral_constant<int, 1>{}, as_came, s1);
        settle(1, as_came);
        put_scales(s2, later);
        next = later;
        vis = vis_next;
        stage = s1;
        E_now = E;
        meet();
        ++t;
    };
    // Queries in pieces as long as the keys allow it, then as they came.
    if (!far) {
        uintx4_t k[KS];
        const int sc = load_keys(0, k);
#pragma unroll
        for (int i = 0; i < 3 * KS; ++i) score(0, i, k, sc);
        do tile(std::false_type{});
        while (t <= t1 && !far);
    }
    m_ref = most < 0.f ? -INFINITY : (kShift - base) / c_log2;
    if (t <= t1) {
        const uint16_t *src = q + (size_t)(b * (long)n + row / G) * ld + (size_t)(hk * G + row % G) * DH + g * 32;
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 4 * KS; ++i) {
            const uintx4_t w = *reinterpret_cast<const uintx4_t *>(src + 64 * (i / 4) + 8 * (i % 4));
            whole[i] = __builtin_bit_cast(bf16x8_t, w);
#pragma unroll
            for (int j = 0; j < 4; ++j) top = max(top, max(w[j] << 16 & 0x7fff0000u, w[j] & 0x7fff0000u));
        }
        // (an infinity makes scores that are not numbers, not some that are all -inf)
        if (top >= 0x7f800000u) whole[0] = __builtin_bit_cast(bf16x8_t, uintx4_t{0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u});
        uintx4_t k[KS];
        const int sc = load_keys(0, k);
#pragma unroll
        for (int i = 0; i < 4 * KS; ++i) score_whole(0, i, k, sc);
        do tile(std::true_type{});
        while (t <= t1);
    }
    // the last half's products
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int i = 0; i < DB; ++i)
            acc[i] = __builtin_amdgcn_mfma_f32_32x32x16_f16(load_v(i, 32 + 16 * u), pf[1][u], acc[i], 0, 0, 0);

    // ---- means, back at their size (see value_scale)
    {
        const auto halves = __builtin_amdgcn_permlane32_swap(__float_as_uint(l_run), __float_as_uint(l_run), false, false);
        l_run = __uint_as_float(halves[0]) + __uint_as_float(halves[1]);
    }
    const float inv = l_run == 0.f ? 0.f : 1.0f / l_run;
    auto mean = [&](float x) { return __builtin_amdgcn_ldexpf(x * inv, acc_E - kTop - 127); };
    const size_t prow = ((size_t)(unit - full_units) * shares + share) * 128 + wave * 32 + rl;
    uint16_t *dst = o + (size_t)(b * (long)n + row / G) * H * DH + (size_t)(hk * G + row % G) * DH;
    // Two quads of results that lie eight apart in the lane's row: four more stand in the lane 32 further, which changes one of its
    // quads for one of these, so that each stores 16 bytes (30 heads of 64: 8 x 231 x 871 25.0 to 24.1 us, 8 x 410 x 1281 69 to 64).  A share's,
    // with its weight, go as they are to the merge.
    auto put = [&](auto divided, int d, float4 x, float4 y) {
        if constexpr (decltype(divided)::value) {
            float *to = part_o + prow * DH + d + 4 * g;
            *reinterpret_cast<float4 *>(to) = x;
            *reinterpret_cast<float4 *>(to + 8) = y;
        } else {
            const auto lo = __builtin_amdgcn_permlane32_swap(pack_bf16x2(x.x, x.y), pack_bf16x2(y.x, y.y), false, false);
            const auto hi = __builtin_amdgcn_permlane32_swap(pack_bf16x2(x.z, x.w), pack_bf16x2(y.z, y.w), false, false);
            *reinterpret_cast<uint4 *>(dst + d + 8 * g) = make_uint4(lo[0], hi[0], lo[1], hi[1]);
        }
    };
    auto put_weight = [&](float m, float l) {
        if (ranges > 1 && g == 0) *reinterpret_cast<float2 *>(part_ml + prow * 2) = make_float2(m, l);
    };
    auto quad_mean = [&](const floatx16_t &x, int e) { return make_float4(mean(x[e]), mean(x[e + 1]), mean(x[e + 2]), mean(x[e + 3])); };
    if constexpr (KG == 1) {
        if (r0 + rl >= R) return;
        auto finish = [&](auto divided) {
#pragma unroll
            for (int i = 0; i < DB; ++i)
#pragma unroll
                for (int e = 0; e < 16; e += 8) put(divided, 32 * i + 2 * e, quad_mean(acc[i], e), quad_mean(acc[i], e + 4));
        };
        if (ranges > 1) finish(std::true_type{});
        else finish(std::false_type{});
        put_weight(m_ref, l_run);
    } else {
        // each group leaves half of its means, its reference and weight where the other finds them, and takes the other half to the end
        constexpr int HB = DB / 2;
        float4 *xo = reinterpret_cast<float4 *>(lds);        // [group][wave][block, quad][lane]
        float2 *xm = reinterpret_cast<float2 *>(xo + 8 * HB * 4 * 64);   // [group][wave][lane]
        auto leave = [&](const floatx16_t *x) {
#pragma unroll
            for (int i = 0; i < HB; ++i)
#pragma unroll
                for (int e = 0; e < 16; e += 4) xo[((kg * 4 + wave) * HB * 4 + i * 4 + e / 4) * 64 + lane] = quad_mean(x[i], e);
        };
        __syncthreads();                                     // the stages have been read
        if (kg) leave(acc);
        else leave(acc + HB);
        xm[(kg * 4 + wave) * 64 + lane] = make_float2(m_ref, l_run);
        __syncthreads();
        if (r0 + rl >= R) return;
        const float2 other = xm[((1 - kg) * 4 + wave) * 64 + lane];
        const float m = fmaxf(m_ref, other.x), fin = reference(m);
        float own = l_run * __builtin_amdgcn_exp2f((m_ref - fin) * c_log2), theirs = other.y * __builtin_amdgcn_exp2f((other.x - fin) * c_log2);
        const float all = own + theirs, each = all == 0.f ? 0.f : 1.0f / all;
        own *= each;
        theirs *= each;
        auto finish = [&](auto divided, const floatx16_t *x) {
            auto joined = [&](int i, int e) {
                const float4 a = quad_mean(x[i], e), b = xo[(((1 - kg) * 4 + wave) * HB * 4 + i * 4 + e / 4) * 64 + lane];
                return make_float4(fmaf(b.x, theirs, a.x * own), fmaf(b.y, theirs, a.y * own), fmaf(b.z, theirs, a.z * own),
                                   fmaf(b.w, theirs, a.w * own));
            };
#pragma unroll
            for (int i = 0; i < HB; ++i)
#pragma unroll
                for (int e = 0; e < 16; e += 8) put(divided, 32 * (kg * HB + i) + 2 * e, joined(i, e), joined(i, e + 4));
        };
        if (ranges > 1) {
            if (kg) finish(std::true_type{}, acc + HB);
            else finish(std::true_type{}, acc);
        } else {
            if (kg) finish(std::false_type{}, acc + HB);
            else finish(std::false_type{}, acc);
        }
        if (!kg) put_weight(m, all);
    }
}

// The shares of rows joined: each is a mean and its weight.  A unit is a block of BR rows of one (sample, kv head); the shares
// of unit first + u lie at [u][share][row].  GROUPS groups of DH/4 threads per row, four head-dim elements a thread: a group takes every
// GROUPS-th share, four at a time, with a running reference and mean (not the sum: a mean times its weight need not be a number that fp32
// holds), and the groups meet in LDS.  One group where the shares are few and the
// rows many; more where a few rows have many shares, whose loads would wait for each other (64 shares of 16 rows: 24 us by one, 3 by 8).
template <typename T, int DH, int GROUPS>
__global__ __launch_bounds__(256) void kvq_attn_merge_kernel(const float *__restrict__ part_o, const float *__restrict__ part_ml,
                                                             int n, int H, int heads, int nrb, int BR, int first, int shares,
                                                             float c_log2, int total, T *__restrict__ o)
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
    if (mine) Quad<T>::store(o + (size_t)(b * n + row / G) * H * DH + (size_t)(hk * G + row % G) * DH + d, acc);
}

// Blocks of how many rows of a (sample, kv head) an attention is run by: 16 (kvq_attn_rows_kernel) or 128 (kvq_attn_tiles_kernel, bf16
// only).  The first starts and ends soonest and is bound by the work, which it does at less than half the other's pace; the other fetches
// and converts for 128 rows whatever there are, and joins groups and shares.  So the work decides, and at half a block and less twice as
// much of it is still by 16.  us by 16 / by 128, 16 heads of 128: 1 x 144 rows x 265 keys 6.3 / 16, 1 x 400 x 921 13 / 24, 1 x 576 x 1497
// 24 / 27, 1 x 200 x 4813 29 / 27, 2 x 128 x 5000 30 / 28, 16 x 100 x 1000 40 / 28, 8 x 64 x 2521 27 / 32, 16 x 64 x 3000 55 / 50,
// 32 x 48 x 3001 81 / 82; 30 heads of 64: 1 x 324 x 640 9.6 / 13, 2 x 231 x 871 14 / 16, 8 x 169 x 316 17 / 15, 8 x 100 x 871 23 / 17.
static int kvq_block(DType dt, int B, int n, int H, int heads, int length)
{
    const int rows = n * (H / heads);
    if (dt != DType::BF16 || rows <= 48) return 16;
    return (long)B * heads * ((rows + 15) / 16) * length <= (rows <= 64 ? 1l << 21 : 1l << 20) ? 16 : 128;
}

// nrb blocks per (sample, kv head), units in all, of which the first `full` take all keys and each other one is divided into `shares`.
// `ragged`: samples of lengths of their own, which only the GPU knows.
// waves: wavefronts of a workgroup, which divide a block's keys (16 rows), or its rows and, if there are 8, keys (128 rows).
struct KvqRun { int block, nrb, units, full, shares, waves; };
constexpr int kGroupsFrom = 2048, kGroupsTo = 4096;          // lengths at which the choice between one and two groups changes
static KvqRun kvq_run(int block, int B, int n, int H, int heads, int Dh, int length, bool ragged)
{
    KvqRun run;
    run.block = block;
    run.nrb = (n * (H / heads) + block - 1) / block;
    run.units = B * heads * run.nrb;
    run.waves = 4;
    if (block == 16) {
        // Where the blocks alone fill the chip and the cache is short, wavefronts without a tile, and the meeting of those with one, cost
        // more than they save: us with 1 / 2 / 4 of them, 17 x 125 rows x 4 keys of 32 heads 14 / 18 / 31, 32 x 64 x 121 of 16 11 / 14 / 17,
        // 8 x 100 x 500 17 / 14.5 / 15.8, 32 x 40 x 800 32 / 27 / 30; but 8 x 64 x 250 10 / 8.8 / 7.5, 32 x 32 x 4000 68 / 51 / 46.
        const int tiles = (length + 31) / 32;
        if (tiles <= 4 && run.units >= 1024) run.waves = 1;
        else if (tiles <= 32 && run.units >= 768 && !ragged) run.waves = 2;
        // Enough workgroups for two on every CU; four where samples differ, so that a CU that has had short ones takes more (32 samples of
        // 8461 keys, 8 kv heads: 512, 1024, 2048 places 53, 59, 59 us; of 1 to 16921 keys 1024, 2048, 4096 places 56, 59, 69 us).  Each with
        // two tiles per wavefront at least, or eight where every CU has a workgroup already and the joining, 3 us, is for nothing else
        // (fp32, 2 x 128 x 552, 16 heads of 64: 6.9 us whole, 10.6 in two shares).
        const int places = ragged ? 1024 : 512, least = run.units < 256 ? 2 : 8;
        const int want = (places + run.units - 1) / run.units, most = tiles / (least * 4);
        run.shares = want < most ? want : most > 0 ? most : 1;
        run.full = run.shares > 1 ? 0 : run.units;
        return run;
    }
    // Up to a workgroup on every CU: two groups of wavefronts in each, and shares where there are half as many or fewer (4 x 300 x 2500 keys
    // of 16 heads 44 us, 52 by one group; 2 x 130 x 2000 24, 25; 1 x 1664 x 6000 88, 99).  Otherwise, and over long caches where shares of
    // one group leave fewer CUs idle (1 x 1152 x 6000, 144 blocks, 76 us, 85 by two groups; 30 heads of 64, 640 x 6000, 150 blocks, 49, 64;
    // but 1 x 1152 x 2500 46, 43), two workgroups on every CU, three of 64-wide rows; those beyond the last full round are divided.
    // Pieces have four tiles at least for each group.  A quarter of a round more than one by two groups, divided, is also soonest done
    // so, if there is enough to divide (272 blocks, 1 x 2176 x 6000 keys of 16 heads 127 us, 159 by one group, x 2500 71, 78, but x 1000 47, 39;
    // 320 blocks, x 6000 139, 159, x 2500 75, 74; 384 blocks, x 2500 83, 77; 30 heads of 64, 270 blocks, 1 x 1152 x 6000 79, 92).
    const int two = Dh == 64 ? 768 : 512;
    bool groups = run.units <= 256 || (run.units <= 320 && length >= kGroupsFrom);
    if (run.units <= 256 && length >= kGroupsTo) groups = (two / run.units) * 256 * 8 <= (256 / run.units) * two * 9;
    const int slots = groups ? 256 : two, rest = run.units % slots, most = (length + 63) / 64 / (groups ? 8 : 4);
    run.waves = groups ? 8 : 4;
    run.full = run.units - rest;
    int want = rest ? slots / rest : 1;
    if (want > 16) want = 16;
    run.shares = want < most ? want : most > 0 ? most : 1;
    if (run.shares == 1) run.full = run.units;
    return run;
}

size_t kvq_attention_scratch_floats(DType dt, int B, int n, int H, int heads, int Dh, int capacity)
{
    // Between those lengths shares never fall as the length grows, nor where samples have lengths of their own, so for either kind of
    // blocks the longest length of each stretch is enough for every call; a shorter length may be run by the other kind.
    size_t most = 0;
    for (int length : {capacity, kGroupsTo - 1, kGroupsFrom - 1}) {
        if (length > capacity) continue;
        for (int block = 16; block <= 128; block *= 8) {
            if (block == 128 ? kvq_block(dt, B, n, H, heads, length) == 16 : kvq_block(dt, B, n, H, heads, 1) == 128) continue;
            const KvqRun run = kvq_run(block, B, n, H, heads, Dh, length, true);
            const size_t floats = (size_t)(run.units - run.full) * run.shares * run.block * (Dh + 2);
            if (floats > most) most = floats;
        }
    }
    return most;
}

// How an attention is run, for the tests: 100000 * rows of a block + 1000 * wavefronts + shares.
int kvq_attention_ways(int bf16, int B, int n, int H, int heads, int Dh, int length, int ragged)
{
    const int block = kvq_block(bf16 ? DType::BF16 : DType::F32, B, n, H, heads, length);
    const KvqRun run = kvq_run(block, B, n, H, heads, Dh, length, ragged != 0);
    return 100000 * block + 1000 * run.waves + run.shares;
}

// Wavefronts of a SIMD that the kernel is built for (see kvq_attn_tiles_kernel); wgs: workgroups of the launch.
static int kvq_waves(DType dt, int Dh, const KvqRun &run, int wgs)
{
    if (run.block == 16) return dt == DType::F32 ? 2 : 3;
    return Dh == 64 && run.waves == 4 && wgs > 512 ? 3 : 2;
}

// The same for the tests.
int kvq_attention_waves_per_simd(int bf16, int B, int n, int H, int heads, int Dh, int length, int ragged)
{
    const DType dt = bf16 ? DType::BF16 : DType::F32;
    const KvqRun run = kvq_run(kvq_block(dt, B, n, H, heads, length), B, n, H, heads, Dh, length, ragged != 0);
    return kvq_waves(dt, Dh, run, run.full + (run.units - run.full) * run.shares);
}

template <typename T, int DH>
static void launch_kvq(DType dt, const void *q, int ld, const KvqCache &c, int extra, int B, int n, int H, float c_log2,
                       void *o, float *part, hipStream_t st)
{
    const int length = c.lens ? c.capacity : c.len + extra;
    const KvqRun run = kvq_run(kvq_block(dt, B, n, H, c.heads, length), B, n, H, c.heads, DH, length, c.lens != nullptr);
    const int divided = run.units - run.full;
    float *part_ml = part + (size_t)divided * run.shares * run.block * DH;
    const unsigned wgs = (unsigned)(run.full + divided * run.shares);
    if (run.block == 16) {
#define FVAR_ROWS(NW, MASKED)                                                                                            \
    launch(kvq_attn_rows_kernel<T, DH, NW, MASKED>, dim3(wgs), dim3(64 * NW), 0, st, (const T *)q, ld, c, extra, n, H,    \
           c_log2, (T *)o, run.nrb, run.shares, part, part_ml)
        if (run.waves == 1) { if (c.mask) FVAR_ROWS(1, true); else FVAR_ROWS(1, false); }
        else if (run.waves == 2) { if (c.mask) FVAR_ROWS(2, true); else FVAR_ROWS(2, false); }
        else { if (c.mask) FVAR_ROWS(4, true); else FVAR_ROWS(4, false); }
#undef FVAR_ROWS
    } else if constexpr (sizeof(T) == 2) {
#define FVAR_TILES(KG, WAVES)                                                                                            \
    launch(kvq_attn_tiles_kernel<DH, KG, WAVES>, dim3(wgs), dim3(256 * KG), 0, st, (const T *)q, ld, c, extra, n, H,      \
           c_log2, (T *)o, run.nrb, run.full, run.shares, part, part_ml)
        if (run.waves == 8) FVAR_TILES(2, 2);
        else if (kvq_waves(dt, DH, run, (int)wgs) == 2) FVAR_TILES(1, 2);
        else if constexpr (DH == 64) FVAR_TILES(1, 3);
#undef FVAR_TILES
    }
    if (divided) {
        const int total = divided * run.block, per = 256 / (DH / 4);
        if (run.shares > 8)
            launch(kvq_attn_merge_kernel<T, DH, 8>, dim3((unsigned)((total + per / 8 - 1) / (per / 8))), dim3(256), 0, st, (const float *)part,
                   (const float *)part_ml, n, H, c.heads, run.nrb, run.block, run.full, run.shares, c_log2, total, (T *)o);
        else
            launch(kvq_attn_merge_kernel<T, DH, 1>, dim3((unsigned)((total + per - 1) / per)), dim3(256), 0, st, (const float *)part,
                   (const float *)part_ml, n, H, c.heads, run.nrb, run.block, run.full, run.shares, c_log2, total, (T *)o);
    }
}

void launch_kvq_attention(DType dt, const void *q, int ld, const KvqCache &c, int extra, int B, int n, int H, int Dh,
                          float scale, void *o, float *part, hipStream_t st)
{
    const float c_log2 = scale * 1.4426950408889634f;
    if (dt == DType::BF16) {
        if (Dh == 64) launch_kvq<uint16_t, 64>(dt, q, ld, c, extra, B, n, H, c_log2, o, part, st);
        else launch_kvq<uint16_t, 128>(dt, q, ld, c, extra, B, n, H, c_log2, o, part, st);
    } else {
        if (Dh == 64) launch_kvq<float, 64>(dt, q, ld, c, extra, B, n, H, c_log2, o, part, st);
        else launch_kvq<float, 128>(dt, q, ld, c, extra, B, n, H, c_log2, o, part, st);
    }
}

}  // namespace fvar
