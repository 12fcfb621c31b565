// Attention over a key/value cache held in 4 bits (format and layout: kvq.hip).
//   o[b,i,h,:] = sum_t p_t V[b,t,h',:],  p = softmax over the visible t of scale * q[b,i,h,:] . K[b,t,h',:],
//   h' = h / (H / heads); t is visible when t < length of sample b and mask[b][t] != 0; o = 0 where nothing is visible.
//
// The query heads of one kv head are further rows of the same problem: row r of a (sample, kv head) is query r / G of
// query head h' * G + r % G, G = H / heads.
#include "common.h"

namespace fvar {

typedef _Float16 f16x2_t __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));
typedef short shortx4_t __attribute__((ext_vector_type(4)));
typedef int intx8_t __attribute__((ext_vector_type(8)));
typedef unsigned uintx6_t __attribute__((ext_vector_type(6)));
typedef float floatx32_t __attribute__((ext_vector_type(32)));
typedef __attribute__((address_space(3))) shortx4_t lds_shortx4_t;

// Values as fp16 operands.  An fp16 number holds an element of the format times 2^-25 to 2^13, so a value goes in as
// value * 2^(kTop - E), E the largest scale byte seen so far and two more: sums are rescaled when a byte exceeds E, which is
// seldom, and blocks 2^-36 and less of the largest vanish.  Weights go in as p * 2^8, with a reference that may be up to
// 2^7 below the true maximum.  Next to bf16 operands (any exponent, 8 bits) the weights keep 11 bits, so that the
// output's own rounding is the only one of note: 1.7e-3 against 2.4e-3 of the result.
constexpr int kTop = 13, kRoom = 2;
constexpr float kShift = 8.f, kLag = 7.f, kMost = 32768.f;

__device__ __forceinline__ float half_scale(uint32_t byte, int E, bool seen)
{
    const int e = (int)byte - E + kTop + 127;
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

// Sixteen rows per workgroup, whose wavefronts take every NW-th tile of 32 keys of the workgroup's share [t0, t1) of the
// key axis, each with a softmax of its own, and meet in LDS at the end.  For the rows of one query or a few, where the
// cache's way from memory is what counts (each wavefront fetches a tile ahead, no barrier in the loop), and for fp32, where the
// three products that make up one of 24 bits are.
//   S^T = K Q^T by 16x16x32 MFMAs: a lane holds 32 (16) elements of one key as they lie in memory, a block or half of one,
//     converts them to bf16 (exact) and multiplies them eight at a time; Q follows that order.
//   O^T = V^T P^T: a lane takes whole blocks of values as they lie in memory, converts them and leaves them in LDS row by
//     row, from where the transposing load brings eight keys of one head-dim element; P is in that order already.
// fp32: Q and P go in as three bf16 numbers each, K and V are exact in one.
template <typename T, int DH, int NW>
__global__ __launch_bounds__(64 * NW) void kvq_attn_rows_kernel(const T *__restrict__ q, int ld, KvqCache c, int extra,
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
    int unit = xcd_contiguous(blockIdx.x, gridDim.x);        // the row blocks of a head share an L2
    const int rb = unit % nrb;
    unit /= nrb;
    const int split = unit % splits;
    unit /= splits;
    const int hk = unit % c.heads, b = unit / c.heads;
    const int G = H / c.heads, R = n * G;
    const int len = kvq_length(c, b, extra);
    const int tiles = (len + 31) / 32;
    const int t0 = (int)((long)tiles * split / splits), t1 = (int)((long)tiles * (split + 1) / splits);

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
    const uint8_t *mask = c.mask ? c.mask + (size_t)b * c.capacity : nullptr;

    struct Tile {
        uint32_t k[2][KW];
        uint4 v[VL];
        uint32_t ks[2], vs[VL], seen;
    };
    auto fetch = [&](int t, Tile &x) {
        const int base = t * 32;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const uint32_t key = (uint32_t)min(base + 16 * u + c16, len - 1);
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
            const uint32_t key = (uint32_t)min(base + (64 * j + lane) / NB, len - 1), blk = lane % NB;
            x.v[j] = *reinterpret_cast<const uint4 *>(Vc + key * (DH / 2) + blk * 16);
            x.vs[j] = Vs[key * NB + blk];
        }
        const int key = base + (lane & 31);
        x.seen = key < len;
        if (mask) x.seen = x.seen && mask[min(key, len - 1)];
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
    const float lag = kLag / c_log2;
    int E = 0;

    Tile cur, nxt;
    if (t0 + wave < t1) fetch(t0 + wave, cur);
    for (int t = t0 + wave; t < t1; t += NW) {
        const bool more = t + NW < t1;
        if (more) fetch(t + NW, nxt);
        const uint32_t vis = (uint32_t)__ballot(cur.seen != 0);
        if (vis) {
            // ---- S^T: lane (c16, g4) gets the keys 4 g4 .. + 3 and 16 more of row c16
            float s[8];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                floatx4_t a = {0};
                const float scale = __uint_as_float(cur.ks[u] << 23);
#pragma unroll
                for (int i = 0; i < KS; ++i) {
                    const bf16x8_t kf = __builtin_bit_cast(bf16x8_t, bf16_eight(cur.k[u][i], scale));
#pragma unroll
                    for (int p = NP - 1; p >= 0; --p)
                        a = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[i][p], a, 0, 0, 0);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) s[4 * u + i] = a[i];
            }
            // ---- values to LDS
            if constexpr (!F32) {
                uint32_t top = 0;
#pragma unroll
                for (int j = 0; j < VL; ++j) {
                    const bool seen = (vis >> ((64 * j + lane) / NB)) & 1;
                    if (seen && cur.vs[j] != 255) top = max(top, cur.vs[j]);
                }
                if (__builtin_expect(__builtin_amdgcn_ballot_w64((int)top > E) != 0, 0)) {   // uniform: the largest block so far
                    const int now = (int)wave_max(top) + kRoom;
                    const float down = __builtin_amdgcn_ldexpf(1.f, max(E - now, -200));
                    E = now;
#pragma unroll
                    for (int i = 0; i < DB; ++i)
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[i][e] *= down;
                }
            }
#pragma unroll
            for (int j = 0; j < VL; ++j) {
                const int key = (64 * j + lane) / NB, blk = lane % NB;
                const bool seen = (vis >> key) & 1;
                const uint32_t w[4] = {cur.v[j].x, cur.v[j].y, cur.v[j].z, cur.v[j].w};
                const float scale = F32 ? (seen ? __uint_as_float(cur.vs[j] << 23) : 0.f) : half_scale(cur.vs[j], E, seen);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int piece = (2 * blk + (i >> 1)) ^ turn(key);
                    *reinterpret_cast<uint4 *>(vl + key * DH + piece * 16 + (i & 1) * 8) = F32 ? bf16_eight(w[i], scale) : half_eight(w[i], scale);
                }
            }
            // ---- softmax
            if (vis != ~0u) {
                const uint32_t mine = vis >> (4 * g4);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (!(mine >> i & 1)) s[i] = -INFINITY;
                    if (!(mine >> (16 + i) & 1)) s[4 + i] = -INFINITY;
                }
            }
            float mx = s[0];
#pragma unroll
            for (int i = 1; i < 8; ++i) mx = fmaxf(mx, s[i]);
            if (__builtin_expect(__builtin_amdgcn_ballot_w64(mx > m_ref + lag) != 0, 0)) {
                const float now = column_max(fmaxf(m_ref, mx));
                const float alpha = __builtin_amdgcn_exp2f((m_ref - fmaxf(now, -1e30f)) * c_log2);
                m_ref = now;
                l_run *= alpha;
#pragma unroll
                for (int i = 0; i < DB; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[i][e] *= alpha;
            }
            const float fin = fmaxf(m_ref, -1e30f), base = fmaf(-fin, c_log2, kShift);
            float p[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                // fp32: the difference first, so that a row's only key weighs exactly 1
                p[i] = __builtin_amdgcn_exp2f(F32 ? (s[i] - fin) * c_log2 : fmaf(s[i], c_log2, base));
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
#pragma unroll
            for (int i = 0; i < DB; ++i) {
                const uint16_t *src = vl + rbase + ((i ^ rturn) << 4);
                const shortx4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4_t *)src);
                const shortx4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4_t *)(src + 16 * DH));
                const auto v = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
                if constexpr (F32) {
#pragma unroll
                    for (int k = NP - 1; k >= 0; --k)
                        acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, v), pf[k], acc[i], 0, 0, 0);
                } else {
                    acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8_t, v), ph, acc[i], 0, 0, 0);
                }
            }
            asm volatile("" ::: "memory");
        }
        cur = nxt;
    }

    // ---- the wavefronts' results: each as the mean of the values it saw, with its weight l at the reference m
    l_run = column_sum(l_run);
    const float inv = l_run == 0.f ? 0.f : 1.0f / l_run;
    float4 *slots = reinterpret_cast<float4 *>(vlds[wave]);
#pragma unroll
    for (int i = 0; i < DB; ++i) {
        float4 v = make_float4(acc[i][0] * inv, acc[i][1] * inv, acc[i][2] * inv, acc[i][3] * inv);
        if constexpr (!F32) {                                // |mean| <= 6 * 2^kTop: back to its size, which may be any
            v.x = __builtin_amdgcn_ldexpf(v.x, E - kTop - 127); v.y = __builtin_amdgcn_ldexpf(v.y, E - kTop - 127);
            v.z = __builtin_amdgcn_ldexpf(v.z, E - kTop - 127); v.w = __builtin_amdgcn_ldexpf(v.w, E - kTop - 127);
        }
        slots[i * 64 + lane] = v;
    }
    if (g4 == 0) ml[wave][c16] = make_float2(m_ref, l_run);
    __syncthreads();
    float m = ml[0][c16].x;
#pragma unroll
    for (int w = 1; w < NW; ++w) m = fmaxf(m, ml[w][c16].x);
    const float fin = fmaxf(m, -1e30f);
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

// 128 rows per workgroup, 32 per wavefront, over tiles of 64 keys; bf16.  For the rows of a whole scale, where the matrix cores and the
// softmax bound the time.
//   S^T = K Q^T by the 32x32x64 block-scaled MFMA: it takes keys in 4 bits with their scale bytes as they lie in memory, so K is
//     neither converted nor staged, and at four times the rate of bf16 where the other operand has 6 bits.  Q goes in as three E2M3
//     numbers per element (sign, 2 bits of exponent, 3 of mantissa, a shared 2^e per 32), each for what the one before leaves and 2^-5
//     smaller: off by at most 2^-13 of the block's largest element.  (Two leave 2^-8 of it, which scores of 20 and more, a
//     few times the usual, show in the output.)
//   O^T = V^T P^T by the 32x32x16 fp16 MFMA: the workgroup converts a tile of values once, into one of two LDS stages.
// In the 32x32 accumulator layout a lane owns a query column, so maximum and sum are lane-local, and P is in the order in which the
// second product takes it, as in attention.hip.
template <int DH>
__global__ __launch_bounds__(256, 2) void kvq_attn_tiles_kernel(const uint16_t *__restrict__ q, int ld, KvqCache c, int extra,
                                                                int n, int H, float c_log2, uint16_t *__restrict__ o, int nrb,
                                                                int full_units, int shares, float *__restrict__ part_o,
                                                                float *__restrict__ part_ml)
{
    constexpr int KS = DH / 64, DB = DH / 32, NB = DH / 32;  // k64 steps of S, 32-row blocks of O^T, scale blocks of a row
    constexpr int VW = DH / 32;                              // words of values per thread
    __shared__ uint4 vlds[2][64 * DH / 8];

    const int tid = threadIdx.x, lane = tid & 63, rl = lane & 31, g = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int unit = blockIdx.x, share = 0, ranges = 1;
    if (unit < full_units) {
        unit = xcd_contiguous(unit, full_units);
    } else {
        const int t = xcd_contiguous(unit - full_units, (int)gridDim.x - full_units);
        unit = full_units + t / shares;
        share = t % shares;
        ranges = shares;
    }
    const int rb = unit % nrb, hk = unit / nrb % c.heads, b = unit / (nrb * c.heads);
    const int G = H / c.heads, R = n * G;
    const int len = kvq_length(c, b, extra);
    const int tiles = (len + 63) / 64;
    // tiles [t0, t1], one at least: where there is none, one in which nothing is seen
    const int t0 = (int)((long)tiles * share / ranges), end = (int)((long)tiles * (share + 1) / ranges);
    const int t1 = max(end - 1, t0), seen_end = min(len, end * 64), last_row = max(len - 1, 0);
    const int r0 = rb * 128 + wave * 32, row = min(r0 + rl, R - 1);
    const bool active = __builtin_amdgcn_readfirstlane(r0 < R ? 1 : 0) != 0;

    // ---- Q in three pieces of 6 bits: lane = row, block 2 s + g of its elements
    intx8_t qf[KS][3];
    int qs[KS];                                              // scale bytes of the pieces, in byte 0, 1, 2
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
            // the smallest 2^e with all elements below 7.75 * 2^e, which round to at most 7.5; 255 makes NaN of what is not finite
            const int e = min(max((int)((top + (1u << 19)) >> 23) - 2, 13), 252);
#pragma unroll
            for (int p = 0; p < 3; ++p) {
                const float size = __uint_as_float((uint32_t)(e - 5 * p) << 23);
                const uintx6_t x = __builtin_amdgcn_cvt_scalef32_2xpk16_fp6_f32(even, odd, size);
                const floatx32_t back = __builtin_amdgcn_cvt_scalef32_pk32_f32_fp6(x, size);
#pragma unroll
                for (int i = 0; i < 16; ++i) { even[i] -= back[2 * i]; odd[i] -= back[2 * i + 1]; }
                qf[s][p] = intx8_t{(int)x[0], (int)x[1], (int)x[2], (int)x[3], (int)x[4], (int)x[5], 0, 0};
            }
            qs[s] = top >= 0x7f800000u ? 0xffffff : e | (e - 5) << 8 | (e - 10) << 16;
        }
    }

    const size_t head = (size_t)(b * c.heads + hk) * c.capacity;
    const uint8_t *Kc = c.k + head * (DH / 2), *Vc = c.v + head * (DH / 2), *Ks = c.k_scale + head * NB, *Vs = c.v_scale + head * NB;
    const uint8_t *mask = c.mask ? c.mask + (size_t)b * c.capacity : nullptr;

    // A tile of keys: every wavefront its own operands.  A tile of values: thread `tid` a quarter of a row, its scale byte; besides, every
    // wavefront all scale bytes (lane = row), so that all of them see the same largest one.
    struct Keys { uint4 k[2][KS]; uint32_t ks[2]; };
    struct Values { uint32_t v[VW], vs, all, seen; };
    // rows of a wavefront's sixteen in an order in which neighbouring quads' chunks lie in different banks (128-wide rows)
    const int vkey = DH == 128 ? wave * 16 + ((lane >> 4) & 3) + (lane >> 2 & 3) * 4 : tid >> 2, vpart = tid & 3;
    auto fetch_keys = [&](int t, Keys &x) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const uint32_t key = (uint32_t)min(t * 64 + 32 * u + rl, last_row);
#pragma unroll
            for (int s = 0; s < KS; ++s) x.k[u][s] = *reinterpret_cast<const uint4 *>(Kc + key * (DH / 2) + (2 * s + g) * 16);
            x.ks[u] = NB == 4 ? *reinterpret_cast<const uint32_t *>(Ks + key * NB) : *reinterpret_cast<const uint16_t *>(Ks + key * NB);
        }
    };
    auto fetch_values = [&](int t, Values &x) {
        const uint32_t key = (uint32_t)min(t * 64 + vkey, last_row);
        if constexpr (VW == 4) {
            const uint4 w = *reinterpret_cast<const uint4 *>(Vc + key * (DH / 2) + vpart * 16);
            x.v[0] = w.x; x.v[1] = w.y; x.v[2] = w.z; x.v[3] = w.w;
        } else {
            const uint2 w = *reinterpret_cast<const uint2 *>(Vc + key * (DH / 2) + vpart * 8);
            x.v[0] = w.x; x.v[1] = w.y;
        }
        x.vs = Vs[key * NB + vpart * NB / 4];
        const int mine = t * 64 + lane;
        const uint32_t held = (uint32_t)min(mine, last_row);
        x.all = NB == 4 ? *reinterpret_cast<const uint32_t *>(Vs + held * NB) : *reinterpret_cast<const uint16_t *>(Vs + held * NB);
        x.seen = mine < seen_end;
        if (mask) x.seen = x.seen && mask[held];
    };

    // ---- LDS: 16-byte chunks of a row are turned so that four rows' 64-byte quarters lie in different banks when they are read
    // (transposing load, as in attention.hip), and the chunks of neighbouring quads of lanes when they are written
    auto turn = [](int key) { return DH == 128 ? ((key & 3) << 2) | ((key >> 2) & 3) : ((key >> 1) & 1) << 2; };
    const int tG = lane >> 4, tj = (lane >> 2) & 3, ta = lane & 3;
    const int vrow = 4 * (tG >> 1) + tj;
    // chunk 4 db + 2 (tG & 1) + (ta >> 1) of row vrow + 16 u + 8 h: `turn` of the row in two parts, h and u only in the low bits
    auto chunk_at = [&](int db, int step8) {
        const int key = vrow + 8 * step8;
        return key * DH + (((4 * db + 2 * (tG & 1) + (ta >> 1)) ^ turn(key)) << 3) + (ta & 1) * 4;
    };

    floatx16_t acc[DB];
#pragma unroll
    for (int i = 0; i < DB; ++i) acc[i] = floatx16_t{0};
    // Scores come in units of log2, with the reference subtracted: Q is scaled by c_log2 and the MFMAs start from -reference + kShift.
    floatx16_t base;
#pragma unroll
    for (int i = 0; i < 16; ++i) base[i] = kShift;
    float m_ref = -INFINITY, l_run = 0.f, most = -1.f;       // most: the sum of a tile's weights from which on a reference is looked for
    int E = 0, acc_E = 0;                                    // of the stage, of the sums

    // the values of a tile, converted, into a stage; the rows that can be seen
    auto stage_values = [&](int stage, const Values &x) -> unsigned long long {
        const unsigned long long vis = __ballot(x.seen != 0);
        uint32_t top = 0;
        if (x.seen) {
#pragma unroll
            for (int i = 0; i < NB; ++i) {
                const uint32_t byte = x.all >> (8 * i) & 255;
                if (byte != 255) top = max(top, byte);
            }
        }
        if (__any((int)top > E)) E = (int)wave_max(top) + kRoom;   // the same in all wavefronts: the largest block so far
        const float scale = half_scale(x.vs, E, (vis >> vkey) & 1);
        uint16_t *dst = reinterpret_cast<uint16_t *>(vlds[stage & 1]) + vkey * DH;
#pragma unroll
        for (int i = 0; i < VW; ++i)
            *reinterpret_cast<uint4 *>(dst + (((vpart * VW + i) ^ turn(vkey)) << 3)) = half_eight(x.v[i], scale);
        return vis;
    };

    Keys keys;
    Values values;
    unsigned long long vis;
    fetch_keys(t0, keys);
    fetch_values(t0, values);
    vis = stage_values(t0, values);
    fetch_values(min(t0 + 1, t1), values);
    __syncthreads();
    if (!active) {                                           // rows past the end: only helps with the values
        for (int t = t0; t <= t1; ++t) {
            stage_values(t + 1, values);
            fetch_values(min(t + 2, t1), values);
            __syncthreads();
        }
        return;
    }
    // What is fetched for past the end is the last tile again, and what is staged then is not used: the loop has one way round.
    int t = t0;
    do {
        // ---- S^T, on top of `from`
        floatx16_t s[2];
        auto scores = [&](const floatx16_t &from) {
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int sc = (int)(keys.ks[u] >> (8 * g));
#define FVAR_S(ks, p, on)                                                                                                \
    s[u] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(                                                              \
        intx8_t{(int)keys.k[u][ks].x, (int)keys.k[u][ks].y, (int)keys.k[u][ks].z, (int)keys.k[u][ks].w, 0, 0, 0, 0},      \
        qf[ks][p], on, 4, 2, 2 * (ks), sc, p, qs[ks])
                FVAR_S(0, 2, from); FVAR_S(0, 1, s[u]); FVAR_S(0, 0, s[u]);
                if constexpr (KS == 2) { FVAR_S(KS - 1, 2, s[u]); FVAR_S(KS - 1, 1, s[u]); FVAR_S(KS - 1, 0, s[u]); }
#undef FVAR_S
            }
            if (vis != ~0ull) {
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const uint32_t mine = (uint32_t)(vis >> (32 * u)) >> (4 * g);
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if (!(mine >> (8 * (i >> 2) + (i & 3)) & 1)) s[u][i] = -INFINITY;
                }
            }
        };
        // ---- weights and their sum
        f16x8_t pf[4];
        float sum;
        auto weigh = [&]() {
            sum = 0.f;
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int i = 0; i < 16; i += 2) {
                    const f16x2_t p = __builtin_convertvector(
                        (floatx2_t{__builtin_amdgcn_exp2f(s[u][i]), __builtin_amdgcn_exp2f(s[u][i + 1])}), f16x2_t);
                    sum = __builtin_amdgcn_fdot2(p, f16x2_t{(_Float16)1.f, (_Float16)1.f}, sum, false);
                    pf[2 * u + (i >> 3)][i & 7] = p[0];
                    pf[2 * u + (i >> 3)][(i & 7) + 1] = p[1];
                }
        };
        scores(base);
        // values of a step of 16 keys are fetched one step ahead of the products that use them
        const uint16_t *vt = reinterpret_cast<const uint16_t *>(vlds[t & 1]);
        f16x8_t vf[2][DB];
        auto load_v = [&](int u, f16x8_t *x) {
#pragma unroll
            for (int i = 0; i < DB; ++i) {
                const shortx4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4_t *)(vt + chunk_at(i, 2 * u)));
                const shortx4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4_t *)(vt + chunk_at(i, 2 * u + 1)));
                x[i] = __builtin_bit_cast(f16x8_t, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
            }
        };
        load_v(0, vf[0]);
        __builtin_amdgcn_sched_barrier(0);
        weigh();
        // The reference is not the running maximum but one that was it; the weights tell when it no longer serves.  A sum of NaN
        // does not ask for another: it stays NaN.
        const bool anew = (__builtin_amdgcn_ballot_w64(sum > most) != 0 && vis != 0) || E != acc_E;
        if (__builtin_expect(anew, 0)) {
            scores(floatx16_t{0});
            float mx = s[0][0];
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[u][i]);
            mx = fmaxf(m_ref, mx);
            const auto halves = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
            const float now = fmaxf(__uint_as_float(halves[0]), __uint_as_float(halves[1]));
            const bool none = now == -INFINITY;              // nothing finite yet
            const float alpha = none ? 0.f : __builtin_amdgcn_exp2f(m_ref - now);
            const float down = __builtin_amdgcn_ldexpf(alpha, max(acc_E - E, -200));
            m_ref = now;
            most = none ? -1.f : kMost;
            acc_E = E;
            l_run *= alpha;
#pragma unroll
            for (int i = 0; i < DB; ++i) {
                acc[i] *= down;
                asm volatile("" : "+v"(acc[i]));
            }
            const float from = none ? kShift : kShift - now;
#pragma unroll
            for (int i = 0; i < 16; ++i) base[i] = from;
            scores(base);
            weigh();
        }
        l_run += sum;
        __builtin_amdgcn_sched_barrier(0);
        fetch_keys(min(t + 1, t1), keys);                    // not before: the scores' registers are free only now
        // ---- O^T += V^T P^T
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            if (u + 1 < 4) load_v(u + 1, vf[(u + 1) & 1]);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < DB; ++i)
                acc[i] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vf[u & 1][i], pf[u], acc[i], 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);
        }
        vis = stage_values(t + 1, values);
        fetch_values(min(t + 2, t1), values);
        __syncthreads();
    } while (++t <= t1);

    // ---- means, back at their size (see half_scale), which is stored or left with its weight for the merge
    {
        const auto halves = __builtin_amdgcn_permlane32_swap(__float_as_uint(l_run), __float_as_uint(l_run), false, false);
        l_run = __uint_as_float(halves[0]) + __uint_as_float(halves[1]);
    }
    const float inv = l_run == 0.f ? 0.f : 1.0f / l_run;
    if (r0 + rl >= R) return;
    const size_t prow = ((size_t)(unit - full_units) * shares + share) * 128 + wave * 32 + rl;
    uint16_t *dst = o + (size_t)(b * (long)n + row / G) * H * DH + (size_t)(hk * G + row % G) * DH;
#pragma unroll
    for (int i = 0; i < DB; ++i)
#pragma unroll
        for (int e = 0; e < 16; e += 4) {
            const int d = 32 * i + 8 * (e >> 2) + 4 * g;
            const float4 v = make_float4(__builtin_amdgcn_ldexpf(acc[i][e] * inv, E - kTop - 127),
                                         __builtin_amdgcn_ldexpf(acc[i][e + 1] * inv, E - kTop - 127),
                                         __builtin_amdgcn_ldexpf(acc[i][e + 2] * inv, E - kTop - 127),
                                         __builtin_amdgcn_ldexpf(acc[i][e + 3] * inv, E - kTop - 127));
            if (ranges > 1) *reinterpret_cast<float4 *>(part_o + prow * DH + d) = v;
            else Quad<uint16_t>::store(dst + d, v);
        }
    if (ranges > 1 && g == 0) *reinterpret_cast<float2 *>(part_ml + prow * 2) = make_float2(m_ref / c_log2, l_run);
}

// The shares of rows joined: each is a mean and its weight.  A unit is a block of BR rows of one (sample, kv head); the shares
// of unit first + u lie at [u][share][row].  One thread per four head-dim elements of a row.
template <typename T, int DH>
__global__ __launch_bounds__(256) void kvq_attn_merge_kernel(const float *__restrict__ part_o, const float *__restrict__ part_ml,
                                                             int n, int H, int heads, int nrb, int BR, int first, int shares,
                                                             float c_log2, long total, T *__restrict__ o)
{
    const long idx = (long)blockIdx.x * 256 + threadIdx.x;
    if (idx >= total) return;
    const int d = (int)(idx % (DH / 4)) * 4;
    const int r = (int)(idx / (DH / 4) % BR), u = (int)(idx / (DH / 4) / BR), unit = first + u;
    const int G = H / heads, row = unit % nrb * BR + r, hk = unit / nrb % heads;
    const long b = unit / nrb / heads;
    if (row >= n * G) return;
    const size_t prow = (size_t)u * shares * BR + r;
    float m = -INFINITY;
    for (int s = 0; s < shares; ++s) m = fmaxf(m, part_ml[(prow + (size_t)s * BR) * 2]);
    const float fin = fmaxf(m, -1e30f);
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    float sum = 0.f;
    for (int s = 0; s < shares; ++s) {
        const float2 ml = *reinterpret_cast<const float2 *>(part_ml + (prow + (size_t)s * BR) * 2);
        const float w = ml.y * __builtin_amdgcn_exp2f((ml.x - fin) * c_log2);
        const float4 v = *reinterpret_cast<const float4 *>(part_o + (prow + (size_t)s * BR) * DH + d);
        acc.x = fmaf(v.x, w, acc.x); acc.y = fmaf(v.y, w, acc.y);
        acc.z = fmaf(v.z, w, acc.z); acc.w = fmaf(v.w, w, acc.w);
        sum += w;
    }
    const float inv = sum == 0.f ? 0.f : 1.0f / sum;
    Quad<T>::store(o + (size_t)(b * n + row / G) * H * DH + (size_t)(hk * G + row % G) * DH + d,
                   make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv));
}

constexpr int kRowWaves = 4;

// How an attention is run: by blocks of 16 rows (kvq_attn_rows_kernel) or of 128 (kvq_attn_tiles_kernel); nrb blocks per
// (sample, kv head), units in all, of which the first `full` take all keys and each other one is divided into `shares`.
struct KvqRun { int block, nrb, units, full, shares; };
static KvqRun kvq_run(DType dt, int B, int n, int H, int heads, int length)
{
    const int rows = n * (H / heads);
    KvqRun run;
    run.block = dt == DType::BF16 && rows > 64 ? 128 : 16;
    run.nrb = (rows + run.block - 1) / run.block;
    run.units = B * heads * run.nrb;
    if (run.block == 16) {
        // enough workgroups for four on every CU, each with two tiles per wavefront at least
        const int want = (1024 + run.units - 1) / run.units, most = (length + 31) / 32 / (2 * kRowWaves);
        run.shares = want < most ? want : most > 0 ? most : 1;
        run.full = run.shares > 1 ? 0 : run.units;
        return run;
    }
    // two workgroups on every CU; those beyond the last full round are divided, into pieces of four tiles at least
    const int slots = 512, rest = run.units % slots, most = (length + 63) / 64 / 4;
    run.full = run.units - rest;
    int want = rest ? slots / rest : 1;
    if (want > 8) want = 8;
    run.shares = want < most ? want : most > 0 ? most : 1;
    if (run.shares == 1) run.full = run.units;
    return run;
}

size_t kvq_attention_scratch_floats(DType dt, int B, int n, int H, int heads, int Dh, int capacity)
{
    // shares never fall as the length grows: what the capacity needs is enough for every length
    const KvqRun run = kvq_run(dt, B, n, H, heads, capacity);
    return (size_t)(run.units - run.full) * run.shares * run.block * (Dh + 2);
}

template <typename T, int DH>
static void launch_kvq(DType dt, const void *q, int ld, const KvqCache &c, int extra, int B, int n, int H, float c_log2,
                       void *o, float *part, hipStream_t st)
{
    const KvqRun run = kvq_run(dt, B, n, H, c.heads, c.lens ? c.capacity : c.len + extra);
    const int divided = run.units - run.full;
    float *part_ml = part + (size_t)divided * run.shares * run.block * DH;
    const unsigned wgs = (unsigned)(run.full + divided * run.shares);
    if (run.block == 16) {
        launch(kvq_attn_rows_kernel<T, DH, kRowWaves>, dim3(wgs), dim3(64 * kRowWaves), 0, st, (const T *)q, ld, c, extra, n, H,
               c_log2, (T *)o, run.nrb, run.shares, part, part_ml);
    } else if constexpr (sizeof(T) == 2) {
        launch(kvq_attn_tiles_kernel<DH>, dim3(wgs), dim3(256), 0, st, (const T *)q, ld, c, extra, n, H, c_log2, (T *)o, run.nrb,
               run.full, run.shares, part, part_ml);
    }
    if (divided) {
        const long total = (long)divided * run.block * (DH / 4);
        launch(kvq_attn_merge_kernel<T, DH>, dim3((unsigned)((total + 255) / 256)), dim3(256), 0, st, (const float *)part,
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
