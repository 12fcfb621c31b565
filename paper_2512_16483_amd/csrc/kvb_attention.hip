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
typedef int intx8_t __attribute__((ext_vector_type(8)));
typedef unsigned uintx4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) const uintx4_t lds_uintx4_t;
typedef __attribute__((address_space(3))) shortx4_t lds_shortx4_t;
typedef __attribute__((address_space(3))) uint8_t lds_byte_t;

// Values as fp16 operands: a value goes in as value * 2^(kTop - E), E the largest exponent of a tile seen so far and kRoom more (sums are
// rescaled when a tile's exceeds E, which is seldom).  A value is at most 448, and fp16 numbers reach down to 2^-24, so tiles are exact
// down to 2^-19 of the largest one's size, and single values down to 2^-33 of the largest value; they lose bits from there on, and are 0
// below 2^-37.  Weights go in as p * 2^kShift, with a reference that may be up to 2^kLag below the true maximum.  Next to bf16 operands the
// weights keep 11 bits, so that the output's own rounding is the only one of note.
// fp32 takes values as they are in bf16, exact, up to tiles of 2^64, and at 2^64 over E from there on: a sum of weights up to 2^7 each stays finite.
constexpr int kTop = 6, kRoom = 2, kLarge = 64;
constexpr float kShift = 8.f, kLag = 7.f, kMost = 32768.f;
constexpr float kPlain = 16.f;                               // largest product of an element of a query and of a key, in units of log2: 11 in a score

__device__ __forceinline__ uint4 half_eight(uint32_t a, uint32_t b, float s)
{
    return make_uint4(kvb_f16<0>(a, s), kvb_f16<1>(a, s), kvb_f16<0>(b, s), kvb_f16<1>(b, s));
}
__device__ __forceinline__ uint4 bf16_eight(uint32_t a, uint32_t b, float s)
{
    return make_uint4(kvb_bf16<0>(a, s), kvb_bf16<1>(a, s), kvb_bf16<0>(b, s), kvb_bf16<1>(b, s));
}
// of four codes those that are no numbers, and 0 for the others
__device__ __forceinline__ uint32_t no_number(uint32_t x) { return x & ((((x & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) >> 7) * 255u; }
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

// Queries in two E4M3 numbers per element, with a power of two per row, 2^e, and 2^(e-4) for what the first leaves: the first leaves at most half
// a step of its binade, eight steps of bf16's eight bits, which the second holds whole.  (Elements below 2^-13 of their row's largest are held to
// 2^-21 of it.)  top: of the row's bits, sign taken off; from it the scale bytes of both pieces, in byte 0 and 1.
// A row with an element that is not finite becomes NaN, and so do its scores.  bf16 goes up to 255 * 2^120, past the cache's largest power: from 464 * 2^119
// on a row's is 2^120, whose largest first piece is 240 * 2^120 (256 would not be a finite fp32 number); 15 * 2^120 and less is left, 240 * 2^116.
__device__ __forceinline__ uint32_t top_of_eight(uint4 w, uint32_t top)
{
    const uint32_t x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) top = max(top, max(x[i] << 16 & 0x7fff0000u, x[i] & 0x7fff0000u));
    return top;
}
__device__ __forceinline__ int piece_bytes(uint32_t top)
{
    const int byte = max((int)kvb_byte(top >= 0x7f800000u ? 0x3f800000u : top), top > 0x7f680000u && top < 0x7f800000u ? 247 : 0);
    return byte | (byte - 4) << 8;
}
__device__ __forceinline__ void two_pieces(uint32_t a, uint32_t b, uint32_t top, int bytes, int &first, int &second)
{
    const float size = __uint_as_float((uint32_t)(bytes & 255) << 23), rest = __uint_as_float((uint32_t)(bytes >> 8) << 23);
    const float most = 240.f * 0x1p120f;
    float x[4] = {bf16_lo(a), bf16_hi(a), bf16_lo(b), bf16_hi(b)}, y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = __builtin_amdgcn_fmed3f(x[i], -most, most);
    const uint32_t one = kvb_four(y, size);
    const floatx2_t lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(one, size, false), hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(one, size, true);
    x[0] -= lo[0]; x[1] -= lo[1]; x[2] -= hi[0]; x[3] -= hi[1];
    const bool odd = top >= 0x7f800000u;
    first = odd ? 0x7f7f7f7f : (int)one;
    second = odd ? 0 : (int)kvb_four(x, rest);
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
//     multiplies eight elements at a time; Q follows that order.  (The block-scaled MFMA takes keys unconverted and is no faster here, where
//     memory is what counts, but adds less exactly, which the rows' weights would show: 2e-5 of them, rms, instead of 1e-7.)
//   O^T = V^T P^T: a lane takes pieces of sixteen values as they lie in memory, converts them and leaves them in LDS row by
//     row, from where the transposing load brings eight keys of one head-dim element; P is in that order already.
// fp32: Q and P go in as three bf16 numbers each, K and V are exact in one.
// stats: null, or for every row what its weights were taken against: reference and sum.  scores: null, or [B * heads][pitch][rows][32] where there
// is one block of rows, and receives them by tiles (not those of tiles without a visible key).
template <typename T, int DH, int NW, bool MASKED>
__global__ __launch_bounds__(64 * NW, 2) void kvb_attn_rows_kernel(const T *__restrict__ q, int ld, KvbCache c, int extra,
                                                                int n, int H, float c_log2, T *__restrict__ o,
                                                                int nrb, int splits, int chunk, float *__restrict__ part_o,
                                                                float *__restrict__ part_ml, float2 *__restrict__ stats,
                                                                float *__restrict__ scores, int pitch)
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
    // shares last: all samples' first shares come first, and the XCDs have as many of them each
    const int problems = (int)(gridDim.x / (nrb * splits)), split = unit / problems;
    unit %= problems;
    const int hk = unit % c.heads, b = unit / c.heads;
    const int G = H / c.heads, R = n * G;
    const int len = kvb_length(c, b, extra);
    const int tiles = (len + 31) / 32;
    // (products below 2^30: at most 2^19 tiles and 1024 shares)
    const int t0 = chunk ? chunk * split : tiles * split / splits, t1 = chunk ? min(t0 + chunk, tiles) : tiles * (split + 1) / splits;
    if (chunk && split > 0 && t0 >= t1) return;              // a share past the sample's end, which the merge knows of
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
        // (loads come back in order: the bytes that are wanted first, first)
        x.ks = Ks[at];
        x.vs = Vs[at];
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
                    for (int p = NP - 1; p >= 0; --p) s[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[i][p], s[u], 0, 0, 0);
                }
            }
            if (scores && c16 < R) {
                float *to = scores + (head * pitch + t) * (size_t)(R * 32) + c16 * 32 + 4 * g4;
                *reinterpret_cast<floatx4_t *>(to) = s[0];
                *reinterpret_cast<floatx4_t *>(to + 16) = s[1];
            }
            // ---- values to LDS
            const int ve = (int)__builtin_amdgcn_readfirstlane((int)x.vs) - 127;
            if (__builtin_expect(ve > E, 0)) E = ve + kRoom;
            const float vsize = power_of_two(ve - E + TOP);
            if (F32 && __builtin_expect(ve - E + TOP < -126, 0)) {
                // below 2^-188 of the largest: 0, as the least scale that there is would make them more than they are
#pragma unroll
                for (int j = 0; j < VL; ++j)
                    x.v[j] = make_uint4(no_number(x.v[j].x), no_number(x.v[j].y), no_number(x.v[j].z), no_number(x.v[j].w));
            }
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
        if (t < t1) fetch(t, x);
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

// 16 bytes per lane global -> LDS; the wavefront fills 1 KiB starting at `lds_addr` in lane order.  The compiler does not see the
// load: it is waited for by hand before a barrier.
__device__ __forceinline__ void tile_dma_b128(const void *base, uint32_t byte_off, uint32_t lds_addr)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
                 :: "s"(lds_addr), "v"(byte_off), "s"(base) : "memory", "m0");
}

// 128 rows per workgroup, 32 per wavefront, over tiles of 64 keys, two blocks of the cache; bf16.  For the rows of a whole scale, where the
// matrix cores and the softmax bound the time.
//   S^T = K Q^T by the 32x32x64 block-scaled MFMA: it takes keys in 8 bits with their scale bytes as they lie in memory, so K is not
//     converted.  Q goes in as two numbers per element (see two_pieces): two products at twice the rate of bf16 take as long as one
//     of bf16 would, without a conversion of K.  It adds eight products of neighbouring elements at a time, and drops of each what lies below 2^-13
//     of the largest: of normal numbers, 2^-15 of the sum of the products' sizes at most, 2^-18 rms, which at sums of 10 is 2^-11 of a weight at most (fp16 holds
//     one to 2^-12); where one channel is far larger than the others, up to 2^-10.  So the scores of keys whose products with the wavefront's queries
//     might pass 11, by their block's power and the queries' largest element, are made once more by bf16 products, which are added in fp32: what a
//     product loses is 2^-9.5 at most.  (Outputs are off by their rounding to bf16 then, 1.67e-3 of their 2-norm; by 1.77e-3 with one channel whose products are
//     11, 2.9e-3 with 16 such.)  4 x 1600 x 12121, 32 heads, one channel 20 times the others', all keys that way: 2100 us (1120 without, and outputs
//     of such keys off by 4.6e-3); where none are, 1171 (1167).  With a limit of 8 a 50th of the wavefronts over normal numbers found some (8 x 231 x 871, 30
//     heads of 64, 25.5 to 31.7 us; 26.1 with 11).
//   O^T = V^T P^T by the 32x32x16 fp16 MFMA: the workgroup converts a tile of values once, into LDS.
// In the 32x32 accumulator layout a lane owns a query column, so the sum is lane-local, and P is in the order in which the second
// product takes it, as in attention.hip.
// Tiles come by DMA two ahead: three of keys in LDS, two of values as they came (each wavefront converts what it fetched itself), and five
// halves of converted values: while some wavefronts still read the second half of the tile before, others write both halves of the next.
// With 128-wide rows that is half of a CU's LDS.
// The loop goes by halves of a tile: beside the softmax of one stand the scores of the next and the products of the one before, in turn.
// KG = 2: two groups of four wavefronts on the same rows, each with half of the keys and LDS of its own, which meet at the end:
// as full a CU as two workgroups make, without partial results in memory.
// WAVES, of a SIMD: 3 with 64-wide rows where there are at least two rounds of workgroups (30 heads, 16 x 410 x 1281 keys 136 to 124 us, 32 x 400 x 3000 513 to 443); with 2 there
// are registers for products that start from the reference, an addition less per weight.
template <int DH, int KG, int WAVES>
__global__ __launch_bounds__(256 * KG, WAVES) void kvb_attn_tiles_kernel(const uint16_t *__restrict__ q, int ld, KvbCache c, int extra,
                                                                int n, int H, float c_log2, uint16_t *__restrict__ o, int nrb,
                                                                int full_units, int shares, float *__restrict__ part_o,
                                                                float *__restrict__ part_ml, float2 *__restrict__ stats)
{
    constexpr int KS = DH / 64, DB = DH / 32;                // k64 steps of S, 32-row blocks of O^T
    constexpr int VW = DH / 32;                              // groups of eight values per thread
    constexpr int RAW = 64 * DH, HALF = 32 * DH * 2;         // bytes of a tile's codes, of half a tile of converted values
    constexpr int VOFF = 3 * RAW, COFF = VOFF + 2 * RAW, GROUP = COFF + 5 * HALF;
    __shared__ uint4 lds[KG * GROUP / 16];                   // [group][3 x keys | 2 x values as they came | 5 x half a tile of values]

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
    const int len = kvb_length(c, b, extra);
    const int tiles = (len + 63) / 64;
    // the group's tiles [t0, t1], one at least and as many as the other's: where there is none, one in which nothing is seen
    const int first_tile = tiles * share / ranges, end = tiles * (share + 1) / ranges;   // (at most 2^18 tiles and 16 shares)
    const int trips = max((end - first_tile + KG - 1) / KG, 1), t0 = first_tile + kg * trips, t1 = t0 + trips - 1;
    const int seen_end = min(len, min(end, t1 + 1) * 64), last_row = max(len - 1, 0);
    const int r0 = rb * 128 + wave * 32, row = min(r0 + rl, R - 1);
    const bool active = __builtin_amdgcn_readfirstlane(r0 < R ? 1 : 0) != 0;

    const size_t head = (size_t)(b * c.heads + hk);
    const uint8_t *Kc = c.k + head * c.capacity * DH, *Vc = c.v + head * c.capacity * DH;
    const uint8_t *Ks = c.k_scale + head * c.blocks(), *Vs = c.v_scale + head * c.blocks();
    const uint8_t *mask = c.mask ? c.mask + (size_t)b * c.capacity : nullptr;
    uint8_t *lds8 = reinterpret_cast<uint8_t *>(lds) + kg * GROUP;
    const uint32_t lds_base = (uint32_t)(uintptr_t)lds + kg * GROUP;

    // ---- A tile by DMA.  K: 16-byte chunks of a row are turned by its number, so that the rows of sixteen lanes that read one chunk
    // lie in all banks.  V: the order in which the threads convert it: 32 bytes (64-wide rows: 16) of a row each, neighbouring quads
    // four rows apart (128-wide rows) so that their writes lie in different banks.  A row past the last is the last again.
    constexpr int CH = DH / 16, DMAS = DH / 64;              // chunks of a row; instructions of a wavefront for a tile
    auto kturn = [](int key) { return DH == 128 ? (key >> 1) & 7 : (key >> 2) & 3; };
    const int vkey = DH == 128 ? wave * 16 + ((lane >> 4) & 3) + (lane >> 2 & 3) * 4 : tid >> 2, vpart = tid & 3;
    uint32_t seen_later = 1, seen_next = 1;                  // mask bytes of the lane's key, two tiles ahead and one
    auto fetch = [&](int t, int kslot, int vslot) {
        const int first = t * 64;
        const bool last = first + 64 > len;                  // uniform
#pragma unroll
        for (int i = 0; i < DMAS; ++i) {
            const int key = (wave * DMAS + i) * (64 / CH) + lane / CH, chunk = (lane % CH) ^ kturn(key);
            const uint32_t at = last ? min(first + key, last_row) : first + key;
            tile_dma_b128(Kc, at * DH + chunk * 16, lds_base + kslot * RAW + (wave * DMAS + i) * 1024);
        }
        const uint32_t vat = last ? min(first + vkey, last_row) : first + vkey;
#pragma unroll
        for (int i = 0; i < DMAS; ++i)
            tile_dma_b128(Vc, vat * DH + (vpart * DMAS + i) * 16, lds_base + VOFF + vslot * RAW + (wave * DMAS + i) * 1024);
        if (mask) seen_later = mask[last ? min(first + lane, last_row) : first + lane];
    };
    fetch(t0, 0, 0);                                         // on their way under what follows
    seen_next = seen_later;
    fetch(min(t0 + 1, t1), 1, 1);

    // ---- scale bytes of 64 blocks, a lane's each: of the tiles from 32 * (t / 32) on
    const int last_block = last_row / kKvbBlock;
    uint32_t kbytes = 0, vbytes = 0;
    int held = -1;
    auto scales_of = [&](int t) {                            // before a byte of tile t is asked for
        if (__builtin_expect((t >> 5) != held, 0)) {
            held = t >> 5;
            const int at = min(held * 64 + lane, last_block);
            kbytes = Ks[at];
            vbytes = Vs[at];
        }
    };
    auto byte_of = [&](uint32_t bytes, int t, int half) { return __builtin_amdgcn_readlane((int)bytes, (t & 31) * 2 + half); };

    // ---- Q in two pieces of 8 bits: lane = row, elements 64 s + 32 g .. + 31
    intx8_t qf[KS][2];
    int qbyte, plain_to;                                     // plain_to: the largest scale byte of keys whose products with these rows stay within kPlain
    {
        const uint16_t *src = q + (size_t)(b * (long)n + row / G) * ld + (size_t)(hk * G + row % G) * DH + g * 32;
        uint4 w[KS][4];
        uint32_t top = 0;
#pragma unroll
        for (int s = 0; s < KS; ++s)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                w[s][i] = *reinterpret_cast<const uint4 *>(src + 64 * s + 8 * i);
                top = top_of_eight(w[s][i], top);
            }
        const auto both = __builtin_amdgcn_permlane32_swap(top, top, false, false);
        top = max(both[0], both[1]);
        qbyte = piece_bytes(top);
        const float largest = __uint_as_float(kvb_wave_max(top >= 0x7f800000u ? 0 : top));
        plain_to = __builtin_amdgcn_readfirstlane((int)(__float_as_uint(kPlain / fabsf(c_log2) / 464.f / largest) >> 23));
#pragma unroll
        for (int s = 0; s < KS; ++s)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                int one, two;
                two_pieces(i & 1 ? w[s][i / 2].z : w[s][i / 2].x, i & 1 ? w[s][i / 2].w : w[s][i / 2].y, top, qbyte, one, two);
                qf[s][0][i] = one;
                qf[s][1][i] = two;
            }
    }

    // everything on its way to LDS is there, for all wavefronts
    auto meet = [&]() {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
    };

    // ---- converted values: chunks of a row are turned so that four rows' 64-byte quarters lie in different banks when they are read
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
    constexpr bool FROM = WAVES == 2;
    float m_ref = 0.f;                                       // the reference; FROM: the products that make scores start from - m_ref
    floatx16_t bases = floatx16_t{0};
    auto set_base = [&](float m) {
        m_ref = m;
        if constexpr (FROM) {
#pragma unroll
            for (int i = 0; i < 16; ++i) bases[i] = -m;
            asm volatile("" : "+v"(bases));
        }
    };
    auto exponent = [&](float score) { return fmaf(FROM ? score : score - m_ref, c_log2, kShift); };
    int E = -200, E_now = -200, acc_E = -200;                // of the values converted last, of the tile at work, of the sums

    // A thread's values as they came; the rows that can be seen, and the size of the values: E is the same in all wavefronts.
    struct Raw { uint32_t v[2 * VW]; };
    auto read_raw = [&](int vslot, Raw &x) {
        const uint8_t *src = lds8 + VOFF + vslot * RAW + wave * DMAS * 1024 + lane * 16;
#pragma unroll
        for (int i = 0; i < DMAS; ++i) {
            const uint4 w = *reinterpret_cast<const uint4 *>(src + i * 1024);
            x.v[4 * i] = w.x; x.v[4 * i + 1] = w.y; x.v[4 * i + 2] = w.z; x.v[4 * i + 3] = w.w;
        }
    };
    float vsize = 0.f;
    auto look = [&](int t, Raw &x, uint32_t seen_byte) -> unsigned long long {
        const unsigned long long vis = __ballot(t * 64 + lane < seen_end && seen_byte != 0);
        scales_of(t);
        const int e0 = byte_of(vbytes, t, 0) - 127, e1 = byte_of(vbytes, t, 1) - 127;
        if ((uint32_t)vis != 0 && e0 > E) E = e0 + kRoom;
        if (vis >> 32 != 0 && e1 > E) E = e1 + kRoom;
        vsize = power_of_two((wave < 2 ? e0 : e1) - E + kTop);
        if (__builtin_expect(vis != ~0ull, 0) && !(vis >> vkey & 1)) {
#pragma unroll
            for (int i = 0; i < 2 * VW; ++i) x.v[i] = 0;
        }
        return vis;
    };
    uint32_t vdst[VW];                                       // where the thread's values go within half a tile, in bytes
#pragma unroll
    for (int i = 0; i < VW; ++i) vdst[i] = COFF + ((vkey & 31) * DH + (((vpart * VW + i) ^ turn(vkey)) << 3)) * 2;
    int cslot = wave >> 1;                                   // the half tile that they go to
    auto convert = [&](const Raw &x, int i) {
        *reinterpret_cast<uint4 *>(lds8 + cslot * HALF + vdst[i]) = half_eight(x.v[2 * i], x.v[2 * i + 1], vsize);
    };
    auto next_half = [](int s, int by) { return s + by >= 5 ? s + by - 5 : s + by; };

    Raw raw;
    meet();
    read_raw(0, raw);
    unsigned long long vis = look(t0, raw, seen_next), vis_next;
#pragma unroll
    for (int i = 0; i < VW; ++i) convert(raw, i);
    cslot = next_half(cslot, 2);
    seen_next = seen_later;
    __syncthreads();
    int kslot = 0, vslot = 0;                                // of the tile at work
    auto after = [](int s) { return s == 2 ? 0 : s + 1; };
    if (!active) {                                           // rows past the end: only helps with the tiles
        for (int t = t0; t <= t1; ++t) {
            read_raw(vslot ^ 1, raw);
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            fetch(min(t + 2, t1), after(after(kslot)), vslot);
            look(min(t + 1, t1), raw, seen_next);
#pragma unroll
            for (int i = 0; i < VW; ++i) convert(raw, i);
            cslot = next_half(cslot, 2);
            seen_next = seen_later;
            kslot = after(kslot);
            vslot ^= 1;
            meet();
        }
        if (KG > 1) {                                        // (the meeting of the groups)
            __syncthreads();
            __syncthreads();
        }
        return;
    }

    // Where the lane reads values of the first 16 keys of half a tile, and the first 32 keys of a tile; further on by constants.
    lds_byte_t *vp[DB][2], *kp[KS][2];
#pragma unroll
    for (int i = 0; i < DB; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h) vp[i][h] = (lds_byte_t *)(lds8 + COFF + HALF + chunk_at(i, h));
#pragma unroll
    for (int s = 0; s < KS; ++s)
#pragma unroll
        for (int j = 0; j < 2; ++j) kp[s][j] = (lds_byte_t *)(lds8 + rl * DH + ((4 * s + 2 * g + j) ^ kturn(rl)) * 16);
    int rslot = 1;                                           // the half tile of values that vp points to

    floatx16_t s[2];                                         // scores of the two halves of a tile
    f16x8_t pf[2][2];                                        // their weights, by steps of 16 keys
    float sum;
    pf[1][0] = pf[1][1] = f16x8_t{0};
    auto load_keys = [&](int half, uintx4_t (&k)[KS][2]) {
#pragma unroll
        for (int x = 0; x < KS; ++x)
#pragma unroll
            for (int j = 0; j < 2; ++j) k[x][j] = *(lds_uintx4_t *)(kp[x][j] + half * (RAW / 2));
    };
#define FVAR_S(half, ks, p, on)                                                                                          \
    s[half] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(                                                           \
        intx8_t{(int)k[ks][0][0], (int)k[ks][0][1], (int)k[ks][0][2], (int)k[ks][0][3], (int)k[ks][1][0], (int)k[ks][1][1],      \
                (int)k[ks][1][2], (int)k[ks][1][3]}, qf[ks][p], on, 0, 0, 0, kb, p, qbyte)
    // product number i of a half's scores: smaller pieces first
    auto score = [&](int half, int i, const uintx4_t (&k)[KS][2], int kb) {
        if (i == 0) FVAR_S(half, 0, 1, bases);
        if (i == 1) FVAR_S(half, KS - 1, KS == 2 ? 1 : 0, s[half]);
        if constexpr (KS == 2) {
            if (i == 2) FVAR_S(half, 0, 0, s[half]);
            if (i == 3) FVAR_S(half, 1, 0, s[half]);
        }
    };
#undef FVAR_S
    // A half's scores once more, by bf16 products of what its keys and the queries' pieces stand for, which are added in fp32.
    auto exact = [&](int half, int kb) __attribute__((always_inline)) {
        const float ksize = __uint_as_float((uint32_t)kb << 23);
        s[half] = bases;
#pragma unroll
        for (int p = 1; p >= 0; --p) {
            float size = __uint_as_float((uint32_t)(qbyte >> (8 * p) & 255) << 23);
            asm volatile("" : "+v"(size));                   // (or the queries are converted ahead of the loop, into registers that there are none of)
#pragma unroll
            for (int i = 0; i < KS * 4; ++i) {
                const uintx4_t w = *(lds_uintx4_t *)(kp[i / 4][i / 2 % 2] + half * (RAW / 2));
                const bf16x8_t kf = __builtin_bit_cast(bf16x8_t, i & 1 ? bf16_eight(w[2], w[3], ksize) : bf16_eight(w[0], w[1], ksize));
                const bf16x8_t qe = __builtin_bit_cast(bf16x8_t, bf16_eight(qf[i / 4][p][i % 4 * 2], qf[i / 4][p][i % 4 * 2 + 1], size));
                s[half] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qe, s[half], 0, 0, 0);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    };
    auto load_v = [&](int i, int rows) -> f16x8_t {
        const shortx4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4_t *)(vp[i][0] + rows * DH * 2));
        const shortx4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4_t *)(vp[i][1] + rows * DH * 2));
        return __builtin_bit_cast(f16x8_t, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    };
    // One half's softmax beside the scores of the other (of the next tile where that is the first) and the products of the other's
    // weights (of the tile before where that is the second).  A step: a product, the weights of a pair or two in three stages.
    auto region = [&](auto which, int kb) {
        constexpr int half = decltype(which)::value, other = 1 - half;
        constexpr int NS = 2 * KS, NPV = 2 * DB, STEPS = NS + NPV, PP = DH == 128 ? 1 : 2;     // PP: pairs of weights per step
        uintx4_t k[KS][2];
        f16x8_t vf[DB];
        load_keys(other, k);
#pragma unroll
        for (int i = 0; i < DB; ++i) vf[i] = load_v(i, 0);
        if constexpr (half == 0) read_raw(vslot ^ 1, raw);
        __builtin_amdgcn_sched_barrier(0);
        float x[16], a, bsum;
#pragma unroll
        for (int step = 0; step < STEPS; ++step) {
            const int before = min((step + 1) / 2, NS);      // scores' products up to here, this one included if it is one
            if ((step & 1) && step / 2 < NS) {
                score(other, step / 2, k, kb);
            } else {
                const int i = step - before;
                acc[i % DB] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vf[i % DB], pf[other][i / DB], acc[i % DB], 0, 0, 0);
                if (i < DB) vf[i] = load_v(i, 16);
            }
#pragma unroll
            for (int w = 0; w < PP; ++w) {
                const int p2 = (step - 2) * PP + w, p1 = (step - 1) * PP + w, p0 = step * PP + w;
                if (p1 >= 0 && p1 < 8) {
                    x[2 * p1] = __builtin_amdgcn_exp2f(x[2 * p1]);
                    x[2 * p1 + 1] = __builtin_amdgcn_exp2f(x[2 * p1 + 1]);
                }
                if (p0 < 8) {
                    x[2 * p0] = exponent(s[half][2 * p0]);
                    x[2 * p0 + 1] = exponent(s[half][2 * p0 + 1]);
                }
                if (p2 >= 0 && p2 < 8) {
                    a = p2 ? a + x[2 * p2] : x[0];
                    bsum = p2 ? bsum + x[2 * p2 + 1] : x[1];
                    asm volatile("" : "+v"(a), "+v"(bsum));  // here, not after the region with all of x alive until then
                    const f16x2v_t p = __builtin_convertvector((floatx2_t{x[2 * p2], x[2 * p2 + 1]}), f16x2v_t);
                    pf[half][p2 >> 2][(2 * p2) & 7] = p[0];
                    pf[half][p2 >> 2][(2 * p2 + 1) & 7] = p[1];
                }
            }
            if constexpr (half == 1) {
                constexpr int from = DH == 128 ? 6 : 3;
                if (step >= from && step - from < VW) convert(raw, step - from);
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
    auto renew = [&](int half) __attribute__((always_inline)) {
        float mx = s[half][0];
#pragma unroll
        for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[half][i]);
        const auto halves = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
        mx = fmaxf(__uint_as_float(halves[0]), __uint_as_float(halves[1]));
        const bool had = most >= 0.f, none = !had && mx == -INFINITY;
        float alpha = 1.f;
        const float over = FROM ? mx : mx - m_ref;
        if (!none && (!had || over > 0.f)) {
            if constexpr (FROM) {
                s[0] -= mx;
                s[1] -= mx;
            }
            set_base(FROM ? m_ref + mx : mx);
            alpha = __builtin_amdgcn_exp2f(-over * c_log2);
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
            const float x = __builtin_amdgcn_exp2f(exponent(s[half][i]));
            const float y = __builtin_amdgcn_exp2f(exponent(s[half][i + 1]));
            sum += x + y;
            const f16x2v_t p = __builtin_convertvector((floatx2_t{x, y}), f16x2v_t);
            pf[half][i >> 3][i & 7] = p[0];
            pf[half][i >> 3][(i & 7) + 1] = p[1];
        }
    };
    auto settle = [&](int half, int kb) __attribute__((always_inline)) {     // kb: of the keys whose scores the region has made
        // The reference is not the running maximum but one that was it; the weights tell when it no longer serves.  A sum of NaN
        // does not ask for another: it stays NaN.
        const bool anew = (__builtin_amdgcn_ballot_w64(sum > most) != 0 && (uint32_t)(vis >> (32 * half)) != 0) || E_now != acc_E;
        if (__builtin_expect(anew || kb > plain_to, 0)) {
            if (kb > plain_to) exact(1 - half, kb);
            if (anew) renew(half);
        }
        l_run += sum;
    };
    auto to_half = [&](int to) {                             // vp goes on to half tile `to`
        const int by = (to - rslot) * HALF;
        rslot = to;
#pragma unroll
        for (int i = 0; i < DB; ++i) { vp[i][0] += by; vp[i][1] += by; }
    };

    E_now = E;
    {
        uintx4_t k[KS][2];
        load_keys(0, k);
        const int kb = byte_of(kbytes, t0, 0);
#pragma unroll
        for (int i = 0; i < 2 * KS; ++i) score(0, i, k, kb);
        if (__builtin_expect(kb > plain_to, 0)) exact(0, kb);
    }
    for (int t = t0; t <= t1; ++t) {
        const int tn = min(t + 1, t1);
        fetch(min(t + 2, t1), after(after(kslot)), vslot);
        hide(0);
        const int kb1 = byte_of(kbytes, t, 1);
        region(std::integral_constant<int, 0>{}, kb1);
        settle(0, kb1);
        {
            // values go on to this tile's first half, keys to the next tile's
            to_half(t == t0 ? 0 : next_half(rslot, 1));
            const int k_by = kslot == 2 ? -2 * RAW : RAW;
#pragma unroll
            for (int i = 0; i < KS; ++i) { kp[i][0] += k_by; kp[i][1] += k_by; }
        }
        hide(1);
        vis_next = look(tn, raw, seen_next);
        const int kb0 = byte_of(kbytes, tn, 0);
        region(std::integral_constant<int, 1>{}, kb0);
        settle(1, kb0);
        to_half(next_half(rslot, 1));
        cslot = next_half(cslot, 2);
        seen_next = seen_later;
        vis = vis_next;
        kslot = after(kslot);
        vslot ^= 1;
        E_now = E;
        meet();
    }
    if (most < 0.f) m_ref = -INFINITY;
    // the last half's products
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int i = 0; i < DB; ++i)
            acc[i] = __builtin_amdgcn_mfma_f32_32x32x16_f16(load_v(i, 16 * u), pf[1][u], acc[i], 0, 0, 0);

    // ---- means, back at their size (see kTop)
    {
        const auto halves = __builtin_amdgcn_permlane32_swap(__float_as_uint(l_run), __float_as_uint(l_run), false, false);
        l_run = __uint_as_float(halves[0]) + __uint_as_float(halves[1]);
    }
    const float inv = l_run == 0.f ? 0.f : 1.0f / l_run;
    auto mean = [&](float x) { return __builtin_amdgcn_ldexpf(x * inv, acc_E - kTop); };
    const size_t prow = ((size_t)(unit - full_units) * shares + share) * 128 + wave * 32 + rl;
    uint16_t *dst = o + (size_t)(b * (long)n + row / G) * H * DH + (size_t)(hk * G + row % G) * DH;
    // Two quads of results that lie eight apart in the lane's row: four more stand in the lane 32 further, which changes one of its
    // quads for one of these, so that each stores 16 bytes.  A share's,
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
        if (g) return;
        if (ranges > 1) *reinterpret_cast<float2 *>(part_ml + prow * 2) = make_float2(m, l);
        else if (stats) stats[head * R + row] = make_float2(m, l * 0.00390625f);   // (without 2^kShift)
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

// Shares of a unit's keys that have been written (see kvb_attn_rows_kernel's chunk).
__device__ __forceinline__ int shares_written(int len, int shares, int chunk)
{
    return chunk ? max(min(((len + 31) / 32 + chunk - 1) / chunk, shares), 1) : shares;
}

// Weights of the rows where one block of sixteen rows is all, and kvb_attn_rows_kernel has left their scores: those are a few bytes for every
// key, which a second look at the keys would be 128 for.  Four keys per thread; workgroup `id` of `blocks` for every head.  The rows' references
// and sums come from stats, or, where the keys have been divided, from the shares' (16 threads a row).
__device__ __forceinline__ void weigh_few(const KvbCache &c, int extra, int R, float c_log2, const float2 *stats, const float *part_ml, int shares,
                                          int chunk, const float *scores, int pitch, float *weights, int add, int id, int blocks, float unit)
{
    __shared__ float2 rows[16];
    const int head = id / blocks, b = head / c.heads, len = kvb_length(c, b, extra), key = (id % blocks * 256 + threadIdx.x) * 4;
    if (id % blocks * 1024 >= len) return;                   // (the whole workgroup)
    const int r = threadIdx.x >> 4, from = threadIdx.x & 15;
    if (part_ml) {
        const int here = shares_written(len, shares, chunk);
        float m = -INFINITY, l = 0.f;
        for (int s = from; s < here; s += 16) {
            const float2 x = *reinterpret_cast<const float2 *>(part_ml + (((size_t)head * shares + s) * 16 + r) * 2);
            const float now = fmaxf(m, x.x);
            l = l * __builtin_amdgcn_exp2f((m - reference(now)) * c_log2) + x.y * __builtin_amdgcn_exp2f((x.x - reference(now)) * c_log2);
            m = now;
        }
#pragma unroll
        for (int o = 1; o < 16; o <<= 1) {
            const float m2 = __shfl_xor(m, o), l2 = __shfl_xor(l, o), now = fmaxf(m, m2);
            l = l * __builtin_amdgcn_exp2f((m - reference(now)) * c_log2) + l2 * __builtin_amdgcn_exp2f((m2 - reference(now)) * c_log2);
            m = now;
        }
        if (from == 0) rows[r] = make_float2(m, l * unit);
    } else if (threadIdx.x < R) {
        rows[threadIdx.x] = stats[(size_t)head * R + threadIdx.x];
    }
    __syncthreads();
    if (key >= len) return;
    const float *src = scores + ((size_t)head * pitch + key / 32) * (R * 32) + key % 32;
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
    for (int r0 = 0; r0 < R; r0 += 4) {                      // four rows' scores at a time on their way
        float4 s[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) s[i] = *reinterpret_cast<const float4 *>(src + min(r0 + i, R - 1) * 32);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 stat = rows[min(r0 + i, R - 1)];
            if (r0 + i >= R || !(stat.y > 0.f)) continue;
            const float m = reference(stat.x), each = 1.0f / stat.y;
            sum[0] += __builtin_amdgcn_exp2f((s[i].x - m) * c_log2) * each;
            sum[1] += __builtin_amdgcn_exp2f((s[i].y - m) * c_log2) * each;
            sum[2] += __builtin_amdgcn_exp2f((s[i].z - m) * c_log2) * each;
            sum[3] += __builtin_amdgcn_exp2f((s[i].w - m) * c_log2) * each;
        }
    }
    const uint8_t *mask = c.mask ? c.mask + (size_t)b * c.capacity : nullptr;
    float *to = weights + (size_t)head * c.capacity;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (key + i >= len) return;
        const float x = !mask || mask[key + i] != 0 ? sum[i] : 0.f;
        to[key + i] = add ? to[key + i] + x : x;
    }
}
__global__ __launch_bounds__(256) void kvb_weights_few_kernel(KvbCache c, int extra, int R, float c_log2, const float2 *__restrict__ stats,
                                                              const float *__restrict__ scores, int pitch, float *__restrict__ weights, int add,
                                                              int blocks)
{
    weigh_few(c, extra, R, c_log2, stats, nullptr, 1, 0, scores, pitch, weights, add, blockIdx.x, blocks, 1.f);
}

// The shares of rows joined: each is a mean and its weight.  A unit is a block of BR rows of one (sample, kv head); the shares
// of unit first + u lie at [u][share][row].  GROUPS groups of DH/4 threads per row, four head-dim elements a thread: a group takes every
// GROUPS-th share, four at a time, with a running reference and mean (not the sum: a mean times its weight need not be a number that fp32
// holds), and the groups meet in LDS.  One group where the shares are few and the
// rows many; more where a few rows have many shares, whose loads would wait for each other (64 shares of 16 rows: 24 us by one, 3 by 8).
template <typename T, int DH, int GROUPS>
__global__ __launch_bounds__(256) void kvb_attn_merge_kernel(const float *__restrict__ part_o, const float *__restrict__ part_ml,
                                                             KvbCache c, int extra, int n, int H, int nrb, int BR, int first, int shares,
                                                             int chunk, float c_log2, int total, T *__restrict__ o, float2 *__restrict__ stats,
                                                             const float *__restrict__ scores, int pitch, float *__restrict__ weights, int add,
                                                             int merges, int blocks)
{
    if (blockIdx.x >= merges) {                              // the rows' weights, which need not wait for the joined results
        weigh_few(c, extra, n * (H / c.heads), c_log2, nullptr, part_ml, shares, chunk, scores, pitch, weights, add, blockIdx.x - merges, blocks,
                  sizeof(T) == 4 ? 1.f : 0.00390625f);
        return;
    }
    constexpr int W = DH / 4, ROWS = 256 / (W * GROUPS);     // threads of a group, rows of a workgroup
    __shared__ float4 lo[GROUPS > 1 ? 256 : 1];
    __shared__ float2 lm[GROUPS > 1 ? 256 / W : 1];
    const int d = threadIdx.x % W * 4, group = threadIdx.x / W % GROUPS, in_wg = threadIdx.x / (W * GROUPS);
    const int idx = blockIdx.x * ROWS + in_wg;               // row among those of the divided units
    const int r = idx % BR, u = idx / BR, unit = first + u;
    const int G = H / c.heads, row = unit % nrb * BR + r, hk = unit / nrb % c.heads;
    const long b = unit / nrb / c.heads;
    const bool mine = idx < total && row < n * G;
    const size_t prow = (size_t)u * shares * BR + r;
    // shares that have been written
    const int here = chunk && mine ? shares_written(kvb_length(c, (int)b, extra), shares, chunk) : shares;
    auto weight = [&](float2 ml, float m) { return ml.y * __builtin_amdgcn_exp2f((ml.x - reference(m)) * c_log2); };
    float m = -INFINITY, sum = 0.f;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    auto put_in = [&](float4 v, float w) {
        acc.x = fmaf(v.x, w, acc.x); acc.y = fmaf(v.y, w, acc.y); acc.z = fmaf(v.z, w, acc.z); acc.w = fmaf(v.w, w, acc.w);
    };
    if (mine) {
        for (int s = group; s < here; s += 4 * GROUPS) {
            float2 ml[4];
            float4 v[4];
            float now = m, w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const bool there = s + i * GROUPS < here;  // (instead of one that is not, the first with a weight of 0)
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
            for (int i = 0; i < 4; ++i) put_in(v[i], w[i] * each);
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
        for (int k = 0; k < GROUPS; ++k) put_in(lo[threadIdx.x + k * W], weight(lm[threadIdx.x / W + k], m) * each);
    }
    if (mine) {
        Quad<T>::store(o + (size_t)(b * n + row / G) * H * DH + (size_t)(hk * G + row % G) * DH + d, acc);
        if (stats && d == 0) stats[(size_t)(unit / nrb) * n * G + row] = make_float2(m, sizeof(T) == 4 ? sum : sum * 0.00390625f);
    }
}

// Weights of the rows: every wavefront holds 64 keys as bf16 operands, takes the scores of all rows of queries against them once more, and
// adds up exp2((s - reference) * c) / sum over the rows, each key's in its own registers: no atomics, one order.  64 rows at a time come
// through LDS for the W wavefronts, by DMA while the ones before are at work (32 in fp32, in three pieces of bf16, and for a single wavefront of 128-wide
// rows, which 64 would run out of registers).  A row whose weights are not numbers adds nothing.
//   A workgroup: a block of 64 W keys of one of `heads` (sample, kv head), and a share of its rows; several shares leave partial sums
// [share][heads][64 W blocks].
template <typename T, int DH, int W>
__global__ __launch_bounds__(64 * W, 2) void kvb_weights_kernel(const T *__restrict__ q, int ld, KvbCache c, int extra, int n, int H, float c_log2,
                                                             const float2 *__restrict__ stats, float *__restrict__ weights, int add,
                                                             float *__restrict__ part, int blocks, int heads, int shares)
{
    constexpr bool F32 = sizeof(T) == 4;
    constexpr int NP = F32 ? 3 : 1, KS = DH / 16, CH = DH / 8;   // CH: chunks of eight elements of a row
    constexpr int SETS = F32 || (W == 1 && DH == 128) ? 1 : 2, ROWS = 32 * SETS, PER = ROWS * CH / (64 * W);
    __shared__ uint4 ql[2][NP][ROWS * CH];
    const int tid = threadIdx.x, lane = tid & 63, rl = lane & 31, g = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    // the blocks of a head, which read the same rows of queries, on one XCD, unless samples differ in length
    const int id = c.lens ? blockIdx.x : xcd_contiguous(blockIdx.x, gridDim.x);
    const int block = id % blocks, head = id / blocks % heads, share = id / blocks / heads, b = head / c.heads, hk = head % c.heads;
    const int G = H / c.heads, R = n * G, len = kvb_length(c, b, extra);
    const int key0 = (block * W + wave) * 64;
    if (block * (64 * W) >= len) return;                          // (of the whole workgroup)
    const int tiles = (R + ROWS - 1) / ROWS, t0 = (int)((long)tiles * share / shares), t1 = (int)((long)tiles * (share + 1) / shares);

    // ---- rows of queries: chunks are turned by the row's number, so that the rows of sixteen lanes that read one chunk lie in all banks
    auto turn = [](int row) { return DH == 128 ? row & 15 : (row >> 1) & 7; };
    const uint32_t lds_base = (uint32_t)(uintptr_t)ql;
    const T *first = q + (size_t)b * n * ld + hk * G * DH;
    const int shift = (G & (G - 1)) == 0 ? __builtin_ctz(G) : -1;    // (a division for every piece would take as long as a third of the products)
    uint4 next[F32 ? PER : 1][2];
    float2 next_stat[SETS];
    auto fetch = [&](int t, int buffer) {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int at = F32 ? i * (64 * W) + tid : (wave * PER + i) * 64 + lane;
            const int in_tile = at / CH, row = min(t * ROWS + in_tile, R - 1);
            const int query = shift >= 0 ? row >> shift : row / G;
            const size_t src = (size_t)query * ld + (row - query * G) * DH;
            if constexpr (F32) {
                next[i][0] = *reinterpret_cast<const uint4 *>(first + src + at % CH * 8);
                next[i][1] = *reinterpret_cast<const uint4 *>(first + src + at % CH * 8 + 4);
            } else {
                // (addresses of any distance from q: 64 bits per lane)
                const uint16_t *from = first + src + ((at % CH) ^ turn(in_tile)) * 8;
                asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off"
                             :: "s"(lds_base + (buffer * ROWS * CH + (wave * PER + i) * 64) * 16), "v"(from) : "memory", "m0");
            }
        }
#pragma unroll
        for (int j = 0; j < SETS; ++j) next_stat[j] = stats[(size_t)head * R + min(t * ROWS + j * 32 + rl, R - 1)];
    };
    auto put = [&](int buffer) {
        if constexpr (F32) {
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const int at = i * (64 * W) + tid, to = at / CH * CH + ((at % CH) ^ turn(at / CH));
                float x[8];
                bf16x8_t pieces[3];
                Elem<float>::unpack(next[i][0], x);
                Elem<float>::unpack(next[i][1], x + 4);
                three_pieces(x, pieces);
#pragma unroll
                for (int p = 0; p < 3; ++p) ql[buffer][p][to] = __builtin_bit_cast(uint4, pieces[p]);
            }
        } else {
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        }
    };
    if (t0 < t1) fetch(t0, 0);

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

    // The weights of 32 rows are made beside the products of the next ones, an exponential or two for each product (fp32, with three products
    // where bf16 has one and no registers for both: after their own).
    floatx16_t acc[2] = {floatx16_t{0}, floatx16_t{0}}, s[2] = {floatx16_t{0}, floatx16_t{0}};
    float m = 0.f, each = 0.f, mc = INFINITY;                  // of the rows whose scores s are: reference, 1 / sum, reference in units of log2
    bool plain = true;
    auto weigh = [&]() {
        // the difference first, exact near the reference; at most 1: scores of 2^20 and more differ by more than that between
        // two ways to add their products up, and 0 for what is not a number
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int i = 0; i < 16; ++i)
                acc[u][i] += __builtin_amdgcn_fmed3f(__builtin_amdgcn_exp2f((s[u][i] - m) * c_log2) * each, 0.f, 1.f);
    };
    // (what mc's rounding leaves is in `each`)
    auto weigh_plain = [&](int e) {
        acc[e >> 4][e & 15] = fmaf(__builtin_amdgcn_exp2f(fmaf(s[e >> 4][e & 15], c_log2, -mc)), each, acc[e >> 4][e & 15]);
    };
    auto finish = [&]() {
        if (plain) {
#pragma unroll
            for (int e = 0; e < 32; ++e) weigh_plain(e);
        } else {
            weigh();
        }
    };
    auto products = [&](auto beside, int buffer, int j) {
        constexpr int EACH = 32 / (2 * KS);
        floatx16_t now[2] = {floatx16_t{0}, floatx16_t{0}};
#pragma unroll
        for (int i = 0; i < KS; ++i) {
            bf16x8_t qf[NP];
#pragma unroll
            for (int p = 0; p < NP; ++p) qf[p] = __builtin_bit_cast(bf16x8_t, ql[buffer][p][(j * 32 + rl) * CH + ((g * KS + i) ^ turn(rl))]);
#pragma unroll
            for (int u = 0; u < 2; ++u) {
#pragma unroll
                for (int p = NP - 1; p >= 0; --p) now[u] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[u][i], qf[p], now[u], 0, 0, 0);
                if constexpr (decltype(beside)::value) {
#pragma unroll
                    for (int e = 0; e < EACH; ++e) weigh_plain((2 * i + u) * EACH + e);
                }
            }
        }
        s[0] = now[0];
        s[1] = now[1];
    };

    if (t0 < t1) put(0);
    for (int t = t0; t < t1; ++t) {
        float2 stat[SETS];
#pragma unroll
        for (int j = 0; j < SETS; ++j) stat[j] = next_stat[j];
        const int buffer = (t - t0) & 1;
        __syncthreads();                                     // this tile's rows are there, the other buffer has been read
        if (t + 1 < t1) fetch(t + 1, buffer ^ 1);
#pragma unroll
        for (int j = 0; j < SETS; ++j) {
            // (a set without a row would be the last row's copies: products for nothing, and where that row's scores are no numbers, no lane would tell)
            if (j && t * ROWS + j * 32 >= R) break;
            if (!F32 && __builtin_expect(plain, 1)) {
                products(std::true_type{}, buffer, j);
            } else {
                if constexpr (!F32) weigh();
                products(std::false_type{}, buffer, j);
            }
            const bool there = t * ROWS + j * 32 + rl < R, counts = there && stat[j].y > 0.f;
            m = counts ? reference(stat[j].x) : 0.f;
            each = counts ? 1.0f / stat[j].y : 0.f;
            mc = counts ? m * c_log2 : INFINITY;             // (a row that does not count: weights of 0, whatever its scores)
            plain = __builtin_amdgcn_ballot_w64(there != counts || (counts && fabsf(mc) >= 4096.f)) == 0;
            if (plain && counts) each *= __builtin_amdgcn_exp2f(-fmaf(m, c_log2, -mc));
            if constexpr (F32) finish();
        }
        if (t + 1 < t1) put(buffer ^ 1);
    }
    if constexpr (!F32) finish();

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
    if (shares > 1) {
        part[((size_t)share * heads + head) * (64 * W * blocks) + key] = mine;
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

// Blocks of how many rows of a (sample, kv head) an attention is run by: 16 (kvb_attn_rows_kernel) or 128 (kvb_attn_tiles_kernel, bf16
// only).  The first starts and ends soonest and is bound by the work, which it does at less than half the other's pace; the other fetches
// and converts for 128 rows whatever there are, and joins groups and shares.  So the work decides, with 64-wide rows, which take the first less, at two
// thirds more, and at half a block and less at five times as much; and a tile of the other's 64 keys that is all there is has nothing to run beside it.  us by 16 / by
// 128, 16 heads of 128: 1 x 144 rows x 265 keys 7 / 15, 1 x 400 x 921 15 / 23, 2 x 400 x 400 16.9 / 17.7, 4 x 400 x 250 18.7 / 15.1, 8 x 400 x 200 27.9 / 20.2,
// 1 x 800 x 600 19.9 / 18.8, 1 x 200 x 4813 33 / 26, 32 x 400 x 60 41 / 45; 8 x 64 x 2521 29 / 34, 16 x 64 x 3000 63 / 50, 8 x 32 x 3001 20 / 35,
// 32 x 32 x 3001 92 / 85, 32 x 48 x 3001 117 / 101; 30 heads of 64: 1 x 324 x 640 10 / 13, 2 x 231 x 871 15 / 16, 4 x 400 x 200 12.8 / 13.6, 25 x 1043 x 29
// 73 / 80; 16 heads of 64, 2 x 128 x 2000, 10.5 / 16.9.
static int kvb_block(DType dt, int B, int n, int H, int heads, int Dh, int length)
{
    const int rows = n * (H / heads);
    if (dt != DType::BF16 || rows <= 16 || length <= 64) return 16;
    return (long)B * heads * ((rows + 15) / 16) * length <= (rows <= 64 ? 16l << 17 : Dh == 64 ? 5l << 17 : 3l << 17) ? 16 : 128;
}

// nrb blocks per (sample, kv head), units in all, of which the first `full` take all keys and each other one is divided into `shares`.
// `ragged`: samples of lengths of their own, which only the GPU knows.
// waves: wavefronts of a workgroup, 1, 2, 4 or 8, which divide a block's keys (16 rows), or 4 or 8, which divide its rows and, if there are 8, keys (128 rows).
// chunk: 16 rows, samples of lengths of their own: tiles of 32 keys of a share, so that workgroups have as much to do whatever the lengths.
struct KvbRun { int block, nrb, units, full, shares, waves, chunk; };
constexpr int kGroupsFrom = 2048, kGroupsTo = 4096;          // lengths at which the choice between one and two groups changes
static KvbRun kvb_run(int block, int B, int n, int H, int heads, int Dh, int length, bool ragged)
{
    KvbRun run;
    run.block = block;
    run.nrb = (n * (H / heads) + block - 1) / block;
    run.units = B * heads * run.nrb;
    run.waves = 4;
    run.chunk = 0;
    if (block == 16) {
        const int tiles = (length + 31) / 32;
        // Eight wavefronts where there are more tiles than that to divide and at most a workgroup for every CU: fewer shares to join, or
        // none (1 query of 16 heads of 128 over 600 keys 8.2 us in one launch, 7.7 + 2.8 by four; fp32, 2 x 128 x 552, 16 heads of 64, 8.8, 10.1).
        // One where there is a single tile, or where blocks alone fill every SIMD's two places, two for two tiles and half as many blocks: no
        // wavefront that waits, nothing to join (us by one / two / four: 9 x 370 rows x 26 keys, 30 heads of 64, 11.6 / - / 27.8; 16 heads of 128, 32 x 64
        // x 119, 13.3 / 15.8 / 20.4, x 500 27.9 / - / 33.7, 16 x 64 x 500 - / 17.6 / 20.4; 2 x 64 x 100 9.1 / - / 5.5).
        run.waves = run.units <= 256 && tiles > 16 && !ragged ? 8 : tiles <= 1 || run.units >= 2048 ? 1 : tiles <= 2 || run.units >= 1024 ? 2 : 4;
        // Enough wavefronts for two on every SIMD; four where samples differ, with shares as long as each other, so that a CU that has had
        // short ones takes more (32 samples of 1 to 16921 keys, 8 kv heads, 512, 1024, 2048, 4096 places: 127, 105, 108, 102 us and a joining of
        // 4.8, 4.8, 4.8, 9.8).  Each with two tiles per wavefront at least, or eight where every CU has a workgroup already.
        const int places = ragged ? 1024 : 2048 / run.waves, least = run.units < 256 ? 2 : 8;
        const int want = (places + run.units - 1) / run.units, most = tiles / (least * run.waves);
        run.shares = want < most ? want : most > 0 ? most : 1;
        if (ragged && run.shares > 1) run.chunk = (tiles + run.shares - 1) / run.shares;
        run.full = run.shares > 1 ? 0 : run.units;
        return run;
    }
    // Up to a workgroup on every CU: two groups of wavefronts in each, and shares where there are half as many or fewer.  Otherwise, and over long
    // caches where shares of one group leave fewer CUs idle, two workgroups on every CU (three of 64-wide rows, where there are two rounds of
    // them); those beyond the last full round are divided.  Pieces have four tiles at least for each group.  A quarter of a round more than one
    // by two groups, divided, is also soonest done so, if there is enough to divide.  us by one / by two groups, 16 heads of 128: 4 x 300 x 2500 keys
    // 55 / 43, 1 x 200 x 4813 31 / 26, 1 x 1152 x 6000 78 / 87, 1 x 1600 x 2500 56 / 44; 30 heads of 64: 8 x 231 x 871 26 / 31, 1 x 640 x 6000 54 / 63, 1 x 1152
    // x 6000 121 / 83.
    const int two = Dh == 64 && run.units >= 2 * 768 ? 768 : 512;
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

// Whether the weights come from scores that the attention leaves (see kvb_weights_few_kernel), and the tiles of them.
static bool few_rows(int rows) { return rows <= 16; }
static size_t score_tiles(int length) { return ((size_t)length + 31) / 32; }

// Shares of the rows of queries for the weights: where the keys alone do not fill the chip.
constexpr int kWeightPlaces = 512;
// A single wavefront for each, where it has all keys there are and the heads alone are as many as the CUs: with four, three would have none (us by one / by
// four, joining included: 30 heads of 64, 9 x 370 rows x 26 keys 12.8 / 15.4, 25 x 1043 x 29 31 / 55; 16 heads of 128, 32 x 400 x 50 21 / 24, 32 x 36 x
// 55 6.3 / 8.1; 8 x 97 x 60, heads of 64, 9.6 / 9.1, 2 x 375 x 2 11.3 / 10.3).
static int weight_waves(DType dt, int B, int heads, int length) { return dt == DType::BF16 && length <= 64 && (long)B * heads >= 256 ? 1 : 4; }
static int weight_shares(int B, int heads, int length, int rows, int waves)
{
    const long wgs = (long)B * heads * ((length + 64 * waves - 1) / (64 * waves));
    long shares = wgs > 0 ? kWeightPlaces * 4 / waves / wgs : 1;
    if (shares > (rows + 31) / 128) shares = (rows + 31) / 128;      // (fewer than 128 rows each are not worth a joining)
    return (int)(shares > 8 ? 8 : shares < 1 ? 1 : shares);
}

// Floats that partial results take, and, before them, what the weights need: every row's reference and sum; their scores, or partial sums of
// at most kWeightPlaces workgroups of 256 keys, or four times as many of 64.
static size_t part_floats(const KvbRun &run, int Dh) { return (size_t)(run.units - run.full) * run.shares * run.block * (Dh + 2); }
static size_t stat_floats(int B, int n, int H) { return (2 * (size_t)B * n * H + 3) / 4 * 4; }
static size_t weight_floats(int B, int n, int H, int heads, int length)
{
    return few_rows(n * (H / heads)) ? (size_t)B * n * H * 32 * score_tiles(length) : 256 * kWeightPlaces;
}

size_t kvb_attention_scratch_floats(DType dt, int B, int n, int H, int heads, int Dh, int capacity, bool weights)
{
    // Between those lengths shares never fall as the length grows, nor where samples have lengths of their own, so for either kind of
    // blocks the longest length of each stretch is enough for every call; a shorter length may be run by the other kind.
    size_t floats = 0;
    for (int length : {capacity, kGroupsTo - 1, kGroupsFrom - 1}) {
        if (length > capacity) continue;
        for (int block = 16; block <= 128; block *= 8) {
            if (block == 128 ? kvb_block(dt, B, n, H, heads, Dh, length) == 16 : kvb_block(dt, B, n, H, heads, Dh, 1) == 128) continue;
            const size_t take = part_floats(kvb_run(block, B, n, H, heads, Dh, length, true), Dh);
            if (take > floats) floats = take;
        }
    }
    return floats + (weights ? stat_floats(B, n, H) + weight_floats(B, n, H, heads, capacity) : 0);
}

// How an attention is run, and the floats that it takes, for the tests: 100000 * rows of a block + 1000 * wavefronts + shares.
int kvb_attention_ways(int bf16, int B, int n, int H, int heads, int Dh, int length, int ragged)
{
    const int block = kvb_block(bf16 ? DType::BF16 : DType::F32, B, n, H, heads, Dh, length);
    const KvbRun run = kvb_run(block, B, n, H, heads, Dh, length, ragged != 0);
    return 100000 * block + 1000 * run.waves + run.shares;
}
long kvb_attention_takes(int bf16, int B, int n, int H, int heads, int Dh, int length, int ragged, int weights)
{
    const int block = kvb_block(bf16 ? DType::BF16 : DType::F32, B, n, H, heads, Dh, length);
    const size_t part = part_floats(kvb_run(block, B, n, H, heads, Dh, length, ragged != 0), Dh);
    return (long)(part + (weights ? stat_floats(B, n, H) + weight_floats(B, n, H, heads, length) : 0));
}

template <typename T, int DH>
static void launch_kvb(const void *q, int ld, const KvbCache &c, int extra, int B, int n, int H, float c_log2, void *o, float *weights, bool add,
                       float *part, hipStream_t st)
{
    const int length = c.lens ? c.capacity : c.len + extra;
    const DType dt = sizeof(T) == 2 ? DType::BF16 : DType::F32;
    const KvbRun run = kvb_run(kvb_block(dt, B, n, H, c.heads, DH, length), B, n, H, c.heads, DH, length, c.lens != nullptr);
    const int divided = run.units - run.full;
    float2 *stats = nullptr;
    float *sums = part, *scores = nullptr;
    const int rows = n * (H / c.heads), pitch = (int)score_tiles(length);
    if (weights) {
        stats = reinterpret_cast<float2 *>(part);
        sums = part + stat_floats(B, n, H);
        scores = few_rows(rows) ? sums : nullptr;
        part = sums + weight_floats(B, n, H, c.heads, length);
    }
    float *part_ml = part + (size_t)divided * run.shares * run.block * DH;
    const unsigned wgs = (unsigned)(run.full + divided * run.shares);
#define FVAR_ROWS(NW, MASKED)                                                                                            \
    launch(kvb_attn_rows_kernel<T, DH, NW, MASKED>, dim3(wgs), dim3(64 * NW), 0, st, (const T *)q, ld, c, extra, n, H,    \
           c_log2, (T *)o, run.nrb, run.shares, run.chunk, part, part_ml, stats, scores, pitch)
    if (run.block == 16) {
        if (run.waves == 8) { if (c.mask) FVAR_ROWS(8, true); else FVAR_ROWS(8, false); }
        else if (run.waves == 4) { if (c.mask) FVAR_ROWS(4, true); else FVAR_ROWS(4, false); }
        else if (run.waves == 2) { if (c.mask) FVAR_ROWS(2, true); else FVAR_ROWS(2, false); }
        else { if (c.mask) FVAR_ROWS(1, true); else FVAR_ROWS(1, false); }
#undef FVAR_ROWS
    } else if constexpr (sizeof(T) == 2) {
#define FVAR_TILES(KG, WAVES)                                                                                            \
    launch(kvb_attn_tiles_kernel<DH, KG, WAVES>, dim3(wgs), dim3(256 * KG), 0, st, (const T *)q, ld, c, extra, n, H,             \
           c_log2, (T *)o, run.nrb, run.full, run.shares, part, part_ml, stats)
        if (run.waves == 8) FVAR_TILES(2, 2);
        else if (DH == 64 && run.units >= 2 * 768) FVAR_TILES(1, DH == 64 ? 3 : 2);
        else FVAR_TILES(1, 2);
#undef FVAR_TILES
    }
    const int few_blocks = (length + 1023) / 1024, few_wgs = scores ? few_blocks * B * c.heads : 0;
    if (divided) {
        const int total = divided * run.block, per = 256 / (DH / 4);
        const bool eight = run.shares > 8 || (run.shares > 2 && total <= 1024);
        const int merges = eight ? (total + per / 8 - 1) / (per / 8) : (total + per - 1) / per;
#define FVAR_MERGE(GROUPS)                                                                                               \
    launch(kvb_attn_merge_kernel<T, DH, GROUPS>, dim3((unsigned)(merges + few_wgs)), dim3(256), 0, st, (const float *)part, (const float *)part_ml, \
           c, extra, n, H, run.nrb, run.block, run.full, run.shares, run.chunk, c_log2, total, (T *)o, stats, (const float *)scores, pitch, weights, \
           add ? 1 : 0, merges, few_blocks)
        if (eight) FVAR_MERGE(8);
        else FVAR_MERGE(1);
#undef FVAR_MERGE
    }
    if (scores) {
        if (!divided && length > 0)
            launch(kvb_weights_few_kernel, dim3((unsigned)few_wgs), dim3(256), 0, st, c, extra, rows, c_log2, (const float2 *)stats,
                   (const float *)scores, pitch, weights, add ? 1 : 0, few_blocks);
    } else if (weights && length > 0) {
        const int waves = weight_waves(dt, B, c.heads, length), blocks = (length + 64 * waves - 1) / (64 * waves), shares = weight_shares(B, c.heads, length, rows, waves);
#define FVAR_WEIGHTS(W)                                                                                                  \
    launch(kvb_weights_kernel<T, DH, W>, dim3((unsigned)(blocks * B * c.heads * shares)), dim3(64 * W), 0, st, (const T *)q, ld, c, extra, n, H, c_log2, \
           (const float2 *)stats, weights, add ? 1 : 0, sums, blocks, B * c.heads, shares)
        if (waves == 4) FVAR_WEIGHTS(4);
        else if constexpr (sizeof(T) == 2) {
            FVAR_WEIGHTS(1);
        }
#undef FVAR_WEIGHTS
        if (shares > 1)
            launch(kvb_weights_join_kernel, dim3((unsigned)((length + 255) / 256), (unsigned)(B * c.heads)), dim3(256), 0, st, c, extra, (const float *)sums,
                   64 * waves * blocks, shares, weights, add ? 1 : 0);
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
