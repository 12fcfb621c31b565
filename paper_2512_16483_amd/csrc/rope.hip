// Rotary positions: the first `dim` elements of every head are `axes` parts of P = dim / axes elements; pair i of a part is turned by the
// angle p * f_i, p the part's component of the row's position and f_i the pair's entry of a table (in turns per position).
//   (x, y) -> magnitude * (x cos - y sin, x sin + y cos);  pairs are (i, i + P / 2), or (2 i, 2 i + 1) where interleaved.
//
// An angle is the fraction of p * f_i in 64 bits, off by 2^-34 of a turn at most for positions up to 10^6; sine and cosine of it in 32.
#include "common.h"

namespace fvar {

// Sixteen elements of a head, eight pairs, per thread; T rows per workgroup.  The angles of the workgroup's rows are made once, in LDS, for all heads
// of queries and keys: 64 of them serve 8192 elements of 32 + 32 heads of 128.  A thread keeps to its pairs and its row and goes from head to
// head with them in registers, FLY heads on their way at a time.  Memory-bound: 6400 rows of 32 + 32 heads of 128 in bf16 take 39.7 us with results
// past the caches (5.3 TB/s), the first heads fetched behind the angles 41.7, through the caches 3 more; four rows per workgroup 46, eight 53.  Few rows take their launch: 32 of 32 + 8 heads 3.7 us.
template <typename E, int DH, int T, bool INTER, bool PAST>
__global__ __launch_bounds__(256) void rope_kernel(RopeTable r, RopeRows q, RopeRows k, const int32_t *__restrict__ pos, int rows)
{
    constexpr int FLY = T == 1 ? 1 : 2, ITEMS = DH / 16, SLOTS = 256 / ITEMS / T, PER = Elem<E>::kPerChunk, HALF = 8 / PER;   // HALF: chunks of eight elements
    __shared__ float2 turn[T][DH / 2];
    const int tid = threadIdx.x, pairs = r.dim / 2, row0 = blockIdx.x * T;
    const int item = tid % ITEMS, t = tid / ITEMS % T, slot = tid / ITEMS / T;
    const size_t row = min(row0 + t, rows - 1);
    const int heads = row0 + t < rows ? q.heads + k.heads : 0;
    const bool turned = item * 16 < r.dim;
    int lo = item * 16, hi = item * 16 + 8;                  // the first of eight elements, and of eight more
    if (turned && !INTER) {
        const int part = r.dim / r.axes, each = part / 16, a = item / each;
        lo = a * part + item % each * 8;
        hi = lo + part / 2;
    }
    // FLY heads on their way at a time, the first of them while the angles are made
    uint4 raw[FLY][2 * HALF];
    E *dst[FLY];
    auto fetch = [&](int h0) __attribute__((always_inline)) {
#pragma unroll
        for (int f = 0; f < FLY; ++f) {
            const int h = min(h0 + f * SLOTS, q.heads + k.heads - 1);
            const bool is_q = h < q.heads;
            const int head = is_q ? h : h - q.heads;
            const E *src = (const E *)(is_q ? q.in : k.in) + row * (size_t)(is_q ? q.ld_in : k.ld_in) + head * DH;
            dst[f] = (E *)(is_q ? q.out : k.out) + row * (size_t)(is_q ? q.ld_out : k.ld_out) + head * DH;
            if (h0 + f * SLOTS >= heads || (!turned && src == dst[f])) dst[f] = nullptr;
#pragma unroll
            for (int i = 0; i < HALF; ++i) {
                raw[f][i] = *reinterpret_cast<const uint4 *>(src + lo + i * PER);
                raw[f][HALF + i] = *reinterpret_cast<const uint4 *>(src + hi + i * PER);
            }
        }
    };
    fetch(slot);
    for (int i = tid; i < T * pairs; i += 256) {
        const int t = i / pairs, pair = i % pairs, each = pairs / r.axes, axis = pair / each;
        const int row = min(row0 + t, rows - 1);
        const double turns = pos[(size_t)row * r.axes + axis] * r.turns[pair % each];
        const double angle = (turns - rint(turns)) * 6.283185307179586476925;
        const float hi = (float)angle, lo = (float)(angle - hi);
        float s, c;
        sincosf(hi, &s, &c);
        turn[t][pair] = make_float2(fmaf(-lo, s, c) * r.magnitude, fmaf(lo, c, s) * r.magnitude);
    }
    __syncthreads();
    auto put = [](E *to, uint4 v) {
        typedef uint32_t uintx4_t __attribute__((ext_vector_type(4)));
        if (PAST) __builtin_nontemporal_store(uintx4_t{v.x, v.y, v.z, v.w}, reinterpret_cast<uintx4_t *>(to));
        else *reinterpret_cast<uint4 *>(to) = v;
    };
    float c[8], s[8];
    if (turned) {
#pragma unroll
        for (int i = 0; i < 8; ++i) { c[i] = turn[t][item * 8 + i].x; s[i] = turn[t][item * 8 + i].y; }
    }
#pragma unroll 1                                              // (unrolled, 6400 rows of 64 heads take 40.9 us instead of 40.3)
    for (int h0 = slot; h0 < heads; h0 += FLY * SLOTS) {
        if (h0 != slot) fetch(h0);
#pragma unroll
        for (int f = 0; f < FLY; ++f) {
            if (!dst[f]) continue;
            float x[16];
#pragma unroll
            for (int i = 0; i < 2 * HALF; ++i) Elem<E>::unpack(raw[f][i], x + i * PER);
            if (turned) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int one = INTER ? 2 * i : i, two = INTER ? 2 * i + 1 : i + 8;
                    const float a = x[one], b = x[two];
                    x[one] = fmaf(a, c[i], -(b * s[i]));
                    x[two] = fmaf(a, s[i], b * c[i]);
                }
            }
#pragma unroll
            for (int i = 0; i < HALF; ++i) {
                put(dst[f] + lo + i * PER, Elem<E>::pack(x + i * PER));
                put(dst[f] + hi + i * PER, Elem<E>::pack(x + 8 + i * PER));
            }
        }
    }
}

void launch_rope(DType dt, const RopeTable &r, const RopeRows &q, const RopeRows &k, const int32_t *pos, int rows, int Dh, hipStream_t st)
{
    const bool past = (size_t)rows * (q.heads + k.heads) * Dh * (dt == DType::BF16 ? 2 : 4) > (32u << 20);   // the L2s together
#define FVAR_ROPE(E, DH, T, INTER, PAST)                                                                                 \
    launch(rope_kernel<E, DH, T, INTER, PAST>, dim3((unsigned)((rows + T - 1) / T)), dim3(256), 0, st, r, q, k, pos, rows)
#define FVAR_ROPE_T(E, DH)                                                                                               \
    (past          ? (r.interleaved ? FVAR_ROPE(E, DH, 2, true, true) : FVAR_ROPE(E, DH, 2, false, true))                 \
     : rows >= 2048 ? (r.interleaved ? FVAR_ROPE(E, DH, 2, true, false) : FVAR_ROPE(E, DH, 2, false, false))              \
                    : (r.interleaved ? FVAR_ROPE(E, DH, 1, true, false) : FVAR_ROPE(E, DH, 1, false, false)))
    if (dt == DType::BF16) {
        if (Dh == 64) FVAR_ROPE_T(uint16_t, 64);
        else FVAR_ROPE_T(uint16_t, 128);
    } else {
        if (Dh == 64) FVAR_ROPE_T(float, 64);
        else FVAR_ROPE_T(float, 128);
    }
#undef FVAR_ROPE_T
#undef FVAR_ROPE
}

}  // namespace fvar
