// A key/value cache held in 8 bits: writing new rows into it, and reading rows back.
//
// Format: elements in E4M3 (sign, 4 bits of exponent, 3 of mantissa, up to 448; 127 is NaN), which share a power of two 2^e, stored as the
// byte e + 127, over a block of 32 consecutive rows of one head.  e is the smallest integer within [-117, 119] with max|x| <= 464 * 2^e over the
// finite elements of the block: up to 464, rounding to 448 is off by no more than half a step.  Within those bounds every value is 0 or a normal
// number of bf16 and fp32, so reading back is exact.  An element that is not finite is NaN, and does not count for e.
//
// Layout: codes [B][heads][capacity][DH], scales [B][heads][ceil(capacity / 32)]: a head's rows are consecutive, as the attention streams
// them, and a tile of 32 keys has one scale, which is the same for a whole wavefront.
#include "kvb.h"

namespace fvar {

// One block of one head's keys or values per workgroup: eight threads per row, Dh / 8 elements each, eight of which lie together.  The new rows'
// largest element and the scale of the rows that the block holds give its scale; where that rises, the rows that it holds are rounded to it.
// grid: (blocks that the rows can touch, B * heads, K or V).  Memory-bound: 4 x 6400 rows of 32 heads of 128 behind 10521 take 105 us (6.0 TB/s; codes
// past the caches 112); a row each of 32 samples 3 us, its launch.
template <typename T, int DH>
__global__ __launch_bounds__(256) void kvb_append_kernel(const T *__restrict__ k, const T *__restrict__ v, int ld, KvbCache c, int rows)
{
    constexpr int N = DH / 64;                               // groups of eight elements of a thread, 64 apart
    __shared__ uint32_t tops[4];
    const int tid = threadIdx.x, r = tid >> 3, at = (tid & 7) * 8;
    const int b = blockIdx.y / c.heads, h = blockIdx.y % c.heads;
    const long len = c.lens ? c.lens[b] : c.len;
    const long first = max(len, 0l), block = first / kKvbBlock + blockIdx.x, pos = block * kKvbBlock + r, j = pos - len;
    if (block * kKvbBlock >= min(len + rows, (long)c.capacity)) return;
    const bool fresh = pos >= first && j < rows && pos < c.capacity, held = pos < first && pos < c.capacity;
    uint8_t *scales = (blockIdx.z ? c.v_scale : c.k_scale) + (size_t)blockIdx.y * c.blocks();
    uint8_t *codes = (blockIdx.z ? c.v : c.k) + ((size_t)blockIdx.y * c.capacity + pos) * DH + at;
    const bool holds = block * kKvbBlock < first;            // rows of the block are held already
    const uint32_t before = holds ? scales[block] : 0;

    float x[N][8];
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) x[i][e] = 0.f;
    if (fresh) {
        const T *src = (blockIdx.z ? v : k) + ((size_t)b * rows + j) * ld + (size_t)h * DH + at;
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (int e = 0; e < 8; e += Elem<T>::kPerChunk)
                Elem<T>::unpack(*reinterpret_cast<const uint4 *>(src + 64 * i + e), x[i] + e);
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(x[i][e]) & 0x7fffffffu);
    }
    const bool odd = top >= 0x7f800000u;                     // an element that is not finite
    if (__builtin_expect(odd, 0)) {
        top = 0;
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) top = max(top, kvb_finite(__float_as_uint(x[i][e]) & 0x7fffffffu));
    }
    top = kvb_wave_max(top);
    if ((tid & 63) == 0) tops[tid >> 6] = top;
    __syncthreads();
    top = max(max(tops[0], tops[1]), max(tops[2], tops[3]));
    const uint32_t byte = max(kvb_byte(top), before);
    if (tid == 0 && byte != before) scales[block] = (uint8_t)byte;
    const float size = __uint_as_float(byte << 23);
    if (held && byte != before) {
        const float old = __uint_as_float(before << 23);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            uint2 w = *reinterpret_cast<const uint2 *>(codes + 64 * i);
            w.x = kvb_again(w.x, old, size);
            w.y = kvb_again(w.y, old, size);
            *reinterpret_cast<uint2 *>(codes + 64 * i) = w;
        }
    }
    if (!fresh) return;
    const float most = 448.f * size;                         // (beyond it only up to 464, and where e is at its bound)
#pragma unroll
    for (int i = 0; i < N; ++i) {
        uint32_t w[2] = {0, 0};
#pragma unroll
        for (int e = 0; e < 8; ++e) x[i][e] = __builtin_amdgcn_fmed3f(x[i][e], -most, most);
#pragma unroll
        for (int p = 0; p < 2; ++p) w[p] = kvb_four(x[i] + 4 * p, size);
        if (__builtin_expect(odd, 0)) {
            const T *src = (blockIdx.z ? v : k) + ((size_t)b * rows + j) * ld + (size_t)h * DH + at + 64 * i;
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if ((__float_as_uint(Elem<T>::load(src + e)) & 0x7fffffffu) >= 0x7f800000u)
                    w[e >> 2] = (w[e >> 2] & ~(255u << (8 * (e & 3)))) | 127u << (8 * (e & 3));
        }
        *reinterpret_cast<uint2 *>(codes + 64 * i) = make_uint2(w[0], w[1]);
    }
}

// Sixteen bytes of a row per thread and piece, two of them, whose codes are fetched first.  Memory-bound; rows go past the caches where L2 would
// not hold them for their reader anyway.  4 x 6400 rows of 32 heads of 128: one piece 118 us, two 108 (5.8 TB/s), four 110; fp32, 16 x 2000
// rows of 16 heads of 64: one 57, two 53.
constexpr int kKvbReadPieces = 2;

template <typename T, int DH, bool PAST>
__global__ __launch_bounds__(256) void kvb_read_kernel(KvbCache c, int first, int rows, T *__restrict__ k, T *__restrict__ v, int only_v)
{
    typedef uint32_t uintx4_t __attribute__((ext_vector_type(4)));
    constexpr int PER = 16 / sizeof(T), CH = DH / PER, N = kKvbReadPieces;   // elements of a piece, pieces of a row
    const int b = blockIdx.y / c.heads, h = blockIdx.y % c.heads;
    const bool is_v = only_v || blockIdx.z;
    const int len = kvb_length(c, b, 0), item = blockIdx.x * (256 * N) + threadIdx.x;
    const uint8_t *codes = is_v ? c.v : c.k, *scales = (is_v ? c.v_scale : c.k_scale) + (size_t)blockIdx.y * c.blocks();
    uint2 word[N];
    uint32_t byte[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int j = (item + 256 * i) / CH, ch = (item + 256 * i) % CH;
        const long pos = (long)(first < 0 ? len : 0) + first + j;
        word[i] = make_uint2(0, 0);
        byte[i] = 127;
        if (j < rows && pos >= 0 && pos < len) {
            const uint8_t *src = codes + ((size_t)blockIdx.y * c.capacity + pos) * DH + ch * PER;
            if constexpr (PER == 8) word[i] = *reinterpret_cast<const uint2 *>(src);
            else word[i].x = *reinterpret_cast<const uint32_t *>(src);
            byte[i] = scales[pos / kKvbBlock];
        }
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int j = (item + 256 * i) / CH, ch = (item + 256 * i) % CH;
        if (j >= rows) return;
        const float size = __uint_as_float(byte[i] << 23);
        uintx4_t x;
        if constexpr (PER == 8) {
            x[0] = kvb_bf16<0>(word[i].x, size);
            x[1] = kvb_bf16<1>(word[i].x, size);
            x[2] = kvb_bf16<0>(word[i].y, size);
            x[3] = kvb_bf16<1>(word[i].y, size);
        } else {
            const floatx2_t p0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(word[i].x, size, false);
            const floatx2_t p1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(word[i].x, size, true);
            x = uintx4_t{__float_as_uint(p0[0]), __float_as_uint(p0[1]), __float_as_uint(p1[0]), __float_as_uint(p1[1])};
        }
        uintx4_t *dst = reinterpret_cast<uintx4_t *>((is_v ? v : k) + (((size_t)b * rows + j) * c.heads + h) * DH + ch * PER);
        if (PAST) __builtin_nontemporal_store(x, dst);
        else *dst = x;
    }
}

void launch_kvb_append(DType dt, const void *k, const void *v, int ld, const KvbCache &c, int B, int rows, int Dh, hipStream_t st)
{
    // rows of unknown beginnings touch at most as many blocks as those that begin with the last row of one
    const long before = c.lens ? kKvbBlock - 1 : c.len % kKvbBlock;
    const dim3 grid((unsigned)((before + rows + kKvbBlock - 1) / kKvbBlock), (unsigned)(B * c.heads), 2);
#define FVAR_APPEND(T, DH) launch(kvb_append_kernel<T, DH>, grid, dim3(256), 0, st, (const T *)k, (const T *)v, ld, c, rows)
    if (dt == DType::BF16) {
        if (Dh == 64) FVAR_APPEND(uint16_t, 64);
        else FVAR_APPEND(uint16_t, 128);
    } else {
        if (Dh == 64) FVAR_APPEND(float, 64);
        else FVAR_APPEND(float, 128);
    }
#undef FVAR_APPEND
}

void launch_kvb_read(DType dt, const KvbCache &c, int B, int first, int rows, int Dh, void *k, void *v, hipStream_t st)
{
    const int per = dt == DType::BF16 ? 8 * 256 * kKvbReadPieces : 4 * 256 * kKvbReadPieces;   // elements per workgroup
    const dim3 grid((unsigned)(((long)rows * Dh + per - 1) / per), (unsigned)(B * c.heads), k && v ? 2 : 1);
    const int only_v = !k;
    const size_t bytes = (size_t)grid.z * B * rows * c.heads * Dh * (dt == DType::BF16 ? 2 : 4);
    const bool past = bytes > (32u << 20);                   // the L2s together
#define FVAR_READ(T, DH)                                                                                                 \
    (past ? launch(kvb_read_kernel<T, DH, true>, grid, dim3(256), 0, st, c, first, rows, (T *)k, (T *)v, only_v)          \
          : launch(kvb_read_kernel<T, DH, false>, grid, dim3(256), 0, st, c, first, rows, (T *)k, (T *)v, only_v))
    if (dt == DType::BF16) {
        if (Dh == 64) FVAR_READ(uint16_t, 64);
        else FVAR_READ(uint16_t, 128);
    } else {
        if (Dh == 64) FVAR_READ(float, 64);
        else FVAR_READ(float, 128);
    }
#undef FVAR_READ
}

}  // namespace fvar
