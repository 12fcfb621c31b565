// A key/value cache held in 4 bits: quantising new rows into it, and reading rows back.
//
// Format, per block of 32 consecutive head-dim elements of one token and head: a power of two 2^e stored as the byte
// e + 127, and elements in E2M1 (0, .5, 1, 1.5, 2, 3, 4, 6 and a sign), element 2i in the low half of byte i.  It is
// the block format that gfx950 converts and multiplies in hardware.  e is the smallest integer with max|x| < 7 * 2^e:
// values up to 7 * 2^e round to at most 6 * 2^e with an error of half a step of their binade, as all smaller ones do.
// It is held to [-124, 125], so that every value of the cache is 0 or a normal number of bf16 and fp32.  A block with an
// infinity or a NaN has the byte 255 and reads as NaN.
//
// Layout: codes [B][heads][capacity][DH/2], scales [B][heads][capacity][DH/32]: a head's rows are consecutive, as the
// attention streams them.
#include "common.h"

namespace fvar {

typedef __bf16 bf16x2v __attribute__((ext_vector_type(2)));

// Byte of the scale from the bits of the block's largest magnitude: exponent field less 2, one more from a mantissa of
// .75 on (1.75 * 4 = 7).  MB: mantissa bits of the type.
template <int MB> __device__ __forceinline__ uint32_t scale_byte(uint32_t top)
{
    const int e = (int)((top + (1u << (MB - 2))) >> MB) - 2;
    return top >= (255u << MB) ? 255u : (uint32_t)min(max(e, 3), 252);
}

__device__ __forceinline__ uint32_t quad_max(uint32_t v)
{
    v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0xb1, 0xf, 0xf, true));    // quad_perm 1,0,3,2
    return max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x4e, 0xf, 0xf, true)); // quad_perm 2,3,0,1
}

// Eight elements per thread, four threads per block of 32: their maximum is two steps in registers.
// grid: (chunks of a head's new rows, B * heads, K or V).  Memory-bound: rows are read as whole lines of one head, and
// written as one run per head (4 x 6400 rows, 32 heads of 128: 107 us, 5.0 TB/s; 32 x 2521, 16 heads 151 us, 5.5; two or four
// rows per thread and reads past the caches are no faster).
template <typename T, int DH>
__global__ __launch_bounds__(256) void kvq_append_kernel(const T *__restrict__ k, const T *__restrict__ v, int ld,
                                                         KvqCache c, int rows)
{
    constexpr int CH = DH / 8;                               // threads of a row
    const int item = blockIdx.x * 256 + threadIdx.x, j = item / CH, ch = item % CH;
    const int b = blockIdx.y / c.heads, h = blockIdx.y % c.heads;
    const long pos = (long)(c.lens ? c.lens[b] : c.len) + j;
    if (j >= rows || pos < 0 || pos >= c.capacity) return;   // whole rows: the threads of a block go together
    const T *src = (blockIdx.z ? v : k) + ((size_t)b * rows + j) * ld + (size_t)h * DH + ch * 8;
    uint32_t top, word = 0, byte;
    if constexpr (sizeof(T) == 2) {
        const uint4 x = *reinterpret_cast<const uint4 *>(src);
        const uint32_t w[4] = {x.x, x.y, x.z, x.w};
        uint32_t hi = 0, lo = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) { hi = max(hi, w[i] & 0x7fff0000u); lo = max(lo, w[i] & 0x7fffu); }
        top = quad_max(max(hi >> 16, lo));
        byte = scale_byte<7>(top);
        const float scale = __uint_as_float(byte << 23);
#define FVAR_PAIR(i) word = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(word, __builtin_bit_cast(bf16x2v, w[i]), scale, i)
        FVAR_PAIR(0); FVAR_PAIR(1); FVAR_PAIR(2); FVAR_PAIR(3);
#undef FVAR_PAIR
    } else {
        const float4 x = *reinterpret_cast<const float4 *>(src), y = *reinterpret_cast<const float4 *>(src + 4);
        const float f[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
        top = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(f[i]) & 0x7fffffffu);
        top = quad_max(top);
        byte = scale_byte<23>(top);
        const float scale = __uint_as_float(byte << 23);
#define FVAR_PAIR(i) word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, f[2 * i], f[2 * i + 1], scale, i)
        FVAR_PAIR(0); FVAR_PAIR(1); FVAR_PAIR(2); FVAR_PAIR(3);
#undef FVAR_PAIR
    }
    if (byte == 255) word = 0;
    const size_t row = (size_t)blockIdx.y * c.capacity + pos;
    reinterpret_cast<uint32_t *>(blockIdx.z ? c.v : c.k)[row * CH + ch] = word;
    if (ch % 4 == 0) (blockIdx.z ? c.v_scale : c.k_scale)[row * (DH / 32) + ch / 4] = (uint8_t)byte;
}

// Sixteen bytes of a row per thread, two such pieces for bf16, whose codes are fetched first.  Every value of the format is exact in
// bf16 and fp32.  Memory-bound: four fifths of the bytes are the rows written, which go past the caches where L2 would not hold
// them for their reader anyway, a lane next to the other (32 bytes a lane in two stores take 108 us for 16 x 2000 fp32 rows of 16 heads
// of 64, these 41).  32 x 2521 rows of 16 heads of 128 from cold caches: 167 us through the caches, 164 past them, 135 with two pieces per
// thread (6.2 TB/s), 139 with four.
template <typename T> constexpr int kReadPieces = sizeof(T) == 2 ? 2 : 1;

template <typename T, int DH, bool PAST>
__global__ __launch_bounds__(256) void kvq_read_kernel(KvqCache c, int first, int rows, T *__restrict__ k,
                                                       T *__restrict__ v, int only_v)
{
    typedef uint32_t uintx4_t __attribute__((ext_vector_type(4)));
    constexpr int PER = 16 / sizeof(T), CH = DH / PER, N = kReadPieces<T>;   // elements of a piece, pieces of a row
    const int b = blockIdx.y / c.heads, h = blockIdx.y % c.heads;
    const bool is_v = only_v || blockIdx.z;
    const int len = kvq_length(c, b, 0), item = blockIdx.x * (256 * N) + threadIdx.x;
    const uint8_t *codes = is_v ? c.v : c.k, *scales = is_v ? c.v_scale : c.k_scale;
    uint32_t word[N], byte[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int j = (item + 256 * i) / CH, ch = (item + 256 * i) % CH;
        const long pos = (long)(first < 0 ? len : 0) + first + j;
        word[i] = 0;
        byte[i] = 127;
        if (j < rows && pos >= 0 && pos < len) {
            const size_t row = (size_t)blockIdx.y * c.capacity + pos;
            word[i] = PER == 8 ? reinterpret_cast<const uint32_t *>(codes)[row * CH + ch]
                               : reinterpret_cast<const uint16_t *>(codes)[row * CH + ch];
            byte[i] = scales[row * (DH / 32) + ch * PER / 32];
        }
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int j = (item + 256 * i) / CH, ch = (item + 256 * i) % CH;
        if (j >= rows) return;
        const float scale = __uint_as_float(byte[i] << 23);  // 255: infinity, which the conversion turns into NaN
        uintx4_t x;
        if constexpr (PER == 8) {
            x[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word[i], scale, 0));
            x[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word[i], scale, 1));
            x[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word[i], scale, 2));
            x[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word[i], scale, 3));
        } else {
            const floatx2_t p0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word[i], scale, 0);
            const floatx2_t p1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word[i], scale, 1);
            x = uintx4_t{__float_as_uint(p0[0]), __float_as_uint(p0[1]), __float_as_uint(p1[0]), __float_as_uint(p1[1])};
        }
        uintx4_t *dst = reinterpret_cast<uintx4_t *>((is_v ? v : k) + (((size_t)b * rows + j) * c.heads + h) * DH + ch * PER);
        if (PAST) __builtin_nontemporal_store(x, dst);
        else *dst = x;
    }
}

void launch_kvq_append(DType dt, const void *k, const void *v, int ld, const KvqCache &c, int B, int rows, int Dh,
                       hipStream_t st)
{
    const dim3 grid((unsigned)(((long)rows * (Dh / 8) + 255) / 256), (unsigned)(B * c.heads), 2);
#define FVAR_APPEND(T, DH) launch(kvq_append_kernel<T, DH>, grid, dim3(256), 0, st, (const T *)k, (const T *)v, ld, c, rows)
    if (dt == DType::BF16) {
        if (Dh == 64) FVAR_APPEND(uint16_t, 64);
        else FVAR_APPEND(uint16_t, 128);
    } else {
        if (Dh == 64) FVAR_APPEND(float, 64);
        else FVAR_APPEND(float, 128);
    }
#undef FVAR_APPEND
}

void launch_kvq_read(DType dt, const KvqCache &c, int B, int first, int rows, int Dh, void *k, void *v, hipStream_t st)
{
    const int per = dt == DType::BF16 ? 8 * 256 * kReadPieces<uint16_t> : 4 * 256 * kReadPieces<float>;   // elements per workgroup
    const dim3 grid((unsigned)(((long)rows * Dh + per - 1) / per), (unsigned)(B * c.heads), k && v ? 2 : 1);
    const int only_v = !k;
    const size_t bytes = (size_t)grid.z * B * rows * c.heads * Dh * (dt == DType::BF16 ? 2 : 4);
    const bool past = bytes > (32u << 20);                   // the L2s together
#define FVAR_READ(T, DH)                                                                                                 \
    (past ? launch(kvq_read_kernel<T, DH, true>, grid, dim3(256), 0, st, c, first, rows, (T *)k, (T *)v, only_v)          \
          : launch(kvq_read_kernel<T, DH, false>, grid, dim3(256), 0, st, c, first, rows, (T *)k, (T *)v, only_v))
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
