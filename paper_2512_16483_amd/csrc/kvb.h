// The elements of the 8-bit cache (format: kvb.hip) on the GPU.
#pragma once
#include "common.h"

namespace fvar {

typedef __bf16 bf16x2v_t __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2v_t __attribute__((ext_vector_type(2)));

// rows of sample b, `extra` more than the cache says, within its capacity
__device__ __forceinline__ int kvb_length(const KvbCache &c, int b, int extra)
{
    const long l = (long)(c.lens ? c.lens[b] : c.len) + extra;
    return (int)(l < 0 ? 0 : l > c.capacity ? c.capacity : l);
}

// Byte of the scale from the fp32 bits of the largest finite magnitude: its exponent less 8, one more from mantissas above that of 464
// (1.8125 * 2^8); e within [-117, 119].
__device__ __forceinline__ uint32_t kvb_byte(uint32_t top)
{
    const int e = (int)((top + 0x17ffffu) >> 23) - 8;
    return (uint32_t)min(max(e, 10), 246);
}
__device__ __forceinline__ uint32_t kvb_finite(uint32_t magnitude) { return magnitude < 0x7f800000u ? magnitude : 0; }

// the largest of 64 lanes' numbers, in each of them
__device__ __forceinline__ uint32_t kvb_wave_max(uint32_t v)
{
    v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0xb1, 0xf, 0xf, true));            // quad_perm 1,0,3,2
    v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x4e, 0xf, 0xf, true));            // quad_perm 2,3,0,1
    v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x141, 0xf, 0xf, true));           // row_half_mirror
    v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x140, 0xf, 0xf, true));           // row_mirror
    const auto a = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    v = max(a[0], a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return max(b[0], b[1]);
}

// Codes of four numbers, which have to be within 464 * size; values of a word's lower (W = 0) or upper two codes.
__device__ __forceinline__ uint32_t kvb_four(const float *x, float size)
{
    typedef short shortx2_t __attribute__((ext_vector_type(2)));
    shortx2_t w = {0, 0};
    w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, x[0], x[1], size, false);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, x[2], x[3], size, true);
    return __builtin_bit_cast(uint32_t, w);
}
template <int W> __device__ __forceinline__ uint32_t kvb_bf16(uint32_t word, float size)
{
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(word, size, W != 0));
}
template <int W> __device__ __forceinline__ uint32_t kvb_f16(uint32_t word, float size)
{
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(word, size, W != 0));
}
// Four codes that stand for their values times `from`, rounded to ones that stand for them times `to`, which hold them.  (What
// is not a number stays so.)
__device__ __forceinline__ uint32_t kvb_again(uint32_t word, float from, float to)
{
    const floatx2_t a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(word, from, false), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(word, from, true);
    const float x[4] = {a[0], a[1], b[0], b[1]};
    return kvb_four(x, to);
}

}  // namespace fvar
