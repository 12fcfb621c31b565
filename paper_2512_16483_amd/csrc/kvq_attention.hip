// Attention over a key/value cache held in 4 bits (format and layout: kvq.hip).
//   o[b,i,h,:] = sum_t p_t V[b,t,h',:],  p = softmax over the visible t of scale * q[b,i,h,:] . K[b,t,h',:],
//   h' = h / (H / heads); t is visible when t < length of sample b and mask[b][t] != 0; o = 0 where nothing is visible.
#include "common.h"

namespace fvar {

// One wavefront per query and head, a lane per key for the scores, a lane per one or two head-dim elements for the sum
// over the values; running maximum and sum in fp32.
template <typename T, int DH>
__global__ __launch_bounds__(64) void kvq_attn_kernel(const T *__restrict__ q, int ld, KvqCache c, int extra, int n, int H,
                                                      float c_log2, T *__restrict__ o)
{
    constexpr int NB = DH / 32, DV = DH / 64;
    __shared__ float qs[DH];
    const int lane = threadIdx.x;
    const int h = blockIdx.x % H;
    const long bi = blockIdx.x / H;
    const int b = (int)(bi / n), hk = h / (H / c.heads);
    const T *src = q + (size_t)bi * ld + (size_t)h * DH;
#pragma unroll
    for (int e = 0; e < DV; ++e) qs[lane * DV + e] = Elem<T>::load(src + lane * DV + e);
    __syncthreads();
    const int len = kvq_length(c, b, extra);
    const size_t head = ((size_t)b * c.heads + hk) * c.capacity;
    const uint4 *Kc = reinterpret_cast<const uint4 *>(c.k) + head * NB;
    const uint8_t *Ks = c.k_scale + head * NB, *Vs = c.v_scale + head * NB, *Vc = c.v + head * (DH / 2);
    float m = -INFINITY, l = 0.f, acc[DV] = {};
    for (int t0 = 0; t0 < len; t0 += 64) {
        const int t = t0 + lane;
        const bool seen = t < len && (!c.mask || c.mask[(size_t)b * c.capacity + t]);
        float s = -INFINITY;
        if (seen) {
            s = 0.f;
#pragma unroll
            for (int k = 0; k < NB; ++k) {
                const uint4 x = Kc[(size_t)t * NB + k];
                const float scale = __uint_as_float((uint32_t)Ks[(size_t)t * NB + k] << 23);
                const uint32_t w[4] = {x.x, x.y, x.z, x.w};
                float part = 0.f;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const floatx2_t p0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[i], scale, 0);
                    const floatx2_t p1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[i], scale, 1);
                    const floatx2_t p2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[i], scale, 2);
                    const floatx2_t p3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[i], scale, 3);
                    const float *qk = qs + 32 * k + 8 * i;
                    part = fmaf(p0[0], qk[0], part); part = fmaf(p0[1], qk[1], part);
                    part = fmaf(p1[0], qk[2], part); part = fmaf(p1[1], qk[3], part);
                    part = fmaf(p2[0], qk[4], part); part = fmaf(p2[1], qk[5], part);
                    part = fmaf(p3[0], qk[6], part); part = fmaf(p3[1], qk[7], part);
                }
                s += part;
            }
        }
        float mx = fmaxf(m, s);
#pragma unroll
        for (int d = 32; d > 0; d >>= 1) mx = fmaxf(mx, __shfl_xor(mx, d));
        const float base = fmaxf(mx, -1e30f);                // nothing finite yet: weights of 0
        const float alpha = __builtin_amdgcn_exp2f((m - base) * c_log2);
        const float p = __builtin_amdgcn_exp2f((s - base) * c_log2);
        m = mx;
        l = l * alpha + wave_sum(p);
#pragma unroll
        for (int e = 0; e < DV; ++e) acc[e] *= alpha;
        unsigned long long vis = __ballot(seen);
        while (vis) {
            const int kk = __builtin_ctzll(vis);
            vis &= vis - 1;
            const float w = __shfl(p, kk);
            const int d0 = lane * DV;
            const float scale = __uint_as_float((uint32_t)Vs[(size_t)(t0 + kk) * NB + d0 / 32] << 23);
            const floatx2_t x = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(Vc[(size_t)(t0 + kk) * (DH / 2) + d0 / 2], scale, 0);
            if constexpr (DV == 2) {
                acc[0] = fmaf(w, x[0], acc[0]);
                acc[1] = fmaf(w, x[1], acc[1]);
            } else {
                acc[0] = fmaf(w, lane & 1 ? x[1] : x[0], acc[0]);
            }
        }
    }
    T *dst = o + (size_t)bi * H * DH + (size_t)h * DH + lane * DV;
#pragma unroll
    for (int e = 0; e < DV; ++e) Elem<T>::store(dst + e, l == 0.f ? 0.f : acc[e] / l);
}

size_t kvq_attention_scratch_floats(DType, int, int, int, int, int, int) { return 0; }

void launch_kvq_attention(DType dt, const void *q, int ld, const KvqCache &c, int extra, int B, int n, int H, int Dh,
                          float scale, void *o, float *, hipStream_t st)
{
    const dim3 grid((unsigned)((long)B * n * H));
    const float c_log2 = scale * 1.4426950408889634f;
#define FVAR_KVQ(T, DH) \
    launch(kvq_attn_kernel<T, DH>, grid, dim3(64), 0, st, (const T *)q, ld, c, extra, n, H, c_log2, (T *)o)
    if (dt == DType::BF16) {
        if (Dh == 64) FVAR_KVQ(uint16_t, 64);
        else FVAR_KVQ(uint16_t, 128);
    } else {
        if (Dh == 64) FVAR_KVQ(float, 64);
        else FVAR_KVQ(float, 128);
    }
#undef FVAR_KVQ
}

}  // namespace fvar
