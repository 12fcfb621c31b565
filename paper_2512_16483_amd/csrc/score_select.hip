// Representative-token scoring and selection (paper, Sec. "Representative Token Restoration").
//
//   score   s_i = fl32(sum_j x_ij^2): one wavefront per token row, 16-byte loads, products and
//           the sum carried in fp64 (exact products; the order of the adds then changes the
//           stored fp32 value only in double-rounding corner cases), butterfly reduction.
//   select  one workgroup per sample: histograms over the order-preserving integer image of the
//           scores yield the k-th largest key T and how many keys equal to T are still needed;
//           then an ordered sweep over the indices with prefix sums writes the kept and the
//           pruned indices, each ascending.  Ties at T go to the lower index.  No atomics touch
//           the outputs, so the result is deterministic.
#include "select.h"

namespace fvar {

template <typename T>
__global__ __launch_bounds__(256) void scores_kernel(const T *__restrict__ x, int rows, int d,
                                                     float *__restrict__ scores)
{
    constexpr int E = Elem<T>::kPerChunk;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int row = blockIdx.x * 4 + wave;
    if (row >= rows) return;
    const uint4 *src = reinterpret_cast<const uint4 *>(x + (size_t)row * d);
    const int nchunk = d / E;
    double acc0 = 0.0, acc1 = 0.0;
    int c = lane;
    // four chunks in flight per lane
    for (; c + 192 < nchunk; c += 256) {
        uint4 v0 = src[c], v1 = src[c + 64], v2 = src[c + 128], v3 = src[c + 192];
        float f[E];
        Elem<T>::unpack(v0, f);
#pragma unroll
        for (int e = 0; e < E; ++e) acc0 = fma((double)f[e], (double)f[e], acc0);
        Elem<T>::unpack(v1, f);
#pragma unroll
        for (int e = 0; e < E; ++e) acc1 = fma((double)f[e], (double)f[e], acc1);
        Elem<T>::unpack(v2, f);
#pragma unroll
        for (int e = 0; e < E; ++e) acc0 = fma((double)f[e], (double)f[e], acc0);
        Elem<T>::unpack(v3, f);
#pragma unroll
        for (int e = 0; e < E; ++e) acc1 = fma((double)f[e], (double)f[e], acc1);
    }
    for (; c < nchunk; c += 64) {
        uint4 v0 = src[c];
        float f[E];
        Elem<T>::unpack(v0, f);
#pragma unroll
        for (int e = 0; e < E; ++e) acc0 = fma((double)f[e], (double)f[e], acc0);
    }
    double acc = wave_sum(acc0 + acc1);
    if (lane == 0) scores[row] = (float)acc;
}

void launch_scores(DType dt, const void *x, int rows, int d, float *scores, hipStream_t st)
{
    dim3 grid((rows + 3) / 4), block(256);
    if (dt == DType::BF16)
        launch(scores_kernel<uint16_t>, grid, block, 0, st, (const uint16_t *)x, rows, d,
                           scores);
    else
        launch(scores_kernel<float>, grid, block, 0, st, (const float *)x, rows, d,
                           scores);
}

constexpr int kSelKeysMax = 12;              // keys per thread that stay in registers

template <int KPT>
__global__ __launch_bounds__(kSelThreads) void select_kernel(const float *__restrict__ scores, int M,
                                                             int k, int32_t *__restrict__ idx_keep,
                                                             int32_t *__restrict__ idx_drop)
{
    __shared__ SelectLds<KPT> sh;
    const int b = blockIdx.x, tid = threadIdx.x;
    const float *s = scores + (size_t)b * M;

    uint32_t key[KPT], lo = 0xffffffffu, hi = 0u;
#pragma unroll
    for (int j = 0; j < KPT; ++j) {
        const int i = j * kSelThreads + tid;
        key[j] = score_key(s[min(i, M - 1)]);            // a copy of the last key does not move the range
        lo = min(lo, key[j]);
        hi = max(hi, key[j]);
    }
    uint32_t T;
    int need_eq;
    select_threshold<KPT>(key, M, k, lo, hi, sh, T, need_eq);
    int32_t *keep_out = idx_keep + (size_t)b * k;
    int32_t *drop_out = idx_drop ? idx_drop + (size_t)b * (M - k) : nullptr;
    select_sweep<KPT>(key, M, T, need_eq, sh, [&](int i, bool keep, int keep_pos) {
        if (keep) keep_out[keep_pos] = i;
        else if (drop_out) drop_out[i - keep_pos] = i;
    });
}

__global__ __launch_bounds__(kSelThreads) void select_large_kernel(const float *__restrict__ scores, int M,
                                                                   int k, int32_t *__restrict__ idx_keep,
                                                                   int32_t *__restrict__ idx_drop)
{
    __shared__ SelectStreamLds sh;
    const int b = blockIdx.x;
    const float *s = scores + (size_t)b * M;
    int32_t *keep_out = idx_keep + (size_t)b * k;
    int32_t *drop_out = idx_drop ? idx_drop + (size_t)b * (M - k) : nullptr;
    select_streamed([&](int i) { return score_key(s[i]); }, M, k, sh, [&](int i, bool keep, int keep_pos) {
        if (keep) keep_out[keep_pos] = i;
        else if (drop_out) drop_out[i - keep_pos] = i;
    });
}

void launch_select(const float *scores, int B, int M, int k, int32_t *idx_keep, int32_t *idx_drop,
                   hipStream_t st)
{
    const dim3 grid(B), block(kSelThreads);
    const int kpt = (M + kSelThreads - 1) / kSelThreads;
#define FVAR_SELECT(KPT) launch(select_kernel<KPT>, grid, block, 0, st, scores, M, k, idx_keep, idx_drop)
    if (kpt <= 1) FVAR_SELECT(1);
    else if (kpt <= 2) FVAR_SELECT(2);
    else if (kpt <= 4) FVAR_SELECT(4);
    else if (kpt <= 8) FVAR_SELECT(8);
    else if (kpt <= kSelKeysMax) FVAR_SELECT(kSelKeysMax);
    else launch(select_large_kernel, grid, block, 0, st, scores, M, k, idx_keep, idx_drop);
#undef FVAR_SELECT
}

}  // namespace fvar
