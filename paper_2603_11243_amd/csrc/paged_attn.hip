// Attention of the newest tokens over the pages of their utterances:
//   s_j = scale q . k_j,  lse = log sum_j exp s_j,  o = sum_j exp(s_j - lse) v_j   over the rows j that the token sees.
#include "pages.h"
#include "tree_attn.h"

namespace ssd {

namespace {

// Element i of row `row` of pages.
template <int PT>
__device__ __forceinline__ float element(const void* p, const float* scales, int64_t row, int hd, int i) {
    const int64_t at = row * hd + i;
    if constexpr (PT == SSD_E4M3) return __builtin_amdgcn_cvt_f32_fp8(((const uint8_t*)p)[at], 0) * scales[row];
    else if constexpr (PT == SSD_I8) return (float)((const int8_t*)p)[at] * scales[row];
    else return Elem<PT>::get(((const typename Elem<PT>::type*)p)[at]);
}

// A workgroup has one query row; chunks of 256 keys, a running maximum and sum.
template <int QT, int PT>
__global__ void __launch_bounds__(256) paged_row_kernel(PagedAttnArgs a) {
    __shared__ float q_s[128], p_s[256], red[4];
    __shared__ int64_t row_s[256];
    typedef Elem<QT> E;
    const int h = blockIdx.x, t = blockIdx.y, b = blockIdx.z, hd = a.p.head_dim, tid = threadIdx.x, kvh = h / a.group;
    const int64_t token = (int64_t)b * a.n_new + t;
    bool bad = false;
    int n = a.p.ctx_len[b];
    if (n < 0 || n > a.p.max_ctx) {
        bad = true;
        n = n < 0 ? 0 : a.p.max_ctx;
    }
    n -= a.n_new - 1 - t;
    if (tid < hd) q_s[tid] = E::get(((const typename E::type*)a.q)[token * a.q_stride + h * hd + tid]);
    float m = -F32_MOST, l = 0.f, o = 0.f;
    const float sc = a.scale * LOG2E;
    for (int k0 = 0; k0 < n; k0 += 256) {
        __syncthreads();
        const int j = k0 + tid;
        const int page = j < n ? page_of(a.p, b, j) : -1;
        bad |= j < n && page < 0;
        float s = -INFINITY;
        const int64_t row = page < 0 ? -1 : row_in_pages(a.p, page, kvh, j);
        if (page >= 0) {
            s = 0.f;
            for (int i = 0; i < hd; ++i) s = fmaf(q_s[i], element<PT>(a.p.k, a.p.k_scale, row, hd, i), s);
            s *= sc;
        }
        float top = group_allreduce<64>(s, OpMax());
        if (tid % 64 == 0) red[tid / 64] = top;
        __syncthreads();
        top = fmaxf(m, fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3])));
        const float alpha = __builtin_amdgcn_exp2f(m - top), w = __builtin_amdgcn_exp2f(s - top);
        m = top;
        p_s[tid] = w * 0x1p-32f;                             // (sums of up to 2^30 values at the end of fp32's range stay inside)
        row_s[tid] = row;
        l = l * alpha + w;
        o *= alpha;
        __syncthreads();
        if (tid < hd)
            for (int i = 0; i < min(256, n - k0); ++i)
                if (row_s[i] >= 0) o = fmaf(p_s[i], element<PT>(a.p.v, a.p.v_scale, row_s[i], hd, tid), o);
    }
    __syncthreads();
    l = group_allreduce<64>(l, OpSum());
    if (tid % 64 == 0) red[tid / 64] = l;
    __syncthreads();
    l = red[0] + red[1] + red[2] + red[3];
    if (tid < hd) ((typename E::type*)a.out)[(token * a.n_q_heads + h) * hd + tid] = E::put(l == 0.f ? 0.f : o / l * 0x1p32f);
    if (a.lse && tid == 0) a.lse[token * a.n_q_heads + h] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * LN2;
    if (bad) raise_flag(a.p.flags, SSD_FLAG_BAD_PAGE);
}

template <int QT, int PT>
void launch_rows(const PagedAttnArgs& a, hipStream_t st) {
    paged_row_kernel<QT, PT><<<dim3(a.n_q_heads, a.n_new, a.p.B), 256, 0, st>>>(a);
}
template <int QT>
void launch_type(const PagedAttnArgs& a, int pages_dtype, hipStream_t st) {
    if (pages_dtype == SSD_E4M3) launch_rows<QT, SSD_E4M3>(a, st);
    else if (pages_dtype == SSD_I8) launch_rows<QT, SSD_I8>(a, st);
    else launch_rows<QT, QT>(a, st);
}

}  // namespace

void launch_paged_attention(const PagedAttnArgs& a, int q_dtype, int pages_dtype, hipStream_t st) {
    if (q_dtype == SSD_F32) launch_type<SSD_F32>(a, pages_dtype, st);
    else if (q_dtype == SSD_BF16) launch_type<SSD_BF16>(a, pages_dtype, st);
    else launch_type<SSD_F16>(a, pages_dtype, st);
}

}  // namespace ssd
