// Eviction of cached rows by the attention weight they have collected: per layer, utterance and K/V head the first n_first rows, the last
// n_recent and, of those between, the ones of the largest weight are copied to another cache in their order.  Rotated keys carry their
// position, and attention does not ask for the order of its rows, so each head may keep rows of its own.
#include "device_utils.h"
#include "tree.h"

namespace ssd {

// Whole numbers in the order of the weights: 0 for NaN, which goes first; both zeros alike.
__device__ __forceinline__ uint32_t ordered(float v) {
    if (v != v) return 0;
    const uint32_t u = __float_as_uint(v + 0.f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

constexpr int SEL_THREADS = 1024;

// Sums of a value over the threads before this one and over all of them.
__device__ __forceinline__ int2 scan(int v, int* waves) {
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    int s = v;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int o = __shfl_up(s, d);
        if (lane >= d) s += o;
    }
    __syncthreads();
    if (lane == 63) waves[wave] = s;
    __syncthreads();
    int before = 0, all = 0;
    for (int w = 0; w < SEL_THREADS / 64; ++w) {
        if (w < wave) before += waves[w];
        all += waves[w];
    }
    return make_int2(before + s - v, all);
}

// One workgroup a (layer, head, utterance): the need-th largest weight bit by bit, then the kept rows in order.
__global__ void __launch_bounds__(SEL_THREADS) evict_select_kernel(EvictArgs a) {
    __shared__ int waves[SEL_THREADS / 64];
    const EvictUtt u = a.utts[blockIdx.x];
    const int64_t lh = blockIdx.y;                           // layer * heads + head
    const float* w = a.mass + lh * a.mass_slots + u.slot0;
    int32_t* rows = a.rows + lh * a.n_kept + u.kept0;
    const int tid = threadIdx.x;
    const bool all = u.keep >= u.n_ctx;
    const int lo = all ? u.n_ctx : a.n_first, hi = all ? u.n_ctx : u.n_ctx - a.n_recent;
    const int need = all ? 0 : u.keep - a.n_first - a.n_recent;
    uint32_t t = 0;                                          // largest value that at least `need` weights reach
    if (need > 0)
        for (int bit = 31; bit >= 0; --bit) {
            const uint32_t c = t | 1u << bit;
            int n = 0;
            for (int i = lo + tid; i < hi; i += SEL_THREADS) n += ordered(w[i]) >= c;
            if (scan(n, waves).y >= need) t = c;
        }
    int n_above = 0;
    if (need > 0) {
        for (int i = lo + tid; i < hi; i += SEL_THREADS) n_above += ordered(w[i]) > t;
        n_above = scan(n_above, waves).y;
    }
    int ties = need - n_above, out = 0;
    for (int i0 = 0; i0 < u.n_ctx; i0 += SEL_THREADS) {
        const int i = i0 + tid;
        const bool between = i >= lo && i < hi;
        const uint32_t o = between ? ordered(w[i]) : 0;
        const int tie = need > 0 && between && o == t;
        const int2 tr = scan(tie, waves);
        const int keep = i < u.n_ctx && (!between || (need > 0 && (o > t || (tie && tr.x < ties))));
        ties -= tr.y;
        const int2 kr = scan(keep, waves);
        if (keep) rows[out + kr.x] = i;
        out += kr.y;
    }
}

// Row `blockIdx.x` of the kept ones, all layers and heads.
__global__ void __launch_bounds__(256) evict_copy_kernel(EvictArgs a) {
    const int r = blockIdx.x;
    int b = 0;
    while (b + 1 < a.B && r >= a.utts[b + 1].kept0) ++b;
    const EvictUtt u = a.utts[b];
    const int64_t dst = u.out0 + (r - u.kept0);
    const int per = a.row_chunks, n = a.n_kv_heads * per;
    const int layer = blockIdx.y;
    for (int i = threadIdx.x; i < n; i += 256) {
        const int h = i / per, c = i % per;
        const int64_t lh = (int64_t)layer * a.n_kv_heads + h;
        const int64_t src = u.slot0 + a.rows[lh * a.n_kept + r];
        const int64_t s = layer * a.layer_stride + h * a.head_stride + src * a.slot_stride + c;
        const int64_t d = layer * a.out_layer_stride + h * a.out_head_stride + dst * a.out_slot_stride + c;
        ((uint4*)a.k_out)[d] = ((const uint4*)a.k)[s];
        ((uint4*)a.v_out)[d] = ((const uint4*)a.v)[s];
        if (a.mass_out && c == 0) a.mass_out[lh * a.mass_out_slots + dst] = a.mass[lh * a.mass_slots + src];
    }
}

void launch_kv_evict(const EvictArgs& a, hipStream_t st) {
    hipLaunchKernelGGL(evict_select_kernel, dim3(a.B, a.n_layers * a.n_kv_heads), dim3(SEL_THREADS), 0, st, a);
    hipLaunchKernelGGL(evict_copy_kernel, dim3(a.n_kept, a.n_layers), dim3(256), 0, st, a);
}

}  // namespace ssd
