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

// Selection: one workgroup of THREADS a (layer, head, utterance), whose weights stay in registers, V a thread, thread t those of rows t V .. t V + V - 1 of each
// CHUNK = THREADS V rows (more than CHUNK rows: read again for every step).  The need-th largest is found digit by digit, 11, 11 and 10 bits from
// the top: a histogram in LDS of the rows that agree with the digits found, of the bins the one in which the count from above reaches `need`.  Then the
// kept rows in order: a thread's rows are consecutive, so that one scan over the threads places them.
constexpr int BINS = 2048;

// Sums of v over the threads before this one, and over all.
template <int THREADS>
__device__ __forceinline__ int2 scan(int v, int* waves) {
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    int s = v;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int o = __shfl_up(s, d);
        if (lane >= d) s += o;
    }
    if constexpr (THREADS == 64) return make_int2(s - v, __shfl(s, 63));
    __syncthreads();
    if (lane == 63) waves[wave] = s;
    __syncthreads();
    int before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) {
        if (w < wave) before += waves[w];
        all += waves[w];
    }
    return make_int2(before + s - v, all);
}

template <int THREADS, int V, bool MORE>
__global__ void __launch_bounds__(THREADS) evict_select_kernel(EvictArgs a) {
    constexpr int CHUNK = THREADS * V, PER = BINS / THREADS;
    __shared__ int hist[BINS];
    __shared__ int waves[THREADS / 64];
    __shared__ int found[2];                                 // digit, rows above it
    const EvictUtt u = a.utts[blockIdx.x];
    const int64_t lh = blockIdx.y;                           // layer * heads + head
    const float* w = a.mass + lh * a.mass_slots + u.slot0;
    int32_t* rows = a.rows + lh * a.n_kept + u.kept0;
    const int tid = threadIdx.x;
    if (u.keep >= u.n_ctx) {
        for (int i = tid; i < u.n_ctx; i += THREADS) rows[i] = i;
        return;
    }
    const int lo = a.n_first, hi = u.n_ctx - a.n_recent;     // rows between, of which `need` stay
    int need = u.keep - a.n_first - a.n_recent;
    uint32_t x[V];
    auto load = [&](int c0) __attribute__((always_inline)) {
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const int i = c0 + tid * V + e;
            x[e] = ordered(w[min(i, u.n_ctx - 1)]);
        }
    };
    load(0);
    uint32_t t = 0, mask = 0;                                // digits found, and which bits they are
    if (need > 0) {
#pragma unroll
        for (int round = 0; round < 3; ++round) {
            const int shift = round == 0 ? 21 : round == 1 ? 10 : 0, bits = round == 2 ? 10 : 11;
            for (int i = tid; i < BINS; i += THREADS) hist[i] = 0;
            __syncthreads();
            for (int c0 = 0; c0 < u.n_ctx; c0 += CHUNK) {
                if (MORE && (round || c0)) load(c0);
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const int i = c0 + tid * V + e;
                    if (i >= lo && i < hi && ((x[e] ^ t) & mask) == 0) atomicAdd(&hist[x[e] >> shift & ((1u << bits) - 1)], 1);
                }
                if (!MORE) break;
            }
            __syncthreads();
            // bins from the top: thread t has bins BINS - 1 - t PER - e
            int mine[PER], sum = 0;
#pragma unroll
            for (int e = 0; e < PER; ++e) sum += mine[e] = hist[BINS - 1 - tid * PER - e];
            int above = scan<THREADS>(sum, waves).x;
#pragma unroll
            for (int e = 0; e < PER; ++e) {
                if (above < need && above + mine[e] >= need) {
                    found[0] = BINS - 1 - tid * PER - e;
                    found[1] = above;
                }
                above += mine[e];
            }
            __syncthreads();
            t |= (uint32_t)found[0] << shift;
            mask |= ((1u << bits) - 1) << shift;
            need -= found[1];
            __syncthreads();
        }
    }
    // rows of the weight t that stay: the first `need` of them
    int ties_before = 0, out = 0;
    for (int c0 = 0; c0 < u.n_ctx; c0 += CHUNK) {
        if (MORE) load(c0);
        int ties = 0, above = 0;                             // of this thread's rows; above: kept whatever the ties are
        uint32_t tie[(V + 31) / 32] = {}, sure[(V + 31) / 32] = {};
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const int i = c0 + tid * V + e;
            const bool between = i >= lo && i < hi;
            if (between && mask && x[e] == t) { tie[e / 32] |= 1u << e % 32; ++ties; }
            if (i < u.n_ctx && (!between || (mask && x[e] > t))) { sure[e / 32] |= 1u << e % 32; ++above; }
        }
        const int2 tr = scan<THREADS>(ties, waves);
        int left = need - ties_before - tr.x;                // ties this thread may keep
        left = min(max(left, 0), ties);
        const int2 kr = scan<THREADS>(above + left, waves);
        int at = out + kr.x;
#pragma unroll
        for (int e = 0; e < V; ++e) {
            bool keep = sure[e / 32] >> e % 32 & 1;
            if ((tie[e / 32] >> e % 32 & 1) && left > 0) { keep = true; --left; }
            if (keep) rows[at++] = c0 + tid * V + e;
        }
        ties_before += tr.y;
        out += kr.y;
        if (!MORE) break;
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
    const dim3 grid(a.B, a.n_layers * a.n_kv_heads);
    if (a.most_ctx <= 256 * 4) hipLaunchKernelGGL((evict_select_kernel<256, 4, false>), grid, dim3(256), 0, st, a);
    else if (a.most_ctx <= 1024 * 8) hipLaunchKernelGGL((evict_select_kernel<1024, 8, false>), grid, dim3(1024), 0, st, a);
    else if (a.most_ctx <= 1024 * 32) hipLaunchKernelGGL((evict_select_kernel<1024, 32, false>), grid, dim3(1024), 0, st, a);
    else hipLaunchKernelGGL((evict_select_kernel<1024, 32, true>), grid, dim3(1024), 0, st, a);
    hipLaunchKernelGGL(evict_copy_kernel, dim3(a.n_kept, a.n_layers), dim3(256), 0, st, a);
}

}  // namespace ssd
