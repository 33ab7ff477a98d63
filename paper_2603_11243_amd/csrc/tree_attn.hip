// Attention of the nodes of drafted trees over cached rows (Sec. 2.2 for more than one continuation).  Node i sees the rows of its
// context, its ancestors and itself; node j is i or an ancestor of i exactly if i's place in depth-first order lies in the span of j's
// subtree, so that two integers a node are the mask of a tree of any shape.
//   s_ij = scale q_i . k_j,  lse_i = log sum_j exp s_ij,  o_i = sum_j exp(s_ij - lse_i) v_j
// and the weight that row j collects: sum over the nodes and the heads of the K/V head's group of exp(s_ij - lse_i).
#include "device_utils.h"
#include "tree.h"

namespace ssd {

template <int DT> struct Elem;
template <> struct Elem<SSD_F32> {
    typedef float type;
    static __device__ __forceinline__ float get(float v) { return v; }
    static __device__ __forceinline__ float put(float v) { return v; }
};
template <> struct Elem<SSD_BF16> {
    typedef bf16_t type;
    static __device__ __forceinline__ float get(bf16_t v) { return bf16_to_f32(v); }
    static __device__ __forceinline__ bf16_t put(float v) { return f32_to_bf16(v); }
};
template <> struct Elem<SSD_F16> {
    typedef f16_t type;
    static __device__ __forceinline__ float get(f16_t v) { return f16_to_f32(v); }
    static __device__ __forceinline__ f16_t put(float v) { return f32_to_f16(v); }
};

__device__ __forceinline__ bool sees(uint32_t node, uint32_t key) {
    const uint32_t at = node & 0xffffu;
    return at >= (key & 0xffffu) && at < (key >> 16);
}

constexpr int MAX_HD = 128;

// One wavefront a query row, one key a lane.
template <int DT>
__global__ void __launch_bounds__(256) tree_attn_kernel(TreeAttnArgs a) {
    typedef Elem<DT> E;
    typedef typename E::type T;
    __shared__ float qs[4][MAX_HD];
    const TreeItem t = a.items[blockIdx.x];
    const int kvh = blockIdx.y, lane = threadIdx.x % 64, wave = threadIdx.x / 64, hd = a.head_dim;
    const int G = a.n_q_heads / a.n_kv_heads;
    const T* k = (const T*)a.k + (int64_t)t.slot0 * a.slot_stride + kvh * a.head_stride;
    const T* v = (const T*)a.v + (int64_t)t.slot0 * a.slot_stride + kvh * a.head_stride;
    for (int row = t.row0 + wave; row < min(t.row0 + TREE_ROWS, t.n_nodes * G); row += 4) {
        const int node = row / G, head = kvh * G + row % G;
        const T* q = (const T*)a.q + (t.node0 + node) * a.q_stride + (int64_t)head * hd;
        for (int d = lane; d < hd; d += 64) qs[wave][d] = E::get(q[d]);
        __builtin_amdgcn_wave_barrier();
        const uint32_t mine = a.spans[t.node0 + node];
        float m = -INFINITY, l = 0.f, o[2] = {0.f, 0.f};
        const int n = t.n_ctx + node + 1;
        for (int k0 = 0; k0 < n; k0 += 64) {
            const int key = k0 + lane;
            float s = -INFINITY;
            if (key < t.n_ctx || (key < n && sees(mine, a.spans[t.node0 + key - t.n_ctx]))) {
                const T* kr = k + key * a.slot_stride;
                s = 0.f;
                for (int d = 0; d < hd; ++d) s = fmaf(qs[wave][d], E::get(kr[d]), s);
                s *= a.scale;
            }
            const float m_new = fmaxf(m, group_allreduce<64>(s, OpMax()));
            const float base = m_new == -INFINITY ? 0.f : m_new;
            const float alpha = expf(m - base), p = s == -INFINITY ? 0.f : expf(s - base);
            l = l * alpha + group_allreduce<64>(p, OpSum());
            o[0] *= alpha;
            o[1] *= alpha;
            m = m_new;
            for (int j = 0; j < min(64, n - k0); ++j) {
                const float pj = __shfl(p, j);
                if (pj == 0.f) continue;                     // a row that is not seen may hold anything
                const T* vr = v + (k0 + j) * a.slot_stride;
                if (lane < hd) o[0] = fmaf(pj, E::get(vr[lane]), o[0]);
                if (lane + 64 < hd) o[1] = fmaf(pj, E::get(vr[lane + 64]), o[1]);
            }
        }
        T* dst = (T*)a.out + ((int64_t)(t.node0 + node) * a.n_q_heads + head) * hd;
        if (lane < hd) dst[lane] = E::put(o[0] / l);
        if (lane + 64 < hd) dst[lane + 64] = E::put(o[1] / l);
        if (a.lse && lane == 0) a.lse[(int64_t)(t.node0 + node) * a.n_q_heads + head] = m + logf(l);
    }
}

// One key a thread, all query rows of its K/V head.
template <int DT>
__global__ void __launch_bounds__(256) tree_mass_kernel(TreeAttnArgs a) {
    typedef Elem<DT> E;
    typedef typename E::type T;
    const TreeItem t = a.mass_items[blockIdx.x];
    const int kvh = blockIdx.y, hd = a.head_dim, G = a.n_q_heads / a.n_kv_heads;
    for (int key = t.k0 + threadIdx.x; key < t.k1; key += 256) {
    const bool in_tree = key >= t.n_ctx;
    const uint32_t span = in_tree ? a.spans[t.node0 + key - t.n_ctx] : 0;
    const T* k = (const T*)a.k + ((int64_t)t.slot0 + key) * a.slot_stride + kvh * a.head_stride;
    float sum = 0.f;
    for (int row = 0; row < t.n_nodes * G; ++row) {
        const int node = row / G, head = kvh * G + row % G;
        if (in_tree && !sees(a.spans[t.node0 + node], span)) continue;
        const T* q = (const T*)a.q + (t.node0 + node) * a.q_stride + (int64_t)head * hd;
        float s = 0.f;
        for (int d = 0; d < hd; ++d) s = fmaf(E::get(q[d]), E::get(k[d]), s);
        sum += expf(s * a.scale - a.lse[(int64_t)(t.node0 + node) * a.n_q_heads + head]);
    }
    float* dst = a.mass + kvh * a.mass_stride + t.slot0 + key;
    *dst = in_tree ? sum : *dst + sum;
    }
}

template <int DT>
static void launch(const TreeAttnArgs& a, hipStream_t st) {
    hipLaunchKernelGGL((tree_attn_kernel<DT>), dim3(a.n_items, a.n_kv_heads), dim3(256), 0, st, a);
    if (a.mass) hipLaunchKernelGGL((tree_mass_kernel<DT>), dim3(a.n_mass_items, a.n_kv_heads), dim3(256), 0, st, a);
}

void launch_tree_attention(const TreeAttnArgs& a, hipStream_t st) {
    if (a.dtype == SSD_F32) launch<SSD_F32>(a, st);
    else if (a.dtype == SSD_BF16) launch<SSD_BF16>(a, st);
    else launch<SSD_F16>(a, st);
}

}  // namespace ssd
