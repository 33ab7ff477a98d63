// What the kernels of tree_attn.hip (16-bit caches) and tree_attn_f32.hip share: element types, the mask, the merge of a workgroup's wavefronts.
#pragma once
#include "gemm_core.h"
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

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr float F32_MOST = 3.4028234663852886e38f;

constexpr int TREE_WAVES = 4;

// The end of an attention workgroup: its wavefronts hold, for 16 NT rows, maxima m (raw scores), sums l (a lane's share) and outputs o[n][i] (row
// 16 n + lane % 16, dims 16 i + 4 (lane / 16) ..) relative to 2^(m sc - bias).  DPASS dims of all rows at a time go through LDS (buf: 16 HD floats a wavefront,
// the 16-byte chunks of a row permuted by its number); every thread adds VPT values of a row and stores them, or the sums of a piece.
template <int DT, int HD, int NT>
__device__ __forceinline__ void merge_wavefronts(const TreeAttnArgs& a, const TreeItem& t, int kvh, const float (&m)[NT], float (&l)[NT], const f32x4_t (&o)[NT][HD / 16],
                                                 float sc, float bias, float* buf, float2* ml_s) {
    typedef Elem<DT> E;
    constexpr int TR = 16 * NT, DPASS = 16 * HD / TR, VPT = HD / 16;
    const int lane = threadIdx.x % 64, kg = lane / 16, dc = lane % 16, wave = threadIdx.x / 64;
    const int G = a.n_q_heads / a.n_kv_heads, R = t.n_nodes * G;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        l[n] += __shfl_xor(l[n], 16);
        l[n] += __shfl_xor(l[n], 32);
        if (kg == 0) ml_s[wave * TR + 16 * n + dc] = make_float2(m[n], l[n]);
    }
    constexpr int CH = DPASS / 4;                            // chunks of a row
    const int orow = threadIdx.x / (256 / TR), ocol = threadIdx.x % (256 / TR) * VPT;
    const int row = t.row0 + orow;
    float w[TREE_WAVES], mt = -F32_MOST, lt = 0.f;
#pragma unroll
    for (int pass = 0; pass < HD / DPASS; ++pass) {
        if (pass) __syncthreads();
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int i = 0; i < DPASS / 16; ++i) {
                const int r = 16 * n + dc, c = 4 * i + kg;
                *reinterpret_cast<f32x4_t*>(buf + (wave * TR + r) * DPASS + (c ^ (r & (CH - 1))) * 4) = o[n][pass * (DPASS / 16) + i];
            }
        __syncthreads();
        if (pass == 0) {
#pragma unroll
            for (int u = 0; u < TREE_WAVES; ++u) mt = fmaxf(mt, ml_s[u * TR + orow].x);
#pragma unroll
            for (int u = 0; u < TREE_WAVES; ++u) {
                const float2 x = ml_s[u * TR + orow];
                w[u] = x.y == 0.f ? 0.f : __builtin_amdgcn_exp2f((x.x - mt) * sc);
                lt = fmaf(x.y, w[u], lt);
            }
        }
        float v[VPT];
#pragma unroll
        for (int e = 0; e < VPT; ++e) v[e] = 0.f;
#pragma unroll
        for (int u = 0; u < TREE_WAVES; ++u)
#pragma unroll
            for (int e = 0; e < VPT; e += 4) {
                const f32x4_t x = *reinterpret_cast<const f32x4_t*>(buf + (u * TR + orow) * DPASS + ((ocol + e) / 4 ^ (orow & (CH - 1))) * 4);
#pragma unroll
                for (int f = 0; f < 4; ++f) v[e + f] = fmaf(x[f], w[u], v[e + f]);
            }
        if (row >= R) continue;
        const int dim = pass * DPASS + ocol;
        if (t.part >= 0) {
            float* dst = a.part_o + ((int64_t)(t.part * a.n_kv_heads + kvh) * TR + orow) * HD + dim;
#pragma unroll
            for (int e = 0; e < VPT; e += 4) *reinterpret_cast<f32x4_t*>(dst + e) = (f32x4_t){v[e], v[e + 1], v[e + 2], v[e + 3]};
        } else {
            const float inv = 1.f / lt;
            typename E::type* dst = (typename E::type*)a.out + ((int64_t)(t.node0 + row / G) * a.n_q_heads + kvh * G + row % G) * a.head_dim + dim;
            if constexpr (DT == SSD_F32) {
#pragma unroll
                for (int e = 0; e < VPT; e += 4)
                    if (dim + e < a.head_dim) *reinterpret_cast<f32x4_t*>(dst + e) = (f32x4_t){v[e] * inv, v[e + 1] * inv, v[e + 2] * inv, v[e + 3] * inv};
            } else {
                uint32_t x[VPT / 2];
#pragma unroll
                for (int e = 0; e < VPT; e += 2) x[e / 2] = op_pack2<DT == SSD_BF16>(v[e] * inv, v[e + 1] * inv);
                if constexpr (VPT == 8) *reinterpret_cast<uint4*>(dst) = make_uint4(x[0], x[1], x[2], x[3]);
                else *reinterpret_cast<uint2*>(dst) = make_uint2(x[0], x[1]);
            }
        }
    }
    if (ocol == 0 && row < R) {
        if (t.part >= 0) a.part_ml[(int64_t)(t.part * a.n_kv_heads + kvh) * TR + orow] = make_float2(mt, lt);
        else if (a.lse) a.lse[(int64_t)(t.node0 + row / G) * a.n_q_heads + kvh * G + row % G] = (mt * sc - bias + __builtin_amdgcn_logf(lt)) * LN2;
    }
}

// The pieces of a long context joined: one group of HD / 4 lanes a query row.
template <int DT, int HD>
__global__ void __launch_bounds__(256) tree_join_kernel(TreeAttnArgs a, int tile_rows, float bias) {
    typedef Elem<DT> E;
    constexpr int LANES = HD / 4, ROWS = 256 / LANES;
    const TreeJoin t = a.joins[blockIdx.x];
    const int kvh = blockIdx.y, G = a.n_q_heads / a.n_kv_heads;
    const int r = blockIdx.z * ROWS + threadIdx.x / LANES, row = t.row0 + r, dim = threadIdx.x % LANES * 4;
    if (r >= tile_rows || row >= t.n_nodes * G) return;
    const float sc = fabsf(a.scale) * LOG2E;
    float mt = -F32_MOST, lt = 0.f;
    for (int p = 0; p < t.n_parts; ++p) mt = fmaxf(mt, a.part_ml[(int64_t)((t.part0 + p * t.stride) * a.n_kv_heads + kvh) * tile_rows + r].x);
    f32x4_t v = {0.f, 0.f, 0.f, 0.f};
    for (int p = 0; p < t.n_parts; ++p) {
        const int64_t at = (int64_t)((t.part0 + p * t.stride) * a.n_kv_heads + kvh) * tile_rows + r;
        const float2 x = a.part_ml[at];
        const float w = x.y == 0.f ? 0.f : __builtin_amdgcn_exp2f((x.x - mt) * sc);
        lt = fmaf(x.y, w, lt);
        const f32x4_t y = *reinterpret_cast<const f32x4_t*>(a.part_o + at * HD + dim);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = fmaf(y[e], w, v[e]);
    }
    const int64_t at = (int64_t)(t.node0 + row / G) * a.n_q_heads + kvh * G + row % G;
    typename E::type* dst = (typename E::type*)a.out + at * a.head_dim + dim;
    const float inv = 1.f / lt;
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (dim + e < a.head_dim) dst[e] = E::put(v[e] * inv);
    if (a.lse && dim == 0) a.lse[at] = (mt * sc - bias + __builtin_amdgcn_logf(lt)) * LN2;
}

// Adds the weights of a 32- or 16-key block: acc[c][r] belongs to key k0 + 16 c + 4 (lane / 16) + r and is a lane's share of it.  fresh: the first rows
// of the tree are in it, so that the entry of a node row is stored; every key has one workgroup and one lane.
template <int C>
__device__ __forceinline__ void add_mass(const TreeAttnArgs& a, const TreeItem& t, int kvh, int k0, bool fresh, f32x4_t (&acc)[C]) {
    const int lane = threadIdx.x % 64, kg = lane / 16, dc = lane % 16;
    float mine = 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const float sum = group_allreduce<16>(acc[c][r], OpSum());
            mine = dc == 4 * c + r ? sum : mine;
        }
    const int key = k0 + 16 * (dc / 4) + 4 * kg + dc % 4;
    if (dc >= 4 * C || key >= t.k1) return;
    float* dst = a.mass + kvh * a.mass_stride + t.slot0 + key;
    *dst = fresh && key >= t.n_ctx ? mine : *dst + mine;
}

void launch_tree_attention32(const TreeAttnArgs& a, hipStream_t st);

}  // namespace ssd
