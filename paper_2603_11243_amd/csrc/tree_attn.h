// What the kernels of tree_attn.hip (16-bit caches) and tree_attn_f32.hip share: element types, the mask, the merge of a workgroup's wavefronts; element
// types and pairs of 16-bit values also with kv_pages.hip and paged_attn.hip.
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

// Pairs of 16-bit values w, as whole numbers (a magnitude plus TO_SIGN reaches the sign bit from the infinities on):
template <bool BF> constexpr uint32_t TO_SIGN = BF ? 0x00800080u : 0x04000400u;
template <bool BF> constexpr uint32_t ONE = BF ? 0x3f80u : 0x3c00u;
constexpr uint32_t SIGNS = 0x80008000u;
template <bool BF> __device__ __forceinline__ uint32_t beyond_of(uint32_t w) { return (w & ~SIGNS) + TO_SIGN<BF>; }   // sign bit: not finite
__device__ __forceinline__ uint32_t not_zero(uint32_t w) { return (w & ~SIGNS) + ~SIGNS; }                               // sign bit: not zero
template <bool BF> __device__ __forceinline__ uint32_t one_where(uint32_t w) { return ((w & SIGNS) >> 15) * ONE<BF>; }
// infinities of a sign (negative: all bits) and NaN as 1, all else 0; what is finite, else 0
template <bool BF> __device__ __forceinline__ uint32_t infinite_of(uint32_t w, uint32_t negative) {
    const uint32_t t = beyond_of<BF>(w);
    return one_where<BF>(t & (~(w ^ negative) | not_zero(t)));
}
template <bool BF> __device__ __forceinline__ uint32_t finite_of(uint32_t w) { return w & ~(((beyond_of<BF>(w) & SIGNS) >> 15) * 0xffffu); }

// Two values to the operand type, round to nearest even, by the conversion instruction of a pair.
typedef float f32x2_t __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
template <bool BF> __device__ __forceinline__ uint32_t pack16(float lo, float hi) {
    const f32x2_t v = {lo, hi};
    if constexpr (BF) return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2_t));
    else return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, f16x2_t));
}
// What the rounding of two values to the pair w left of them, exact in fp32, as another pair.
template <bool BF> __device__ __forceinline__ uint32_t rest16(float lo, float hi, uint32_t w) {
    if constexpr (BF) return pack16<BF>(lo - __uint_as_float(w << 16), hi - __uint_as_float(w & 0xffff0000u));
    else {
        const f16x2_t h = __builtin_bit_cast(f16x2_t, w);
        return pack16<BF>(lo - (float)h.x, hi - (float)h.y);
    }
}

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr float F32_MOST = 3.4028234663852886e38f;

// Scores are taken times a positive scale: the queries carry its sign, and are zero for a scale of zero, whose logits are (so that -infinity, a masked
// score, stays what it is).
__device__ __forceinline__ float scale_of(const TreeAttnArgs& a) { return a.scale == 0.f ? LOG2E : fabsf(a.scale) * LOG2E; }

// Node of a query row (rows are fewer than 2^19, groups at most 512: the product is exact).
__device__ __forceinline__ int node_of(const TreeAttnArgs& a, int row) { return a.group_magic ? (int)__umulhi((uint32_t)row, a.group_magic) : row; }

// An item of work: what its words say.
struct Work { int slot0, n_ctx, n_nodes, node0, row0, k0, k1, index; };
// Query row's number among those of all heads, [node][query head].
__device__ __forceinline__ int64_t row_at(const TreeAttnArgs& a, const Work& t, int kvh, int row) {
    const int node = node_of(a, row);
    return (int64_t)(t.node0 + node) * a.n_q_heads + kvh * a.group + row - node * a.group;
}
__device__ __forceinline__ int64_t query_at(const TreeAttnArgs& a, const Work& t, int kvh, int row, int head_dim) {
    const int node = node_of(a, row);
    return (int64_t)(t.node0 + node) * a.q_stride + (int64_t)(kvh * a.group + row - node * a.group) * head_dim;
}
template <class M>
__device__ __forceinline__ void utterance_of(const TreeAttnArgs& a, const M& w, int b, Work& t) {
    t.slot0 = (int)w(a.utts + 2 * b);
    t.n_ctx = (int)w(a.utts + 2 * b + 1);
    t.node0 = (int)w(a.cu + b);
    t.n_nodes = (int)w(a.cu + b + 1) - t.node0;
}
template <class M>
__device__ __forceinline__ Work item_of(const TreeAttnArgs& a, const M& w, int index, int tile_rows) {
    Work t;
    const uint32_t x = w(6 * index + 3);
    t.index = index;
    t.slot0 = (int)w(6 * index);
    t.n_ctx = (int)w(6 * index + 1);
    t.node0 = (int)w(6 * index + 2);
    t.n_nodes = (int)(x & 0x7ffu);
    t.row0 = (int)(x >> 11) * tile_rows;
    const int node = node_of(a, min(t.n_nodes * a.group, t.row0 + tile_rows) - 1);       // no row of the tile sees a later one
    t.k0 = (int)w(6 * index + 4);
    t.k1 = min(t.n_ctx + node + 1, (int)w(6 * index + 5));
    return t;
}
template <class M>
__device__ __forceinline__ Work mass_item_of(const TreeAttnArgs& a, const M& w, int index) {
    Work t;
    const uint32_t x = w(a.mass_items + index);
    utterance_of(a, w, x & 0xffffu, t);
    const int64_t k0 = (int64_t)(x >> 16) * a.mass_step;
    t.index = index;
    t.row0 = 0;
    t.k0 = (int)k0;
    t.k1 = (int)min((int64_t)t.n_ctx + t.n_nodes, k0 + a.mass_step);
    return t;
}

constexpr int MASS_WAVES = 4;                // wavefronts of a workgroup of the weights
// Wavefronts of a workgroup that split the keys.  Eight leave room for one workgroup a CU, four for two: 16 rows over 150 in 38 utterances, 16 heads on 8 of 128,
// 12.2 and 8.5 us, one row over 106 5.4 and 4.5; 16 over 200000 163 and 164.
constexpr int KEY_WAVES = 4;

// Spans of the keys around the nodes in LDS: SPANS_BEFORE cached rows, the nodes, SPANS_BEHIND keys behind them, as far as a block with a node in it
// reaches.  Every node's place lies in the span of a cached row, nobody's in that of a key behind the nodes (a node does not see a
// later one; a range of keys that ends before the last node ends with a block, or where its rows see nothing more).
constexpr int SPANS_BEFORE = 192, SPANS_BEHIND = 64, SPANS = SPANS_BEFORE + MAX_TREE_NODES + SPANS_BEHIND;
// mine: the span of node threadIdx.x, requested before.
template <int THREADS, class M>
__device__ __forceinline__ void store_spans(uint32_t* span_s, const TreeAttnArgs& a, const M& w, const Work& t, uint32_t mine) {
    const int i = threadIdx.x;
    if (i < SPANS_BEFORE) span_s[i] = 0xffff0000u;
    if (i < SPANS_BEHIND) span_s[SPANS_BEFORE + t.n_nodes + i] = 0u;
    if (i < t.n_nodes) span_s[SPANS_BEFORE + i] = mine;
    for (int j = i + THREADS; j < t.n_nodes; j += THREADS) span_s[SPANS_BEFORE + j] = w(a.spans + t.node0 + j);
    static_assert(THREADS >= SPANS_BEFORE && SPANS_BEFORE >= SPANS_BEHIND, "one pass");
}
// Those of a lane's keys k0 + 16 c + 4 (lane / 16) + r (blocks far before the nodes: of other cached rows, which are alike).
template <int C>
__device__ __forceinline__ void key_spans(uint32_t (&key)[C][4], const Work& t, int k0, const uint32_t* span_s) {
    const uint32_t* from = span_s + max(SPANS_BEFORE + k0 - t.n_ctx, 0) + 4 * (threadIdx.x % 64 / 16);
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int r = 0; r < 4; ++r) key[c][r] = from[16 * c + r];
}

// Weights times values near the end of fp32's range (bfloat16 has the same) can leave it in the sum over many keys, though the division by the sum of
// the weights would bring it back.  A pass with such an output is repeated, in the rows that have one, with weights 2^-DOWN of theirs: 2^30 keys of weight 2^-DOWN
// sum up to 1/2.  Wavefronts and pieces are joined as means with shares of 1 in all, which stay inside.
constexpr float DOWN = 31.f;
__device__ __forceinline__ float lifted(float l, float down) { return down > 0.f ? l * 0x1p31f : l; }

// Rows of a wavefront's output with an infinity or NaN; whether there are any.
template <int NT, int DT>
__device__ __forceinline__ bool not_finite(const f32x4_t (&o)[NT][DT], bool (&odd)[NT]) {
    bool any = false;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        float t = 0.f;
#pragma unroll
        for (int i = 0; i < DT; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) t = fmaf(o[n][i][r], 0.f, t);
        odd[n] = t != t;
        any |= odd[n];
    }
    if (!__any(any)) return false;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        int x = odd[n];
        x |= __shfl_xor(x, 16);
        x |= __shfl_xor(x, 32);
        odd[n] = x != 0;
    }
    return true;
}

// The end of an attention workgroup: its wavefronts hold, for 16 NT rows, maxima m (raw scores), sums l (a lane's share) and outputs o[n][i] (row
// 16 n + lane % 16, dims 16 i + 4 (lane / 16) ..) relative to 2^(m sc - bias + down).  DPASS dims of all rows at a time go through LDS (buf: 16 HD floats a wavefront,
// the 16-byte chunks of a row permuted by its number) as means; every thread adds VPT values of a row, each by its wavefront's share of the weights, and stores them.
template <int DT, int HD, int NT, int WAVES>
__device__ __forceinline__ void merge_wavefronts(const TreeAttnArgs& a, const Work& t, int kvh, const float (&m)[NT], float (&l)[NT], const f32x4_t (&o)[NT][HD / 16],
                                                 const float (&down)[NT], float sc, float bias, float* buf, float2* ml_s) {
    typedef Elem<DT> E;
    constexpr int TR = 16 * NT, DPASS = 16 * HD / TR, VPT = TR * DPASS / (64 * WAVES), TPR = 64 * WAVES / TR;      // values of a thread, threads of a row
    const int lane = threadIdx.x % 64, kg = lane / 16, dc = lane % 16, wave = threadIdx.x / 64;
    const int G = a.group, R = t.n_nodes * G;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        l[n] += __shfl_xor(l[n], 16);
        l[n] += __shfl_xor(l[n], 32);
        if (kg == 0) ml_s[wave * TR + 16 * n + dc] = make_float2(m[n], lifted(l[n], down[n]));
        l[n] = l[n] == 0.f ? 0.f : 1.f / l[n];               // (nothing seen, nothing added)
    }
    static_assert(VPT == 2 || VPT == 4 || VPT == 8, "values of a thread");
    constexpr int CH = DPASS / 4;                            // chunks of a row
    const int orow = threadIdx.x / TPR, ocol = threadIdx.x % TPR * VPT;
    const int row = t.row0 + orow;
    float w[WAVES], mt = -F32_MOST, lt = 0.f;
#pragma unroll
    for (int pass = 0; pass < HD / DPASS; ++pass) {
        if (pass) __syncthreads();
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int i = 0; i < DPASS / 16; ++i) {
                const int r = 16 * n + dc, c = 4 * i + kg;
                *reinterpret_cast<f32x4_t*>(buf + (wave * TR + r) * DPASS + (c ^ (r & (CH - 1))) * 4) = o[n][pass * (DPASS / 16) + i] * l[n];
            }
        __syncthreads();
        if (pass == 0) {
#pragma unroll
            for (int u = 0; u < WAVES; ++u) mt = fmaxf(mt, ml_s[u * TR + orow].x);
#pragma unroll
            for (int u = 0; u < WAVES; ++u) {
                const float2 x = ml_s[u * TR + orow];
                w[u] = x.y == 0.f ? 0.f : x.y * __builtin_amdgcn_exp2f((x.x - mt) * sc);
                lt += w[u];
            }
            const float inv = 1.f / lt;
#pragma unroll
            for (int u = 0; u < WAVES; ++u) w[u] *= inv;
        }
        float v[VPT];
#pragma unroll
        for (int e = 0; e < VPT; ++e) v[e] = 0.f;
#pragma unroll
        for (int u = 0; u < WAVES; ++u)
#pragma unroll
            for (int e = 0; e < VPT; ++e) v[e] = fmaf(buf[(u * TR + orow) * DPASS + ((ocol + e) / 4 ^ (orow & (CH - 1))) * 4 + (ocol + e) % 4], w[u], v[e]);
        if (row >= R) continue;
        const int dim = pass * DPASS + ocol;
        if (t.index < a.n_parts) {
            float* dst = a.part_o + ((int64_t)(t.index * a.n_kv_heads + kvh) * TR + orow) * HD + dim;
#pragma unroll
            for (int e = 0; e < VPT; ++e) dst[e] = v[e];
        } else {
            typename E::type* dst = (typename E::type*)a.out + (row_at(a, t, kvh, row)) * a.head_dim + dim;
            if constexpr (DT == SSD_F32) {                   // (head_dim is a multiple of 4 and may end among a thread's 8 values)
                static_assert(VPT % 4 == 0, "groups of four");
#pragma unroll
                for (int e = 0; e < VPT; e += 4)
                    if (dim + e < a.head_dim) *reinterpret_cast<f32x4_t*>(dst + e) = (f32x4_t){v[e], v[e + 1], v[e + 2], v[e + 3]};
            } else {
                uint32_t x[VPT / 2];
#pragma unroll
                for (int e = 0; e < VPT; e += 2) x[e / 2] = op_pack2<DT == SSD_BF16>(v[e], v[e + 1]);
                if constexpr (VPT == 8) *reinterpret_cast<uint4*>(dst) = make_uint4(x[0], x[1], x[2], x[3]);
                else if constexpr (VPT == 4) *reinterpret_cast<uint2*>(dst) = make_uint2(x[0], x[1]);
                else *reinterpret_cast<uint32_t*>(dst) = x[0];
            }
        }
    }
    if (ocol == 0 && row < R) {
        if (t.index < a.n_parts) a.part_ml[(int64_t)(t.index * a.n_kv_heads + kvh) * TR + orow] = make_float2(mt, lt);
        else if (a.lse) a.lse[row_at(a, t, kvh, row)] = (mt * sc - bias + __builtin_amdgcn_logf(lt)) * LN2;
    }
}

// The pieces of a long context, a mean of values each, joined.  A workgroup has a query row: groups of HD / 4 lanes take its pieces in turn, each with a running
// maximum and mean, and are joined through LDS: 48 rows of 8 heads in 64 pieces 5.9 us (one lane a dim over all pieces: 125, the pieces' latencies one after the other).
template <int DT, int HD, class M>
__global__ void __launch_bounds__(256) tree_join_kernel(TreeAttnArgs a, M w, float bias) {
    typedef Elem<DT> E;
    constexpr int LANES = HD / 4, GROUPS = 256 / LANES;
    __shared__ f32x4_t o_s[GROUPS][LANES];
    __shared__ float2 ml_s[GROUPS];
    const int j = blockIdx.x / a.tile_rows, r = blockIdx.x % a.tile_rows, kvh = blockIdx.y, G = a.group;
    const uint32_t x = w(a.joins + 3 * j);
    const int item0 = (int)w(a.joins + 3 * j + 1), n_parts = (int)w(a.joins + 3 * j + 2);
    Work t;
    utterance_of(a, w, x & 0xffffu, t);
    const int R = t.n_nodes * G, tiles = (R + a.tile_rows - 1) / a.tile_rows, row = (int)(x >> 16) * a.tile_rows + r;
    if (row >= R) return;
    const float sc = scale_of(a);
    const int group = threadIdx.x / LANES, dim = threadIdx.x % LANES * 4;
    float m = -F32_MOST, l = 0.f;
    f32x4_t v = {0.f, 0.f, 0.f, 0.f};
    constexpr int U = 4;                                     // pieces requested at once
    for (int p0 = group; p0 < n_parts; p0 += U * GROUPS) {
        float2 y[U];
        f32x4_t z[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int p = min(p0 + u * GROUPS, n_parts - 1);
            const int64_t at = ((int64_t)(item0 + p * tiles) * a.n_kv_heads + kvh) * a.tile_rows + r;
            y[u] = a.part_ml[at];
            z[u] = *reinterpret_cast<const f32x4_t*>(a.part_o + at * HD + dim);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (p0 + u * GROUPS >= n_parts || y[u].y == 0.f) continue;                     // (a piece whose keys no row of the tile sees)
            const float top = fmaxf(m, y[u].x), old = l * __builtin_amdgcn_exp2f((m - top) * sc), now = y[u].y * __builtin_amdgcn_exp2f((y[u].x - top) * sc);
            m = top;
            l = old + now;
            const float inv = 1.f / l;
            v = v * (old * inv) + z[u] * (now * inv);
        }
    }
    o_s[group][dim / 4] = v;
    if (dim == 0) ml_s[group] = make_float2(m, l);
    __syncthreads();
    if (group) return;
    float mt = -F32_MOST, lt = 0.f;
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) mt = fmaxf(mt, ml_s[g].x);
    f32x4_t s = {0.f, 0.f, 0.f, 0.f};
    float f[GROUPS];
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
        const float2 y = ml_s[g];
        f[g] = y.y == 0.f ? 0.f : y.y * __builtin_amdgcn_exp2f((y.x - mt) * sc);
        lt += f[g];
    }
    const float inv = 1.f / lt;
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) s += o_s[g][dim / 4] * (f[g] * inv);
    const int64_t at = row_at(a, t, kvh, row);
    typename E::type* dst = (typename E::type*)a.out + at * a.head_dim + dim;
    if (dim < a.head_dim)
#pragma unroll
        for (int e = 0; e < 4; ++e) dst[e] = E::put(s[e]);
    if (a.lse && dim == 0) a.lse[at] = (mt * sc - bias + __builtin_amdgcn_logf(lt)) * LN2;
}

// Adds the weights of a 32- or 16-key block: acc[c][r] belongs to key k0 + 16 c + 4 (lane / 16) + r and is a lane's share of it.  fresh: the first rows
// of the tree are in it, so that the entry of a node row is stored; every key has one workgroup and one lane.
template <int C>
__device__ __forceinline__ void add_mass(const TreeAttnArgs& a, const Work& t, int kvh, int k0, bool fresh, f32x4_t (&acc)[C]) {
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
    float* dst = a.mass + (int64_t)kvh * a.mass_stride + t.slot0 + key;
    *dst = fresh && key >= t.n_ctx ? mine : *dst + mine;
}

template <class M> void launch_tree_attention32(const TreeAttnArgs& a, const M& w, hipStream_t st);

}  // namespace ssd
