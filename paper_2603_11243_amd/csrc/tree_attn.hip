// Attention of the nodes of drafted trees over cached rows (Sec. 2.2 for more than one continuation).  Node i sees the rows of its
// context, its ancestors and itself; node j is i or an ancestor of i exactly if i's place in depth-first order lies in the span of j's
// subtree, so that two integers a node are the mask of a tree of any shape.
//   s_ij = scale q_i . k_j,  lse_i = log sum_j exp s_ij,  o_i = sum_j exp(s_ij - lse_i) v_j
// and the weight that row j collects: sum over the nodes and the heads of the K/V head's group of exp(s_ij - lse_i).
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

// ---- 16-bit caches ----------------------------------------------------------------------------------------------------------------
// A workgroup is four wavefronts and serves 16 NT query rows (node, head of the group) of one K/V head over a range of keys.  The
// wavefronts take the 32-key blocks of the range in turn, so that every cached row is read once for all of these rows, and merge their
// (max, sum, output) through LDS.  Both products are v_mfma_f32_16x16x32: S^T = K Q^T with the key rows straight from memory in operand
// registers, O^T += V^T P^T with the values in LDS (global -> LDS loads, read back through the transposing ds_read_b64_tr_b16); keys
// 4g .. 4g + 3 and 16 + 4g .. of a block are a lane's scores and its operand of the second product alike.
// The maximum that the exponents refer to may lag behind the true one by 2^LAG: it is raised (and the output rescaled) only by a score
// beyond that, which spares nearly every block the exchange between lanes and the rescaling.  Probabilities enter the second product in
// the type of the cache, their sum does not: half a step of the type each, as the output's own rounding.  IEEE half holds them times
// 2^BIAS, so that those down to 2^-31 of the largest count (2^(BIAS + LAG) is in its range); bfloat16 has the range of fp32, and there they
// stay below 1 so that values near its end do not overflow the sums.
constexpr int TREE_WAVES = 4;
constexpr int TREE_KEYS = 32;
constexpr float LAG = 8.f;
template <bool BF> constexpr float BIAS = BF ? -LAG : 6.f;

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

template <bool BF, int HD, int NT>
__global__ void __launch_bounds__(64 * TREE_WAVES, NT == 4 ? 1 : 2) tree_attn16_kernel(TreeAttnArgs a) {
    constexpr int ROW = HD * 2, BLOCK = TREE_KEYS * ROW, STEP = TREE_KEYS * TREE_WAVES;
    constexpr int KS = HD / 32, DT = HD / 16, TR = 16 * NT;
    constexpr int ROW_CHUNKS = ROW / 16, V_ROWS = 64 / ROW_CHUNKS, V_LOADS = TREE_KEYS / V_ROWS, K_LOADS = 2 * KS;
    constexpr int DPASS = 16 * HD / TR, VPT = HD / 16;       // dims of a merge pass; values of a thread in it
    __shared__ __align__(1024) unsigned char v_s[TREE_WAVES][BLOCK];
    __shared__ float2 ml_s[TREE_WAVES][TR];
    __shared__ uint32_t span_s[MAX_TREE_NODES];
    const int lane = threadIdx.x % 64, kg = lane / 16, dc = lane % 16;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int work = xcd_contiguous_index(blockIdx.x, gridDim.x);
    const TreeItem t = a.items[work / a.n_kv_heads];
    const int kvh = work % a.n_kv_heads;
    const int G = a.n_q_heads / a.n_kv_heads, R = t.n_nodes * G;
    const int last = max(t.k0, t.k1 - 1);                    // (a range without keys: any row)
    const int n_spans = t.k1 > t.n_ctx ? t.n_nodes : 0;
    const uint32_t span = (int)threadIdx.x < n_spans ? a.spans[t.node0 + threadIdx.x] : 0u;
    const int stride2 = (int)a.slot_stride * 2;
    const int64_t first = (int64_t)t.slot0 * a.slot_stride + kvh * a.head_stride;
    const uint16_t* kbase = (const uint16_t*)a.k + first;
    const uint16_t* vbase = (const uint16_t*)a.v + first;

    // Keys k0 .. k0 + 31: lane (row dc of a half of 16, dims 8 kg + 32 s) in registers.  Values: rows of an instruction one behind the
    // other, the 16-byte chunks of a row permuted by its number so that the 32-byte pieces that half a wavefront reads lie in all LDS
    // banks.  Rows behind the range are copies of its last one: masked, or of a block behind the wavefront's last, which is requested all the same.
    u32x4_t kr[2][KS];
    auto load_keys = [&](int k0) {
        const int r0 = min(k0, last), beyond = last - r0;
        const __amdgpu_buffer_rsrc_t rsrc = make_rsrc(kbase + (int64_t)r0 * a.slot_stride);
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const int off = min(16 * c + dc, beyond) * stride2 + kg * 16;
#pragma unroll
            for (int s = 0; s < KS; ++s) kr[c][s] = __builtin_amdgcn_raw_buffer_load_b128(rsrc, off + 64 * s, 0, 0);
        }
    };
    auto swizzle = [](int row) { return HD == 128 ? 4 * (row & 3) + 2 * (row >> 2 & 1) : 2 * (row >> 1 & 3); };
    auto load_values = [&](int k0) {
        const int r0 = min(k0, last), beyond = last - r0;
        const __amdgpu_buffer_rsrc_t rsrc = make_rsrc(vbase + (int64_t)r0 * a.slot_stride);
#pragma unroll
        for (int i = 0; i < V_LOADS; ++i) {
            const int row = V_ROWS * i + lane / ROW_CHUNKS;
            const int off = min(row, beyond) * stride2 + ((lane % ROW_CHUNKS) ^ swizzle(row)) * 16;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (lds_void_t*)(v_s[wave] + i * 1024), 16, off, 0, 0, 0);
        }
    };
    int k0 = t.k0 + wave * TREE_KEYS;
    load_keys(k0);
    load_values(k0);

    // queries: column dc of tile n is row row0 + 16 n + dc (a copy of the last one behind it); a negative scale is theirs
    f16x8_t qf[NT][KS];
    const uint32_t flip = a.scale < 0.f ? 0x80008000u : 0u;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int row = min(t.row0 + 16 * n + dc, R - 1);
        const uint16_t* q = (const uint16_t*)a.q + (int64_t)(t.node0 + row / G) * a.q_stride + (kvh * G + row % G) * HD + kg * 8;
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            uint4 w = *reinterpret_cast<const uint4*>(q + 32 * s);
            w.x ^= flip; w.y ^= flip; w.z ^= flip; w.w ^= flip;
            qf[n][s] = as_f16x8(w);
        }
    }
    const float sc = fabsf(a.scale) * LOG2E;
    float m[NT], l[NT];
    f32x4_t o[NT][DT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        m[n] = -F32_MOST;
        l[n] = 0.f;
#pragma unroll
        for (int i = 0; i < DT; ++i) o[n][i] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
    }
    if ((int)threadIdx.x < n_spans) span_s[threadIdx.x] = span;
    for (int i = threadIdx.x + 64 * TREE_WAVES; i < n_spans; i += 64 * TREE_WAVES) span_s[i] = a.spans[t.node0 + i];
    // the spans have been written; a barrier with a fence would wait for the rows as well
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0xC07F);
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");

    // transposing read: lane i of 16 passes row i / 4 and dims 4 (i % 4) .. + 3 of a 16-dim block, lane j receives dim j of four rows
    const int v_row = 4 * kg + dc / 4, v_low = (dc % 4) / 2, v_sub = (dc % 2) * 8;
    auto block = [&](auto masked_c, int k0) {
        constexpr bool MASKED = decltype(masked_c)::value;
        f32x4_t s[NT][2];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                s[n][c] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int e = 0; e < KS; ++e) s[n][c] = mfma_16x16x32<BF>(__builtin_bit_cast(f16x8_t, kr[c][e]), qf[n][e], s[n][c]);
            }
        __builtin_amdgcn_sched_barrier(0);
        load_keys(k0 + STEP);
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (MASKED) {
            uint32_t key[2][4];                              // the keys' spans: all of the context, nothing behind the range
#pragma unroll
            for (int c = 0; c < 2; ++c)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int at = k0 + 16 * c + 4 * kg + r;
                    key[c][r] = at < t.n_ctx ? 0xffff0000u : at < t.k1 ? span_s[at - t.n_ctx] : 0u;
                }
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const uint32_t mine = span_s[min(t.row0 + 16 * n + dc, R - 1) / G];
#pragma unroll
                for (int c = 0; c < 2; ++c)
#pragma unroll
                    for (int r = 0; r < 4; ++r) s[n][c][r] = sees(mine, key[c][r]) ? s[n][c][r] : -INFINITY;
            }
        }
        float mx[NT];
        bool above = false;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            mx[n] = fmaxf(fmaxf(fmaxf(s[n][0][0], s[n][0][1]), fmaxf(s[n][0][2], s[n][0][3])), fmaxf(fmaxf(s[n][1][0], s[n][1][1]), fmaxf(s[n][1][2], s[n][1][3])));
            above |= (mx[n] - m[n]) * sc > LAG;
        }
        if (__any(above)) {
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                float top = fmaxf(mx[n], __shfl_xor(mx[n], 16));
                top = fmaxf(m[n], fmaxf(top, __shfl_xor(top, 32)));
                const float alpha = __builtin_amdgcn_exp2f((m[n] - top) * sc);
                m[n] = top;
                l[n] *= alpha;
#pragma unroll
                for (int i = 0; i < DT; ++i) o[n][i] *= alpha;
            }
        }
        f16x8_t pf[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const float base = BIAS<BF> - m[n] * sc;
            uint32_t pw[4];
#pragma unroll
            for (int c = 0; c < 2; ++c) {
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float p = __builtin_amdgcn_exp2f(fmaf(s[n][c][r], sc, base));
                    s[n][c][r] = MASKED && s[n][c][r] == -INFINITY ? 0.f : p;
                    l[n] += s[n][c][r];
                }
                pw[2 * c] = op_pack2<BF>(s[n][c][0], s[n][c][1]);
                pw[2 * c + 1] = op_pack2<BF>(s[n][c][2], s[n][c][3]);
            }
            pf[n] = as_f16x8(make_uint4(pw[0], pw[1], pw[2], pw[3]));
        }
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_waitcnt(0x0F70 | K_LOADS);        // the values of this block have landed (a wavefront reads its own only)
        __builtin_amdgcn_sched_barrier(0);
        tr_v4i16 vf[DT][2];
#pragma unroll
        for (int i = 0; i < DT; ++i) {
            const unsigned char* p = v_s[wave] + v_row * ROW + (((2 * i) | v_low) ^ swizzle(v_row)) * 16 + v_sub;
            vf[i][0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_tr_v4i16*)p);
            vf[i][1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_tr_v4i16*)(p + 16 * ROW));
        }
        __builtin_amdgcn_sched_barrier(0);
        // A value that is not finite would reach the rows that do not see it as 0 times infinity.  In a block that holds one the products run
        // on the others, and two more count the infinities of either sign (a NaN as both) that rows with a probability meet.
        uint32_t odd = 0;
        if constexpr (MASKED) {
#pragma unroll
            for (int i = 0; i < DT; ++i)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const uint2 w = __builtin_bit_cast(uint2, vf[i][e]);
                    odd |= beyond_of<BF>(w.x) | beyond_of<BF>(w.y);
                }
        }
        if (MASKED && __any(odd & SIGNS)) {
            f16x8_t there[NT];
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const uint4 w = __builtin_bit_cast(uint4, pf[n]);
                there[n] = as_f16x8(make_uint4(one_where<BF>(not_zero(w.x)), one_where<BF>(not_zero(w.y)), one_where<BF>(not_zero(w.z)), one_where<BF>(not_zero(w.w))));
            }
#pragma unroll
            for (int i = 0; i < DT; ++i) {
                __builtin_amdgcn_sched_barrier(0);           // (one after the other: registers, not speed)
                const uint2 x = __builtin_bit_cast(uint2, vf[i][0]), y = __builtin_bit_cast(uint2, vf[i][1]);
                const f16x8_t up = as_f16x8(make_uint4(infinite_of<BF>(x.x, 0), infinite_of<BF>(x.y, 0), infinite_of<BF>(y.x, 0), infinite_of<BF>(y.y, 0)));
                const f16x8_t down = as_f16x8(make_uint4(infinite_of<BF>(x.x, ~0u), infinite_of<BF>(x.y, ~0u), infinite_of<BF>(y.x, ~0u), infinite_of<BF>(y.y, ~0u)));
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    const f32x4_t zero = {0.f, 0.f, 0.f, 0.f}, u = mfma_16x16x32<BF>(up, there[n], zero), d = mfma_16x16x32<BF>(down, there[n], zero);
#pragma unroll
                    for (int r = 0; r < 4; ++r) o[n][i][r] += (u[r] > 0.f ? INFINITY : 0.f) - (d[r] > 0.f ? INFINITY : 0.f);
                }
                vf[i][0] = __builtin_bit_cast(tr_v4i16, make_uint2(finite_of<BF>(x.x), finite_of<BF>(x.y)));
                vf[i][1] = __builtin_bit_cast(tr_v4i16, make_uint2(finite_of<BF>(y.x), finite_of<BF>(y.y)));
            }
        }
#pragma unroll
        for (int i = 0; i < DT; ++i) {
            const f16x8_t v = __builtin_bit_cast(f16x8_t, __builtin_shufflevector(vf[i][0], vf[i][1], 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
            for (int n = 0; n < NT; ++n) o[n][i] = mfma_16x16x32<BF>(v, pf[n], o[n][i]);
        }
        __builtin_amdgcn_s_waitcnt(0xC07F);                  // the reads of this block are done
        __builtin_amdgcn_sched_barrier(0);
        load_values(k0 + STEP);
    };
    for (; k0 + TREE_KEYS <= min(t.n_ctx, t.k1); k0 += STEP) block(std::false_type(), k0);
    for (; k0 < t.k1; k0 += STEP) block(std::true_type(), k0);
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt(0x0F70);                      // the values behind the last block: they land where the output goes
    __builtin_amdgcn_sched_barrier(0);

    // ---- merge: DPASS dims of all rows at a time through the wavefronts' blocks of values, the 16-byte chunks of a row permuted
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        l[n] += __shfl_xor(l[n], 16);
        l[n] += __shfl_xor(l[n], 32);
        if (kg == 0) ml_s[wave][16 * n + dc] = make_float2(m[n], l[n]);
    }
    constexpr int CH = DPASS / 4;                            // chunks of a row
    float* mine = reinterpret_cast<float*>(v_s[wave]);
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
                *reinterpret_cast<f32x4_t*>(mine + r * DPASS + (c ^ (r & (CH - 1))) * 4) = o[n][pass * (DPASS / 16) + i];
            }
        __syncthreads();
        if (pass == 0) {
#pragma unroll
            for (int u = 0; u < TREE_WAVES; ++u) mt = fmaxf(mt, ml_s[u][orow].x);
#pragma unroll
            for (int u = 0; u < TREE_WAVES; ++u) {
                const float2 x = ml_s[u][orow];
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
                const f32x4_t x = *reinterpret_cast<const f32x4_t*>(reinterpret_cast<const float*>(v_s[u]) + orow * DPASS + ((ocol + e) / 4 ^ (orow & (CH - 1))) * 4);
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
            uint32_t x[VPT / 2];
#pragma unroll
            for (int e = 0; e < VPT; e += 2) x[e / 2] = op_pack2<BF>(v[e] * inv, v[e + 1] * inv);
            uint16_t* dst = (uint16_t*)a.out + ((int64_t)(t.node0 + row / G) * a.n_q_heads + kvh * G + row % G) * HD + dim;
            if constexpr (VPT == 8) *reinterpret_cast<uint4*>(dst) = make_uint4(x[0], x[1], x[2], x[3]);
            else *reinterpret_cast<uint2*>(dst) = make_uint2(x[0], x[1]);
        }
    }
    if (ocol == 0 && row < R) {
        if (t.part >= 0) a.part_ml[(int64_t)(t.part * a.n_kv_heads + kvh) * TR + orow] = make_float2(mt, lt);
        else if (a.lse) a.lse[(int64_t)(t.node0 + row / G) * a.n_q_heads + kvh * G + row % G] = (mt * sc - BIAS<BF> + __builtin_amdgcn_logf(lt)) * LN2;
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
    for (int row = t.row0 + wave; row < min(t.row0 + a.tile_rows, t.n_nodes * G); row += 4) {
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

template <bool BF, int HD>
static void launch16(const TreeAttnArgs& a, hipStream_t st) {
    const dim3 grid(a.n_items * a.n_kv_heads);
    if (a.tile_rows == 16) hipLaunchKernelGGL((tree_attn16_kernel<BF, HD, 1>), grid, dim3(64 * TREE_WAVES), 0, st, a);
    else if (a.tile_rows == 32) hipLaunchKernelGGL((tree_attn16_kernel<BF, HD, 2>), grid, dim3(64 * TREE_WAVES), 0, st, a);
    else hipLaunchKernelGGL((tree_attn16_kernel<BF, HD, 4>), grid, dim3(64 * TREE_WAVES), 0, st, a);
    constexpr int DT = BF ? SSD_BF16 : SSD_F16, ROWS = 256 / (HD / 4);
    if (a.n_joins)
        hipLaunchKernelGGL((tree_join_kernel<DT, HD>), dim3(a.n_joins, a.n_kv_heads, (a.tile_rows + ROWS - 1) / ROWS), dim3(256), 0, st, a, a.tile_rows, BIAS<BF>);
}

template <int DT>
static void launch(const TreeAttnArgs& a, hipStream_t st) {
    if constexpr (DT == SSD_F32) hipLaunchKernelGGL((tree_attn_kernel<DT>), dim3(a.n_items, a.n_kv_heads), dim3(256), 0, st, a);
    else if (a.head_dim == 64) launch16<DT == SSD_BF16, 64>(a, st);
    else launch16<DT == SSD_BF16, 128>(a, st);
    if (a.mass) hipLaunchKernelGGL((tree_mass_kernel<DT>), dim3(a.n_mass_items, a.n_kv_heads), dim3(256), 0, st, a);
}

void launch_tree_attention(const TreeAttnArgs& a, hipStream_t st) {
    if (a.dtype == SSD_F32) launch<SSD_F32>(a, st);
    else if (a.dtype == SSD_BF16) launch<SSD_BF16>(a, st);
    else launch<SSD_F16>(a, st);
}

}  // namespace ssd
