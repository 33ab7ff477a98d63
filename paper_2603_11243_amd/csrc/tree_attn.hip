// Attention of the nodes of drafted trees over cached rows (Sec. 2.2 for more than one continuation).  Node i sees the rows of its
// context, its ancestors and itself; node j is i or an ancestor of i exactly if i's place in depth-first order lies in the span of j's
// subtree, so that two integers a node are the mask of a tree of any shape.
//   s_ij = scale q_i . k_j,  lse_i = log sum_j exp s_ij,  o_i = sum_j exp(s_ij - lse_i) v_j
// and the weight that row j collects: sum over the nodes and the heads of the K/V head's group of exp(s_ij - lse_i).
#include "tree_attn.h"

namespace ssd {

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
    __shared__ __align__(1024) unsigned char v_s[TREE_WAVES][BLOCK];
    __shared__ float2 ml_s[TREE_WAVES * TR];
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
            const float base = fminf(BIAS<BF> - m[n] * sc, F32_MOST);    // (finite: a score may be -infinity)
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

    merge_wavefronts<BF ? SSD_BF16 : SSD_F16, HD, NT>(a, t, kvh, m, l, o, sc, BIAS<BF>, reinterpret_cast<float*>(v_s), ml_s);
}

// The weight of every row: the scores once more, now that the log-sum-exps are known.  A workgroup owns a range of keys of a K/V head, a wavefront
// 32-key blocks of it, in operand registers; MASS_ROWS query rows at a time lie in LDS, their 16-byte chunks permuted so that the 16 rows of an operand
// read spread over all banks.
constexpr int MASS_ROWS = 128;

template <bool BF, int HD>
__global__ void __launch_bounds__(64 * TREE_WAVES, 2) tree_mass16_kernel(TreeAttnArgs a) {
    constexpr int ROW = HD * 2, STEP = TREE_KEYS * TREE_WAVES, KS = HD / 32, CHUNKS = ROW / 16;
    __shared__ __align__(1024) unsigned char q_s[MASS_ROWS * ROW];
    __shared__ float lse_s[MASS_ROWS];
    __shared__ uint32_t row_span[MASS_ROWS], span_s[MAX_TREE_NODES];
    const int lane = threadIdx.x % 64, kg = lane / 16, dc = lane % 16;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int work = xcd_contiguous_index(blockIdx.x, gridDim.x);
    const TreeItem t = a.mass_items[work / a.n_kv_heads];
    const int kvh = work % a.n_kv_heads;
    const int G = a.n_q_heads / a.n_kv_heads, R = t.n_nodes * G, last = t.k1 - 1;
    const int stride2 = (int)a.slot_stride * 2;
    const uint16_t* kbase = (const uint16_t*)a.k + (int64_t)t.slot0 * a.slot_stride + kvh * a.head_stride;
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
    const int first = t.k0 + wave * TREE_KEYS;
    load_keys(first);
    if (t.k1 > t.n_ctx)
        for (int i = threadIdx.x; i < t.n_nodes; i += 64 * TREE_WAVES) span_s[i] = a.spans[t.node0 + i];
    auto swizzle = [](int row) { return HD == 128 ? row & 15 : row >> 1 & 7; };
    const float sc = fabsf(a.scale) * LOG2E;
    const uint32_t flip = a.scale < 0.f ? 0x80008000u : 0u;
    for (int r0 = 0; r0 < R; r0 += MASS_ROWS) {
        const int rows = min(MASS_ROWS, R - r0), tiles = (rows + 15) / 16;
        if (r0) __syncthreads();
        for (int i = threadIdx.x; i < tiles * 16 * CHUNKS; i += 64 * TREE_WAVES) {
            const int r = i / CHUNKS, c = i % CHUNKS, row = min(r0 + r, R - 1);
            uint4 w = *reinterpret_cast<const uint4*>((const uint16_t*)a.q + (int64_t)(t.node0 + row / G) * a.q_stride + (kvh * G + row % G) * HD + c * 8);
            w.x ^= flip; w.y ^= flip; w.z ^= flip; w.w ^= flip;
            *reinterpret_cast<uint4*>(q_s + r * ROW + (c ^ swizzle(r)) * 16) = w;
        }
        for (int r = threadIdx.x; r < tiles * 16; r += 64 * TREE_WAVES) {
            const int row = min(r0 + r, R - 1);
            lse_s[r] = r < rows ? a.lse[(int64_t)(t.node0 + row / G) * a.n_q_heads + kvh * G + row % G] * -LOG2E : -INFINITY;   // (rows behind the last: no weight)
            row_span[r] = r < rows ? a.spans[t.node0 + row / G] : 0xffffu;
        }
        __syncthreads();
        if (r0) load_keys(first);
        for (int k0 = first; k0 < t.k1; k0 += STEP) {
            f32x4_t acc[2];
#pragma unroll
            for (int c = 0; c < 2; ++c) acc[c] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
            const bool masked = k0 + TREE_KEYS > t.n_ctx;
            uint32_t key[2][4];
            if (masked)
#pragma unroll
                for (int c = 0; c < 2; ++c)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const int at = k0 + 16 * c + 4 * kg + r;
                        key[c][r] = at < t.n_ctx ? 0xffff0000u : at < t.k1 ? span_s[at - t.n_ctx] : 0u;
                    }
            for (int n = 0; n < tiles; ++n) {
                const int r = 16 * n + dc;
                f32x4_t s[2];
#pragma unroll
                for (int c = 0; c < 2; ++c) s[c] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int e = 0; e < KS; ++e) {
                    const f16x8_t q = as_f16x8(*reinterpret_cast<const uint4*>(q_s + r * ROW + ((kg + 4 * e) ^ swizzle(r)) * 16));
#pragma unroll
                    for (int c = 0; c < 2; ++c) s[c] = mfma_16x16x32<BF>(__builtin_bit_cast(f16x8_t, kr[c][e]), q, s[c]);
                }
                const float base = lse_s[r];
                const uint32_t mine = row_span[r];
#pragma unroll
                for (int c = 0; c < 2; ++c)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float p = __builtin_amdgcn_exp2f(fmaf(s[c][e], sc, base));
                        acc[c][e] += masked && !sees(mine, key[c][e]) ? 0.f : p;
                    }
            }
            load_keys(k0 + STEP);
            add_mass(a, t, kvh, k0, r0 == 0, acc);
        }
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
    if (a.mass) hipLaunchKernelGGL((tree_mass16_kernel<BF, HD>), dim3(a.n_mass_items * a.n_kv_heads), dim3(64 * TREE_WAVES), 0, st, a);
}

void launch_tree_attention(const TreeAttnArgs& a, hipStream_t st) {
    if (a.dtype == SSD_F32) launch_tree_attention32(a, st);
    else if (a.head_dim == 64) a.dtype == SSD_BF16 ? launch16<true, 64>(a, st) : launch16<false, 64>(a, st);
    else a.dtype == SSD_BF16 ? launch16<true, 128>(a, st) : launch16<false, 128>(a, st);
}

}  // namespace ssd
