// The same for fp32 caches, head_dim a multiple of 4 up to 128, on v_mfma_f32_16x16x4_f32 (fp32 products and sums): the layout of tree_attn.hip with
// 16-key blocks.  A lane's four dims 16 c + 4 g .. of a key row are its elements of four products, in the same order for the queries; a
// lane's scores of keys 4 g .. 4 g + 3 are its elements of the second product, key r of every group in product r.  Products and sums are
// fp32 throughout, and every larger score raises the maximum: weights are at most 1, and rows whose sums leave the range are taken again with smaller ones.  Only the shape that splits the keys, with 16 or 32 rows: the fp32 models are small.  20 rows
// over 70, 4 heads of 64, 4 utterances: 8.1 us (eight wavefronts were 0.7 slower), the launch and the chain words, keys, values, merge.
#include "tree_attn.h"

namespace ssd {

constexpr int TREE32_KEYS = 16;

__device__ __forceinline__ f32x4_t mfma_16x16x4(float a, float b, const f32x4_t& c) { return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0); }

// Rows of a block in operand registers: row lane % 16, dims 16 c + 4 (lane / 16) ..; dims from head_dim on are zero.
template <int HD>
__device__ __forceinline__ void load_rows32(f32x4_t (&x)[HD / 16], const float* row, int head_dim, int kg) {
#pragma unroll
    for (int c = 0; c < HD / 16; ++c) {
        const int d = 16 * c + 4 * kg;
        const f32x4_t v = *reinterpret_cast<const f32x4_t*>(row + (d < head_dim ? d : 0));
        x[c] = d < head_dim ? v : (f32x4_t){0.f, 0.f, 0.f, 0.f};
    }
}

template <int HD, int NT, class M>
__global__ void __launch_bounds__(64 * KEY_WAVES, 2) tree_attn32_kernel(TreeAttnArgs a, M w) {
    constexpr int ROW = HD * 4, BLOCK = TREE32_KEYS * ROW, STEP = TREE32_KEYS * KEY_WAVES, DT = HD / 16, TR = 16 * NT;
    constexpr int ROW_CHUNKS = ROW / 16, V_ROWS = 64 / ROW_CHUNKS, V_LOADS = TREE32_KEYS / V_ROWS;
    __shared__ __align__(1024) unsigned char v_s[KEY_WAVES][BLOCK];
    __shared__ float2 ml_s[KEY_WAVES * TR];
    __shared__ uint32_t span_s[SPANS];
    const int lane = threadIdx.x % 64, kg = lane / 16, dc = lane % 16;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const Work t = item_of(a, w, blockIdx.y, TR);
    const int kvh = blockIdx.x, hd = a.head_dim;
    const int R = t.n_nodes * a.group;
    const int last = max(t.k0, t.k1 - 1);                    // (a range without keys: any row)
    const int n_spans = t.k1 > t.n_ctx ? t.n_nodes : 0;
    if (n_spans) store_spans<64 * KEY_WAVES>(span_s, a, w, t, (int)threadIdx.x < n_spans ? w(a.spans + t.node0 + (int)threadIdx.x) : 0u);
    const int64_t first = (int64_t)t.slot0 * a.slot_stride + kvh * a.head_stride;
    const float* kbase = (const float*)a.k + first;
    const float* vbase = (const float*)a.v + first;
    f32x4_t kr[DT];
    auto load_keys = [&](int k0) { load_rows32<HD>(kr, kbase + (int64_t)min(k0 + dc, last) * a.slot_stride, hd, kg); };
    // values: the 16-byte chunks of row r permuted by r / 4, so that the four rows of a read lie in different banks; dims from head_dim on
    // hold copies of the first ones (their outputs are not stored)
    auto load_values = [&](int k0) {
        const int r0 = min(k0, last), beyond = last - r0;
        const __amdgpu_buffer_rsrc_t rsrc = make_rsrc(vbase + (int64_t)r0 * a.slot_stride);
#pragma unroll
        for (int i = 0; i < V_LOADS; ++i) {
            const int row = V_ROWS * i + lane / ROW_CHUNKS, chunk = (lane % ROW_CHUNKS) ^ (row / 4 % 4 * 4);
            const int off = min(row, beyond) * (int)a.slot_stride * 4 + (chunk * 4 < hd ? chunk * 16 : 0);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (lds_void_t*)(v_s[wave] + i * 1024), 16, off, 0, 0, 0);
        }
    };
    const int k_first = t.k0 + wave * TREE32_KEYS;
    load_keys(k_first);
    f32x4_t qf[NT][DT];
    const float sign = a.scale < 0.f ? -1.f : a.scale == 0.f ? 0.f : 1.f;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int row = min(t.row0 + 16 * n + dc, R - 1);
        load_rows32<HD>(qf[n], (const float*)a.q + query_at(a, t, kvh, row, hd), hd, kg);
#pragma unroll
        for (int c = 0; c < DT; ++c) qf[n][c] *= sign;
    }
    const float sc = scale_of(a);
    float m[NT], l[NT], down[NT] = {};
    f32x4_t o[NT][DT];
    __syncthreads();
    load_values(k_first);
    const float* vr = reinterpret_cast<const float*>(v_s[wave]);
    for (int turn = 1;; ++turn) {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            m[n] = -F32_MOST;
            l[n] = 0.f;
#pragma unroll
            for (int i = 0; i < DT; ++i) o[n][i] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
        }
        for (int k0 = k_first; k0 < t.k1; k0 += STEP) {
            f32x4_t s[NT];
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                s[n] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int c = 0; c < DT; ++c)
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[n] = mfma_16x16x4(kr[c][e], qf[n][c][e], s[n]);
            }
            const bool masked = k0 + TREE32_KEYS > min(t.n_ctx, t.k1);
            if (masked) {
                uint32_t key[1][4];
                key_spans<1>(key, t, k0, span_s);
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    const uint32_t mine = span_s[SPANS_BEFORE + node_of(a, min(t.row0 + 16 * n + dc, R - 1))];
#pragma unroll
                    for (int r = 0; r < 4; ++r) s[n][r] = sees(mine, key[0][r]) ? s[n][r] : -INFINITY;
                }
            }
            bool above = false;
            float mx[NT];
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                mx[n] = fmaxf(fmaxf(s[n][0], s[n][1]), fmaxf(s[n][2], s[n][3]));
                above |= mx[n] > m[n];
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
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const float base = fminf(-down[n] - m[n] * sc, F32_MOST);
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    s[n][r] = __builtin_amdgcn_exp2f(fmaf(s[n][r], sc, base));
                    l[n] += s[n][r];
                }
            }
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_waitcnt(0x0F70);
            __builtin_amdgcn_sched_barrier(0);
            load_keys(k0 + STEP);
            // A value that is not finite would reach the rows that do not see it as 0 times infinity: as in tree_attn.hip, the products run on the
            // others, and two more count the infinities of either sign (a NaN as both) that rows with a probability meet.
#pragma unroll
            for (int i = 0; i < DT; ++i) {
                float v[4];
                bool odd = false;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    v[r] = vr[(4 * kg + r) * HD + ((16 * i + dc) ^ (kg * 16))];
                    odd |= !(fabsf(v[r]) <= F32_MOST);
                }
                if ((masked || turn > 1) && __any(odd)) {
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        f32x4_t up = {0.f, 0.f, 0.f, 0.f}, below = up;
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            const float there = s[n][r] > 0.f || s[n][r] != s[n][r] ? 1.f : 0.f;
                            up = mfma_16x16x4(!(v[r] <= F32_MOST) ? 1.f : 0.f, there, up);
                            below = mfma_16x16x4(!(v[r] >= -F32_MOST) ? 1.f : 0.f, there, below);
                        }
#pragma unroll
                        for (int r = 0; r < 4; ++r) o[n][i][r] += (up[r] > 0.f ? INFINITY : 0.f) - (below[r] > 0.f ? INFINITY : 0.f);
                    }
#pragma unroll
                    for (int r = 0; r < 4; ++r) v[r] = fabsf(v[r]) <= F32_MOST ? v[r] : 0.f;
                }
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int r = 0; r < 4; ++r) o[n][i] = mfma_16x16x4(v[r], s[n][r], o[n][i]);
            }
            __builtin_amdgcn_s_waitcnt(0xC07F);                  // the reads of this block are done
            __builtin_amdgcn_sched_barrier(0);
            load_values(k0 + STEP);
        }
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_waitcnt(0x0F70);                      // the values behind the last block: they land where the output goes
        __builtin_amdgcn_sched_barrier(0);
        bool odd[NT];
        if (turn == 2 || !not_finite(o, odd)) break;
#pragma unroll
        for (int n = 0; n < NT; ++n) down[n] = odd[n] ? DOWN : 0.f;
        load_keys(k_first);
        load_values(k_first);
    }
    merge_wavefronts<SSD_F32, HD, NT, KEY_WAVES>(a, t, kvh, m, l, o, down, sc, 0.f, reinterpret_cast<float*>(v_s), ml_s);
}

constexpr int MASS32_ROWS = 64;

template <int HD, class M>
__global__ void __launch_bounds__(64 * MASS_WAVES, 2) tree_mass32_kernel(TreeAttnArgs a, M w) {
    constexpr int STEP = TREE32_KEYS * MASS_WAVES, DT = HD / 16, CHUNKS = HD / 4;
    __shared__ __align__(1024) float q_s[MASS32_ROWS * HD];
    __shared__ float lse_s[MASS32_ROWS];
    __shared__ uint32_t row_span[MASS32_ROWS], span_s[SPANS];
    const int lane = threadIdx.x % 64, kg = lane / 16, dc = lane % 16;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const Work t = mass_item_of(a, w, blockIdx.y);
    const int kvh = blockIdx.x, hd = a.head_dim;
    const int R = t.n_nodes * a.group, last = t.k1 - 1;
    const float* kbase = (const float*)a.k + (int64_t)t.slot0 * a.slot_stride + kvh * a.head_stride;
    f32x4_t kr[DT];
    auto load_keys = [&](int k0) { load_rows32<HD>(kr, kbase + (int64_t)min(k0 + dc, last) * a.slot_stride, hd, kg); };
    const int first = t.k0 + wave * TREE32_KEYS;
    load_keys(first);
    if (t.k1 > t.n_ctx) store_spans<64 * MASS_WAVES>(span_s, a, w, t, (int)threadIdx.x < t.n_nodes ? w(a.spans + t.node0 + (int)threadIdx.x) : 0u);
    const float sc = scale_of(a), sign = a.scale < 0.f ? -1.f : a.scale == 0.f ? 0.f : 1.f;
    for (int r0 = 0; r0 < R; r0 += MASS32_ROWS) {
        const int rows = min(MASS32_ROWS, R - r0), tiles = (rows + 15) / 16;
        if (r0) __syncthreads();
        for (int i = threadIdx.x; i < tiles * 16 * CHUNKS; i += 64 * MASS_WAVES) {
            const int r = i / CHUNKS, c = i % CHUNKS, row = min(r0 + r, R - 1);
            f32x4_t x = {0.f, 0.f, 0.f, 0.f};
            if (c * 4 < hd) x = *reinterpret_cast<const f32x4_t*>((const float*)a.q + query_at(a, t, kvh, row, hd) + c * 4);
            *reinterpret_cast<f32x4_t*>(q_s + r * HD + (c ^ (r & 15)) * 4) = x * sign;
        }
        for (int r = threadIdx.x; r < tiles * 16; r += 64 * MASS_WAVES) {
            const int row = min(r0 + r, R - 1);
            lse_s[r] = r < rows ? a.lse[row_at(a, t, kvh, row)] * -LOG2E : -INFINITY;   // (rows behind the last: no weight)
            row_span[r] = r < rows ? w(a.spans + t.node0 + node_of(a, row)) : 0xffffu;
        }
        __syncthreads();
        if (r0) load_keys(first);
        for (int k0 = first; k0 < t.k1; k0 += STEP) {
            f32x4_t acc[1] = {(f32x4_t){0.f, 0.f, 0.f, 0.f}};
            const bool masked = k0 + TREE32_KEYS > t.n_ctx;
            uint32_t key[1][4];
            if (masked) key_spans<1>(key, t, k0, span_s);
            for (int n = 0; n < tiles; ++n) {
                const int r = 16 * n + dc;
                f32x4_t s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int c = 0; c < DT; ++c) {
                    const f32x4_t q = *reinterpret_cast<const f32x4_t*>(q_s + r * HD + ((4 * c + kg) ^ (r & 15)) * 4);
#pragma unroll
                    for (int e = 0; e < 4; ++e) s = mfma_16x16x4(kr[c][e], q[e], s);
                }
                const float base = lse_s[r];
                const uint32_t mine = row_span[r];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float p = __builtin_amdgcn_exp2f(fmaf(s[e], sc, base));
                    acc[0][e] += masked && !sees(mine, key[0][e]) ? 0.f : p;
                }
            }
            load_keys(k0 + STEP);
            add_mass(a, t, kvh, k0, r0 == 0, acc);
        }
    }
}

template <int HD, class M>
static void launch32(const TreeAttnArgs& a, const M& w, hipStream_t st) {
    const dim3 grid(a.n_kv_heads, a.n_items);
    if (a.tile_rows == 16) hipLaunchKernelGGL((tree_attn32_kernel<HD, 1, M>), grid, dim3(64 * KEY_WAVES), 0, st, a, w);
    else hipLaunchKernelGGL((tree_attn32_kernel<HD, 2, M>), grid, dim3(64 * KEY_WAVES), 0, st, a, w);
    if (a.n_joins) hipLaunchKernelGGL((tree_join_kernel<SSD_F32, HD, M>), dim3(a.n_joins * a.tile_rows, a.n_kv_heads), dim3(256), 0, st, a, w, 0.f);
    if (a.mass) hipLaunchKernelGGL((tree_mass32_kernel<HD, M>), dim3(a.n_kv_heads, a.n_mass), dim3(64 * MASS_WAVES), 0, st, a, w);
}

template <class M>
void launch_tree_attention32(const TreeAttnArgs& a, const M& w, hipStream_t st) {
    if (a.head_dim <= 64) launch32<64>(a, w, st);
    else launch32<128>(a, w, st);
}
template void launch_tree_attention32(const TreeAttnArgs&, const MetaWords&, hipStream_t);
template void launch_tree_attention32(const TreeAttnArgs&, const MetaArray&, hipStream_t);

}  // namespace ssd
