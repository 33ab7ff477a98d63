// Attention of the nodes of drafted trees over cached rows (Sec. 2.2 for more than one continuation).  Node i sees the rows of its
// context, its ancestors and itself; node j is i or an ancestor of i exactly if i's place in depth-first order lies in the span of j's
// subtree, so that two integers a node are the mask of a tree of any shape.
//   s_ij = scale q_i . k_j,  lse_i = log sum_j exp s_ij,  o_i = sum_j exp(s_ij - lse_i) v_j
// and the weight that row j collects: sum over the nodes and the heads of the K/V head's group of exp(s_ij - lse_i).
#include <string.h>

#include "tree_attn.h"

namespace ssd {

// ---- 16-bit caches ----------------------------------------------------------------------------------------------------------------
// Both products are v_mfma_f32_16x16x32: S^T = K Q^T, then O^T += V^T P^T with the values in LDS (global -> LDS loads, read back through the
// transposing ds_read_b64_tr_b16): keys 4g .. 4g + 3 and 16 + 4g .. of 32 are the scores of lane group g and its operand of the second product alike.
// The maximum that the exponents refer to may lag behind the true one by 2^LAG: it is raised (and the output rescaled) only by a score
// beyond that, which spares nearly every block the exchange between lanes and the rescaling.  Probabilities enter the second product in
// two pieces of the cache's type, rounded and what the rounding left, where the output has one; their sum is of the fp32 ones.  bfloat16: 16 bits of each;
// it has the range of fp32, and they are at most 1.  IEEE half holds them times 2^BIAS (2^(BIAS + LAG) is in its range): 22 bits of those down to 2^-14 of the largest,
// and of smaller ones the bits down to 2^-36 of it, below what fp32 sums keep.  The second piece costs 3 to 5 % with up to 64 rows a K/V head, 8 % in 90 trees of 48 nodes
// over 220 rows (24 heads on 8: 70 -> 76 us) and 19 % where 120 rows share long contexts (200001 rows 174 -> 206), whose blocks wait for the matrix cores.
template <bool BF> constexpr float LAG = BF ? 8.f : 4.f;
template <bool BF> constexpr float BIAS = BF ? -LAG<BF> : 11.f;

// Passes at most: as it is; with care for values that are not finite; of bfloat16 with smaller weights in rows that are not finite still.
template <bool BF> constexpr int TURNS = BF ? 3 : 2;

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

// Weights in the operand type: rounded ones and the rest of each.
struct Weights { f16x8_t top, rest; };

// Scores of 32 keys to weights; maxima, sums and outputs follow.
template <bool BF, int NT, int DT>
__device__ __forceinline__ void weights_of(f32x4_t (&s)[NT][2], float (&m)[NT], float (&l)[NT], f32x4_t (&o)[NT][DT], float sc, const float (&down)[NT], Weights (&p)[NT]) {
    float mx[NT];
    bool above = false;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        mx[n] = -INFINITY;
#pragma unroll
        for (int c = 0; c < 2; ++c) mx[n] = fmaxf(mx[n], fmaxf(fmaxf(s[n][c][0], s[n][c][1]), fmaxf(s[n][c][2], s[n][c][3])));
        above |= (mx[n] - m[n]) * sc > LAG<BF>;
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
        const float base = fminf(BIAS<BF> - down[n] - m[n] * sc, F32_MOST);    // (finite: a score may be -infinity)
        uint32_t pw[4], rw[4];
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            f32x4_t& x = s[n][c];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                x[r] = __builtin_amdgcn_exp2f(fmaf(x[r], sc, base));
                l[n] += x[r];
            }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                pw[2 * c + e] = pack16<BF>(x[2 * e], x[2 * e + 1]);
                rw[2 * c + e] = rest16<BF>(x[2 * e], x[2 * e + 1], pw[2 * c + e]);
            }
        }
        p[n].top = as_f16x8(make_uint4(pw[0], pw[1], pw[2], pw[3]));
        p[n].rest = as_f16x8(make_uint4(rw[0], rw[1], rw[2], rw[3]));
    }
}

// Place of the 16-byte chunks of value row `row` in LDS: the 32-byte pieces that half a wavefront reads lie in all banks.
template <int HD> __device__ __forceinline__ int v_swizzle(int row) { return HD == 128 ? 4 * (row & 3) + 2 * (row >> 2 & 1) : 2 * (row >> 1 & 3); }

// The same for key and query rows, of which an operand read takes the same chunk of 16.
template <int HD> __device__ __forceinline__ int k_swizzle(int row) { return HD == 128 ? row & 15 : row >> 1 & 7; }

// The operands of 32 key rows at k: rows 16 c + lane % 16, dims 8 (lane / 16) + 32 e.  Written out because the compiler waits for all loads into LDS
// before a plain read of it, those of the next block among them, which go elsewhere.
template <int HD>
__device__ __forceinline__ void read_keys(const unsigned char* k, f16x8_t (&kf)[2][HD / 32]) {
    const int kg = threadIdx.x % 64 / 16, dc = threadIdx.x % 16;
    const uint32_t base = (uint32_t)(uintptr_t)(lds_void_t*)k + dc * HD * 2;
    const uint32_t a0 = base + (kg ^ k_swizzle<HD>(dc)) * 16, a1 = base + ((kg + 4) ^ k_swizzle<HD>(dc)) * 16;
    u32x4_t x[2][HD / 32];
    if constexpr (HD == 128) {
        const uint32_t a2 = base + ((kg + 8) ^ k_swizzle<HD>(dc)) * 16, a3 = base + ((kg + 12) ^ k_swizzle<HD>(dc)) * 16;
        asm volatile("ds_read_b128 %0, %8\n\tds_read_b128 %1, %9\n\tds_read_b128 %2, %10\n\tds_read_b128 %3, %11\n\t"
                     "ds_read_b128 %4, %8 offset:4096\n\tds_read_b128 %5, %9 offset:4096\n\tds_read_b128 %6, %10 offset:4096\n\tds_read_b128 %7, %11 offset:4096\n\t"
                     "s_waitcnt lgkmcnt(0)"
                     : "=&v"(x[0][0]), "=&v"(x[0][1]), "=&v"(x[0][2]), "=&v"(x[0][3]), "=&v"(x[1][0]), "=&v"(x[1][1]), "=&v"(x[1][2]), "=&v"(x[1][3])
                     : "v"(a0), "v"(a1), "v"(a2), "v"(a3) : "memory");
    } else {
        asm volatile("ds_read_b128 %0, %4\n\tds_read_b128 %1, %5\n\tds_read_b128 %2, %4 offset:2048\n\tds_read_b128 %3, %5 offset:2048\n\t"
                     "s_waitcnt lgkmcnt(0)"
                     : "=&v"(x[0][0]), "=&v"(x[0][1]), "=&v"(x[1][0]), "=&v"(x[1][1]) : "v"(a0), "v"(a1) : "memory");
    }
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int e = 0; e < HD / 32; ++e) kf[c][e] = __builtin_bit_cast(f16x8_t, x[c][e]);
}

template <int NT, int DT>
__device__ __forceinline__ void start(float (&m)[NT], float (&l)[NT], f32x4_t (&o)[NT][DT]) {
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        m[n] = -F32_MOST;
        l[n] = 0.f;
#pragma unroll
        for (int i = 0; i < DT; ++i) o[n][i] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
    }
}

// O^T += V^T P^T over the 32 value rows at v, four 16-dim tiles at a time (read as in read_keys, for the same reason).  Transposing read: lane i of 16 passes row i / 4 and dims 4 (i % 4) .. + 3 of a
// 16-dim tile, lane j receives dim j of four rows.
template <bool BF, int HD, int NT, bool MASKED>
__device__ __forceinline__ void add_values(const unsigned char* v, const Weights (&p)[NT], f32x4_t (&o)[NT][HD / 16], bool careful) {
    constexpr int ROW = HD * 2;
    const int lane = threadIdx.x % 64, kg = lane / 16, dc = lane % 16;
    const int v_row = 4 * kg + dc / 4, v_low = (dc % 4) / 2;
    const uint32_t base = (uint32_t)(uintptr_t)(lds_void_t*)v + v_row * ROW + (dc % 2) * 8;
#pragma unroll
    for (int g = 0; g < HD / 16; g += 4) {
        u32x2_t vf[4][2];
        uint32_t at[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) at[i] = base + (((2 * (g + i)) | v_low) ^ v_swizzle<HD>(v_row)) * 16;
        if constexpr (HD == 128)
            asm volatile("ds_read_b64_tr_b16 %0, %8\n\tds_read_b64_tr_b16 %1, %8 offset:4096\n\tds_read_b64_tr_b16 %2, %9\n\tds_read_b64_tr_b16 %3, %9 offset:4096\n\t"
                         "ds_read_b64_tr_b16 %4, %10\n\tds_read_b64_tr_b16 %5, %10 offset:4096\n\tds_read_b64_tr_b16 %6, %11\n\tds_read_b64_tr_b16 %7, %11 offset:4096\n\t"
                         "s_waitcnt lgkmcnt(0)"
                         : "=&v"(vf[0][0]), "=&v"(vf[0][1]), "=&v"(vf[1][0]), "=&v"(vf[1][1]), "=&v"(vf[2][0]), "=&v"(vf[2][1]), "=&v"(vf[3][0]), "=&v"(vf[3][1])
                         : "v"(at[0]), "v"(at[1]), "v"(at[2]), "v"(at[3]) : "memory");
        else
            asm volatile("ds_read_b64_tr_b16 %0, %8\n\tds_read_b64_tr_b16 %1, %8 offset:2048\n\tds_read_b64_tr_b16 %2, %9\n\tds_read_b64_tr_b16 %3, %9 offset:2048\n\t"
                         "ds_read_b64_tr_b16 %4, %10\n\tds_read_b64_tr_b16 %5, %10 offset:2048\n\tds_read_b64_tr_b16 %6, %11\n\tds_read_b64_tr_b16 %7, %11 offset:2048\n\t"
                         "s_waitcnt lgkmcnt(0)"
                         : "=&v"(vf[0][0]), "=&v"(vf[0][1]), "=&v"(vf[1][0]), "=&v"(vf[1][1]), "=&v"(vf[2][0]), "=&v"(vf[2][1]), "=&v"(vf[3][0]), "=&v"(vf[3][1])
                         : "v"(at[0]), "v"(at[1]), "v"(at[2]), "v"(at[3]) : "memory");
        // A value that is not finite reaches the rows that do not see it as 0 times infinity, and those that see it as the sum of its products with both pieces of
        // a probability: a NaN that stays.  A pass whose output is not finite is repeated with care: where a block holds such values the products run on the
        // others, and two more count the infinities of either sign (a NaN as both) that rows with a probability meet.
        uint32_t odd = 0;
        if (MASKED && careful) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int e = 0; e < 2; ++e) odd |= beyond_of<BF>(vf[i][e].x) | beyond_of<BF>(vf[i][e].y);
        }
        if (MASKED && careful && __any(odd & SIGNS)) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                __builtin_amdgcn_sched_barrier(0);           // (one after the other: registers, not speed)
                const u32x2_t x = vf[i][0], y = vf[i][1];
                const f16x8_t up = as_f16x8(make_uint4(infinite_of<BF>(x.x, 0), infinite_of<BF>(x.y, 0), infinite_of<BF>(y.x, 0), infinite_of<BF>(y.y, 0)));
                const f16x8_t down = as_f16x8(make_uint4(infinite_of<BF>(x.x, ~0u), infinite_of<BF>(x.y, ~0u), infinite_of<BF>(y.x, ~0u), infinite_of<BF>(y.y, ~0u)));
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    const uint4 t = __builtin_bit_cast(uint4, p[n].top), e = __builtin_bit_cast(uint4, p[n].rest);
                    const f16x8_t there = as_f16x8(make_uint4(one_where<BF>(not_zero(t.x) | not_zero(e.x)), one_where<BF>(not_zero(t.y) | not_zero(e.y)),
                                                              one_where<BF>(not_zero(t.z) | not_zero(e.z)), one_where<BF>(not_zero(t.w) | not_zero(e.w))));
                    const f32x4_t zero = {0.f, 0.f, 0.f, 0.f}, u = mfma_16x16x32<BF>(up, there, zero), d = mfma_16x16x32<BF>(down, there, zero);
#pragma unroll
                    for (int r = 0; r < 4; ++r) o[n][g + i][r] += (u[r] > 0.f ? INFINITY : 0.f) - (d[r] > 0.f ? INFINITY : 0.f);
                }
                vf[i][0] = (u32x2_t){finite_of<BF>(x.x), finite_of<BF>(x.y)};
                vf[i][1] = (u32x2_t){finite_of<BF>(y.x), finite_of<BF>(y.y)};
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const f16x8_t x = __builtin_bit_cast(f16x8_t, __builtin_shufflevector(vf[i][0], vf[i][1], 0, 1, 2, 3));
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                o[n][g + i] = mfma_16x16x32<BF>(x, p[n].top, o[n][g + i]);
                o[n][g + i] = mfma_16x16x32<BF>(x, p[n].rest, o[n][g + i]);
            }
        }
    }
}

// Queries as operands: column lane % 16 of tile n is query row row0 + 16 n + lane % 16 (a copy of the last one behind it); a negative scale is theirs.
template <int HD, int NT>
__device__ __forceinline__ void load_queries(f16x8_t (&qf)[NT][HD / 32], const TreeAttnArgs& a, const Work& t, int kvh, int row0) {
    const int lane = threadIdx.x % 64;
    const uint32_t flip = a.scale < 0.f ? 0x80008000u : 0u, keep = a.scale == 0.f ? 0u : ~0u;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int row = min(row0 + 16 * n + lane % 16, t.n_nodes * a.group - 1);
        const uint16_t* q = (const uint16_t*)a.q + query_at(a, t, kvh, row, HD) + lane / 16 * 8;
#pragma unroll
        for (int s = 0; s < HD / 32; ++s) {
            uint4 x = *reinterpret_cast<const uint4*>(q + 32 * s);
            x.x = (x.x ^ flip) & keep; x.y = (x.y ^ flip) & keep; x.z = (x.z ^ flip) & keep; x.w = (x.w ^ flip) & keep;
            qf[n][s] = as_f16x8(x);
        }
    }
}

// What all wavefronts have stored to LDS, and with it what they loaded straight into it and have waited for; a barrier with a fence would wait for
// every load in flight.
__device__ __forceinline__ void lds_barrier() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0xC07F);
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// ---- few query rows: 16 of a K/V head a workgroup, whose wavefronts take the 32-key blocks of the range in turn, so that every cached row is read once,
// and merge their (maximum, sum, output) through LDS.  Key rows come straight from memory in operand registers; a wavefront's values are its own
// and need no barrier.  One token over 106 rows, 16 heads on 8: 4.5 us in a graph, the launch and three ways to memory and back one behind the other (words, keys
// and queries, values); the kernel below, in which one wavefront has all 16 rows, takes 6.0, over 200000 rows 161 in place of 164 and for 38 utterances of 150 rows
// 7.9 in place of 8.5.
template <bool BF, int HD, class M>
__global__ void __launch_bounds__(64 * KEY_WAVES, 2) tree_keys16_kernel(TreeAttnArgs a, M w) {
    constexpr int NT = 1, KEYS = 32, ROW = HD * 2, BLOCK = KEYS * ROW, STEP = KEYS * KEY_WAVES;
    constexpr int KS = HD / 32, DT = HD / 16, TR = 16 * NT;
    constexpr int ROW_CHUNKS = ROW / 16, V_ROWS = 64 / ROW_CHUNKS, V_LOADS = KEYS / V_ROWS, K_LOADS = 2 * KS;
    __shared__ __align__(1024) unsigned char v_s[KEY_WAVES][BLOCK];
    __shared__ float2 ml_s[KEY_WAVES * TR];
    __shared__ uint32_t span_s[SPANS];
    const int lane = threadIdx.x % 64, kg = lane / 16, dc = lane % 16;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const Work t = item_of(a, w, blockIdx.y, TR);
    const int kvh = blockIdx.x;
    const int R = t.n_nodes * a.group;
    const int last = max(t.k0, t.k1 - 1);                    // (a range without keys: any row)
    const uint32_t span = (int)threadIdx.x < t.n_nodes ? w(a.spans + t.node0 + (int)threadIdx.x) : 0u;
    const int stride2 = (int)a.slot_stride * 2;
    const int64_t first = (int64_t)t.slot0 * a.slot_stride + kvh * a.head_stride;
    const uint16_t* kbase = (const uint16_t*)a.k + first;
    const uint16_t* vbase = (const uint16_t*)a.v + first;

    // Keys k0 .. k0 + 31: lane (row dc of a half of 16, dims 8 kg + 32 s) in registers.  Values: rows of an instruction one behind the other.  Rows behind
    // the range are copies of its last one: masked, or of a block behind the wavefront's last, which is requested all the same.
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
    auto load_values = [&](int k0) {
        const int r0 = min(k0, last), beyond = last - r0;
        const __amdgpu_buffer_rsrc_t rsrc = make_rsrc(vbase + (int64_t)r0 * a.slot_stride);
#pragma unroll
        for (int i = 0; i < V_LOADS; ++i) {
            const int row = V_ROWS * i + lane / ROW_CHUNKS;
            const int off = min(row, beyond) * stride2 + ((lane % ROW_CHUNKS) ^ v_swizzle<HD>(row)) * 16;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (lds_void_t*)(v_s[wave] + i * 1024), 16, off, 0, 0, 0);
        }
    };
    const int k_first = t.k0 + wave * KEYS;
    load_keys(k_first);
    f16x8_t qf[NT][KS];
    load_queries<HD, NT>(qf, a, t, kvh, t.row0);
    load_values(k_first);
    const float sc = scale_of(a);
    float m[NT], l[NT], down[NT] = {};
    f32x4_t o[NT][DT];
    store_spans<64 * KEY_WAVES>(span_s, a, w, t, span);
    lds_barrier();
    uint32_t mine[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) mine[n] = span_s[SPANS_BEFORE + node_of(a, min(t.row0 + 16 * n + dc, R - 1))];
    bool careful = false;
    auto block = [&](auto masked_c, int k0) __attribute__((always_inline)) {
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
            uint32_t key[2][4];
            key_spans<2>(key, t, k0, span_s);
#pragma unroll
            for (int n = 0; n < NT; ++n) {
#pragma unroll
                for (int c = 0; c < 2; ++c)
#pragma unroll
                    for (int r = 0; r < 4; ++r) s[n][c][r] = sees(mine[n], key[c][r]) ? s[n][c][r] : -INFINITY;
            }
        }
        Weights p[NT];
        weights_of<BF, NT, DT>(s, m, l, o, sc, down, p);
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_waitcnt(0x0F70 | K_LOADS);        // the values of this block have landed (a wavefront reads its own only)
        __builtin_amdgcn_sched_barrier(0);
        add_values<BF, HD, NT, MASKED>(v_s[wave], p, o, careful);
        __builtin_amdgcn_s_waitcnt(0xC07F);                  // the reads of this block are done
        __builtin_amdgcn_sched_barrier(0);
        load_values(k0 + STEP);
    };
    for (int turn = 1;; ++turn) {
        start<NT, DT>(m, l, o);
        int k0 = k_first;
        if (!careful)
            for (; k0 + KEYS <= min(t.n_ctx, t.k1); k0 += STEP) block(std::false_type(), k0);
        for (; k0 < t.k1; k0 += STEP) block(std::true_type(), k0);
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_waitcnt(0x0F70);                  // the values behind the last block: they land where the output goes
        __builtin_amdgcn_sched_barrier(0);
        bool odd[NT];
        if (turn == TURNS<BF> || !not_finite(o, odd)) break;
        if (careful)
#pragma unroll
            for (int n = 0; n < NT; ++n) down[n] = odd[n] ? DOWN : 0.f;
        careful = true;
        load_keys(k_first);
        load_values(k_first);
    }
    merge_wavefronts<BF ? SSD_BF16 : SSD_F16, HD, NT, KEY_WAVES>(a, t, kvh, m, l, o, down, sc, BIAS<BF>, reinterpret_cast<float*>(v_s), ml_s);
}

// ---- many query rows: a wavefront has 16 NT of a K/V head for itself, the ROW_WAVES of a workgroup share 64-key blocks of keys and values in LDS, two of them
// in turn: the next one loads while this one is used.  Two workgroups a CU (LDS, and the registers of NT 2; NT 3 and 4 spill).
// 48 rows over 200001 and 32 to 66 over 20000 to 40000 cached ones, 8 K/V heads of 128: 160 and 94 us, 5.1 and 5.2 TB/s, what memory gives.  96 to 192 rows over 100 to 340,
// 90 utterances: 64 us, 2.5 TB/s; the vector ALU is 31 % busy, the matrix cores 17, LDS 2, and the rest is the few blocks of a workgroup one after
// the other, a barrier at each end.  With weights as one value (58 and 90 us) four workgroups a CU on 32-key blocks (NT 1) took 62 there and 104 over the long ones; all reads
// of a block's values at once, or two waits for them, the same.
constexpr int ROW_WAVES = 4;

template <bool BF, int HD, int NT, class M>
__global__ void __launch_bounds__(64 * ROW_WAVES, 2) tree_rows16_kernel(TreeAttnArgs a, M w) {
    constexpr int KEYS = 64, ROW = HD * 2, BLOCK = KEYS * ROW, KS = HD / 32, DT = HD / 16, TR = 16 * NT * ROW_WAVES;
    constexpr int CHUNKS = ROW / 16, L_ROWS = 64 / CHUNKS, LOADS = KEYS / L_ROWS / ROW_WAVES;
    __shared__ __align__(1024) unsigned char kv_s[2][2][BLOCK];
    __shared__ uint32_t span_s[SPANS];
    const int lane = threadIdx.x % 64, kg = lane / 16, dc = lane % 16;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const Work t = item_of(a, w, blockIdx.y, TR);
    const int kvh = blockIdx.x;
    const int R = t.n_nodes * a.group;
    const int last = max(t.k0, t.k1 - 1), row0 = t.row0 + wave * 16 * NT;
    const uint32_t span = (int)threadIdx.x < t.n_nodes ? w(a.spans + t.node0 + (int)threadIdx.x) : 0u;
    const int stride2 = (int)a.slot_stride * 2;
    const int64_t first = (int64_t)t.slot0 * a.slot_stride + kvh * a.head_stride;
    const uint16_t* kbase = (const uint16_t*)a.k + first;
    const uint16_t* vbase = (const uint16_t*)a.v + first;
    // Instruction i of a wavefront fills L_ROWS rows of the block.  Rows behind the range are copies of its last one.
    auto load = [&](int k0, int stage) __attribute__((always_inline)) {
        const int r0 = min(k0, last), beyond = last - r0;
        const __amdgpu_buffer_rsrc_t k_rsrc = make_rsrc(kbase + (int64_t)r0 * a.slot_stride), v_rsrc = make_rsrc(vbase + (int64_t)r0 * a.slot_stride);
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int row = (i * ROW_WAVES + wave) * L_ROWS + lane / CHUNKS, off = min(row, beyond) * stride2, c = lane % CHUNKS;
            const int k_off = off + (c ^ k_swizzle<HD>(row)) * 16, v_off = off + (c ^ v_swizzle<HD>(row)) * 16, at = (i * ROW_WAVES + wave) * 1024;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(k_rsrc, (lds_void_t*)(kv_s[stage][0] + at), 16, k_off, 0, 0, 0);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(v_rsrc, (lds_void_t*)(kv_s[stage][1] + at), 16, v_off, 0, 0, 0);
        }
    };
    f16x8_t qf[NT][KS];
    load_queries<HD, NT>(qf, a, t, kvh, row0);
    load(t.k0, 0);
    load(t.k0 + KEYS, 1);
    store_spans<64 * ROW_WAVES>(span_s, a, w, t, span);
    lds_barrier();
    uint32_t mine[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) mine[n] = span_s[SPANS_BEFORE + node_of(a, min(row0 + 16 * n + dc, R - 1))];
    const float sc = scale_of(a);
    float m[NT], l[NT], down[NT] = {};
    f32x4_t o[NT][DT];
    bool careful = false;
    const bool live = row0 < R;
    auto half = [&](auto masked_c, int k0, const unsigned char* k, const unsigned char* v) __attribute__((always_inline)) {      // 32 keys
        constexpr bool MASKED = decltype(masked_c)::value;
        f32x4_t s[NT][2];
        f16x8_t kf[2][KS];
        read_keys<HD>(k, kf);
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                s[n][c] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int e = 0; e < KS; ++e) s[n][c] = mfma_16x16x32<BF>(kf[c][e], qf[n][e], s[n][c]);
            }
        if constexpr (MASKED) {
            uint32_t key[2][4];
            key_spans<2>(key, t, k0, span_s);
#pragma unroll
            for (int n = 0; n < NT; ++n) {
#pragma unroll
                for (int c = 0; c < 2; ++c)
#pragma unroll
                    for (int r = 0; r < 4; ++r) s[n][c][r] = sees(mine[n], key[c][r]) ? s[n][c][r] : -INFINITY;
            }
        }
        Weights p[NT];
        weights_of<BF, NT, DT>(s, m, l, o, sc, down, p);
        add_values<BF, HD, NT, MASKED>(v, p, o, careful);
    };
    auto block = [&](auto masked_c, int k0, int stage) __attribute__((always_inline)) {
        constexpr bool MASKED = decltype(masked_c)::value;
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_waitcnt(0x0F70 | 2 * LOADS);      // this block; the next one may be in flight
        lds_barrier();
        if (live) {
            half(masked_c, k0, kv_s[stage][0], kv_s[stage][1]);
            if (!MASKED || k0 + 32 < t.k1) half(masked_c, k0 + 32, kv_s[stage][0] + 32 * ROW, kv_s[stage][1] + 32 * ROW);
        }
        lds_barrier();                                       // all wavefronts are done with the block
        load(k0 + 2 * KEYS, stage);
    };
    for (int turn = 1;; ++turn) {
        start<NT, DT>(m, l, o);
        int stage = 0, k0 = t.k0;
        if (!careful)
            for (; k0 + KEYS <= min(t.n_ctx, t.k1); k0 += KEYS, stage ^= 1) block(std::false_type(), k0, stage);
        for (; k0 < t.k1; k0 += KEYS, stage ^= 1) block(std::true_type(), k0, stage);
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_waitcnt(0x0F70);                  // nothing lands in LDS after the end
        __builtin_amdgcn_sched_barrier(0);
        bool odd[NT];
        if (turn == TURNS<BF> || !__syncthreads_or(live && not_finite(o, odd))) break;
        if (careful && live)
#pragma unroll
            for (int n = 0; n < NT; ++n) down[n] = odd[n] ? DOWN : 0.f;
        careful = true;
        load(t.k0, 0);
        load(t.k0 + KEYS, 1);
    }
    if (!live) return;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        l[n] += __shfl_xor(l[n], 16);
        l[n] += __shfl_xor(l[n], 32);
        const int r = 16 * n + dc, row = row0 + r;
        if (row >= R) continue;
        const int64_t at = row_at(a, t, kvh, row);
        const float inv = 1.f / l[n];                        // (a piece whose keys this row does not see: not used)
        l[n] = lifted(l[n], down[n]);
        if (t.index < a.n_parts) {
            const int64_t part = ((int64_t)t.index * a.n_kv_heads + kvh) * TR + wave * 16 * NT + r;
#pragma unroll
            for (int i = 0; i < DT; ++i) *reinterpret_cast<f32x4_t*>(a.part_o + part * HD + 16 * i + 4 * kg) = o[n][i] * inv;
            if (kg == 0) a.part_ml[part] = make_float2(m[n], l[n]);
        } else {
#pragma unroll
            for (int i = 0; i < DT; ++i)
                *reinterpret_cast<uint2*>((uint16_t*)a.out + at * HD + 16 * i + 4 * kg) = make_uint2(op_pack2<BF>(o[n][i][0] * inv, o[n][i][1] * inv), op_pack2<BF>(o[n][i][2] * inv, o[n][i][3] * inv));
            if (a.lse && kg == 0) a.lse[at] = (m[n] * sc - BIAS<BF> + __builtin_amdgcn_logf(l[n])) * LN2;
        }
    }
}

// The weight of every row: the scores once more, now that the log-sum-exps are known.  A workgroup owns a range of keys of a K/V head, a wavefront
// 32-key blocks of it, in operand registers; MASS_ROWS query rows at a time lie in LDS, their 16-byte chunks permuted so that the 16 rows of an operand
// read spread over all banks.  No atomics: a weight is one lane's, in one order.  93 rows over 63000 in two utterances, 8 heads of 128: 29 us, 4.4 TB/s of key rows;
// three workgroups a CU, which the compiler's choice of registers gives, take 36, and without the second block in flight 48.
constexpr int MASS_ROWS = 128;

template <bool BF, int HD, class M>
__global__ void __launch_bounds__(64 * MASS_WAVES, 4) tree_mass16_kernel(TreeAttnArgs a, M w) {
    constexpr int MASS_KEYS = 32, ROW = HD * 2, STEP = MASS_KEYS * MASS_WAVES, KS = HD / 32, CHUNKS = ROW / 16;
    __shared__ __align__(1024) unsigned char q_s[MASS_ROWS * ROW];
    __shared__ float lse_s[MASS_ROWS];
    __shared__ uint32_t row_span[MASS_ROWS], span_s[SPANS];
    const int lane = threadIdx.x % 64, kg = lane / 16, dc = lane % 16;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const Work t = mass_item_of(a, w, blockIdx.y);
    const int kvh = blockIdx.x;
    const int R = t.n_nodes * a.group, last = t.k1 - 1;
    const int stride2 = (int)a.slot_stride * 2;
    const uint16_t* kbase = (const uint16_t*)a.k + (int64_t)t.slot0 * a.slot_stride + kvh * a.head_stride;
    // two blocks of keys: the next one loads while one is used
    u32x4_t kr[2][2][KS];
    auto load_keys = [&](int k0, u32x4_t (&x)[2][KS]) __attribute__((always_inline)) {
        const int r0 = min(k0, last), beyond = last - r0;
        const __amdgpu_buffer_rsrc_t rsrc = make_rsrc(kbase + (int64_t)r0 * a.slot_stride);
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const int off = min(16 * c + dc, beyond) * stride2 + kg * 16;
#pragma unroll
            for (int s = 0; s < KS; ++s) x[c][s] = __builtin_amdgcn_raw_buffer_load_b128(rsrc, off + 64 * s, 0, 0);
        }
    };
    const int first = t.k0 + wave * MASS_KEYS;
    load_keys(first, kr[0]);
    if (t.k1 > t.n_ctx) store_spans<64 * MASS_WAVES>(span_s, a, w, t, (int)threadIdx.x < t.n_nodes ? w(a.spans + t.node0 + (int)threadIdx.x) : 0u);
    const float sc = scale_of(a);
    const uint32_t flip = a.scale < 0.f ? 0x80008000u : 0u, keep = a.scale == 0.f ? 0u : ~0u;
    for (int r0 = 0; r0 < R; r0 += MASS_ROWS) {
        const int rows = min(MASS_ROWS, R - r0), tiles = (rows + 15) / 16;
        if (r0) __syncthreads();
        for (int i = threadIdx.x; i < tiles * 16 * CHUNKS; i += 64 * MASS_WAVES) {
            const int r = i / CHUNKS, c = i % CHUNKS, row = min(r0 + r, R - 1);
            uint4 x = *reinterpret_cast<const uint4*>((const uint16_t*)a.q + query_at(a, t, kvh, row, HD) + c * 8);
            x.x = (x.x ^ flip) & keep; x.y = (x.y ^ flip) & keep; x.z = (x.z ^ flip) & keep; x.w = (x.w ^ flip) & keep;
            *reinterpret_cast<uint4*>(q_s + r * ROW + (c ^ k_swizzle<HD>(r)) * 16) = x;
        }
        for (int r = threadIdx.x; r < tiles * 16; r += 64 * MASS_WAVES) {
            const int row = min(r0 + r, R - 1);
            lse_s[r] = r < rows ? a.lse[row_at(a, t, kvh, row)] * -LOG2E : -INFINITY;   // (rows behind the last: no weight)
            row_span[r] = r < rows ? w(a.spans + t.node0 + node_of(a, row)) : 0xffffu;
        }
        __syncthreads();
        if (r0) load_keys(first, kr[0]);
        auto block = [&](auto masked_c, int k0, const u32x4_t (&x)[2][KS]) __attribute__((always_inline)) {
            constexpr bool MASKED = decltype(masked_c)::value;
            f32x4_t acc[2];
#pragma unroll
            for (int c = 0; c < 2; ++c) acc[c] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
            uint32_t key[2][4];
            if constexpr (MASKED) key_spans<2>(key, t, k0, span_s);
            for (int n = 0; n < tiles; ++n) {
                const int r = 16 * n + dc;
                f32x4_t s[2];
#pragma unroll
                for (int c = 0; c < 2; ++c) s[c] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int e = 0; e < KS; ++e) {
                    const f16x8_t q = as_f16x8(*reinterpret_cast<const uint4*>(q_s + r * ROW + ((kg + 4 * e) ^ k_swizzle<HD>(r)) * 16));
#pragma unroll
                    for (int c = 0; c < 2; ++c) s[c] = mfma_16x16x32<BF>(__builtin_bit_cast(f16x8_t, x[c][e]), q, s[c]);
                }
                const float base = lse_s[r];
                const uint32_t mine = MASKED ? row_span[r] : 0u;
#pragma unroll
                for (int c = 0; c < 2; ++c)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float p = __builtin_amdgcn_exp2f(fmaf(s[c][e], sc, base));
                        acc[c][e] += MASKED && !sees(mine, key[c][e]) ? 0.f : p;
                    }
            }
            add_mass(a, t, kvh, k0, r0 == 0, acc);
        };
        auto step = [&](auto masked_c, int k0) __attribute__((always_inline)) {          // two blocks
            load_keys(k0 + STEP, kr[1]);
            __builtin_amdgcn_sched_barrier(0);
            block(masked_c, k0, kr[0]);
            __builtin_amdgcn_sched_barrier(0);
            load_keys(k0 + 2 * STEP, kr[0]);
            __builtin_amdgcn_sched_barrier(0);
            if (k0 + STEP < t.k1) block(masked_c, k0 + STEP, kr[1]);
        };
        int k0 = first;
        for (; k0 + STEP + MASS_KEYS <= min(t.n_ctx, t.k1); k0 += 2 * STEP) step(std::false_type(), k0);
        if (t.k1 <= t.n_ctx) {                               // a range that ends inside the context consists of whole blocks: one is left, or none
            if (k0 < t.k1) block(std::false_type(), k0, kr[0]);
        } else
            for (; k0 < t.k1; k0 += 2 * STEP) step(std::true_type(), k0);
    }
}

template <bool BF, int HD, class M>
static void launch16(const TreeAttnArgs& a, const M& w, hipStream_t st) {
    const dim3 grid(a.n_kv_heads, a.n_items);
    if (a.tile_rows == 16) hipLaunchKernelGGL((tree_keys16_kernel<BF, HD, M>), grid, dim3(64 * KEY_WAVES), 0, st, a, w);
    else if (a.tile_rows == 64) hipLaunchKernelGGL((tree_rows16_kernel<BF, HD, 1, M>), grid, dim3(64 * ROW_WAVES), 0, st, a, w);
    else hipLaunchKernelGGL((tree_rows16_kernel<BF, HD, 2, M>), grid, dim3(64 * ROW_WAVES), 0, st, a, w);
    if (a.n_joins)
        hipLaunchKernelGGL((tree_join_kernel<BF ? SSD_BF16 : SSD_F16, HD, M>), dim3(a.n_joins * a.tile_rows, a.n_kv_heads), dim3(256), 0, st, a, w, BIAS<BF>);
    if (a.mass) hipLaunchKernelGGL((tree_mass16_kernel<BF, HD, M>), dim3(a.n_kv_heads, a.n_mass), dim3(64 * MASS_WAVES), 0, st, a, w);
}

template <class M>
static void launch_any(const TreeAttnArgs& a, const M& w, hipStream_t st) {
    if (a.dtype == SSD_F32) launch_tree_attention32(a, w, st);
    else if (a.head_dim == 64) a.dtype == SSD_BF16 ? launch16<true, 64>(a, w, st) : launch16<false, 64>(a, w, st);
    else a.dtype == SSD_BF16 ? launch16<true, 128>(a, w, st) : launch16<false, 128>(a, w, st);
}

void launch_tree_attention(const TreeAttnArgs& a, const uint32_t* words, int n, const uint32_t* dev_words, hipStream_t st) {
    static_assert(sizeof(TreeAttnArgs) + sizeof(MetaWords) + 16 <= 4096, "arguments of a launch");
    if (!words) { launch_any(a, MetaArray{dev_words}, st); return; }
    MetaWords w;
    w.n = n;
    memcpy(w.word, words, (size_t)n * 4);
    launch_any(a, w, st);
}

}  // namespace ssd
