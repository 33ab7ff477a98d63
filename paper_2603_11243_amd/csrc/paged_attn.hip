// Attention of the newest tokens over the pages of their utterances:
//   s_j = scale q . k_j,  lse = log sum_j exp s_j,  o = sum_j exp(s_j - lse) v_j   over the rows j that the token sees.
//
// One pass over the rows with a running maximum and sum.  A workgroup has 16 or 32 query rows of a K/V head (tokens times heads of the group), a column each of the
// matrix instructions, and a piece of a context; its four wavefronts take blocks of KEYS rows in turn and are joined through LDS, the pieces of a context
// by a second kernel.  S^T = K Q^T, then O^T += V^T P^T:
//   first product   lane (dc = lane % 16, g = lane / 16) holds row dc of a tile of 16 keys, the dims that its loads of 16 bytes bring (queries in the same order)
//   its result      column dc, keys 4 g + r
//   second product  the same lane's keys: so the weights are operands where they are, and the values of rows 4 g + r, dims DPL dc .. are loaded into the lane that
//                   needs them: a byte permutation inside its registers makes operands of them.  No LDS and no barrier in the loop; lanes exchange the maximum alone.
// 16-bit pages and codes go through v_mfma_f32_16x16x32 (half pages, and the first product of half queries with codes: half; all else bfloat16; both hold the codes of
// the 8-bit types exactly), fp32 pages through v_mfma_f32_16x16x4_f32.  The scale of a key row multiplies its score, that of a value row its weight.
//
// Bound by memory: a block is 32 registers a lane of keys and values each, requested again as soon as they are used, with two workgroups a CU (head_dim 128) 16 KB a
// wavefront on the way (codes 8 KB; twice as many keys a block changed nothing over long contexts and cost 90 short ones of int8 15.5 -> 20 us).  Eight K/V heads of 128, two query
// heads each: 200001 rows of bfloat16 144 us, 5.7 TB/s; four of 40000 rows of half 118 us (5.6), e4m3 66 (5.2), int8 67 (5.0); eight of 60000, e4m3, 179 (5.7).  Three workgroups a CU
// were slower (four recordings of e4m3 60 against 54 us: fewer, fuller rounds).  A context of 106 rows is 5.1 us in a graph: a launch, and length, page numbers, keys and
// merge one behind the other; every further block of a wavefront 1.3 us.  32 columns where that pays (paged_tile_rows): 27 rows over 16 contexts of int8 62 -> 50 us;
// with fp32 pages of 128 dims they spill 73 registers a lane and value loads wait for one another (12 tokens over 40 contexts of 2000 to 4000 rows 336 us, 201 by bytes), with 16-bit ones four.
#include "pages.h"
#include "tree_attn.h"

namespace ssd {

namespace {

constexpr int WAVES = KEY_WAVES;
constexpr float F16_END = 65520.f;                           // what rounds to half's largest value or less is smaller

template <int QT, int PT> struct Kind {
    static constexpr bool CODES = PT == SSD_E4M3 || PT == SSD_I8, F32 = PT == SSD_F32, BF = PT != SSD_F16;
    static constexpr int SIZE = CODES ? 1 : F32 ? 4 : 2;                     // bytes of an element
    static constexpr int KEYS = CODES ? 32 : F32 ? 16 : 32, TILES = KEYS / 16;     // 64 registers a lane of keys and values in flight
    static constexpr bool QBF = CODES ? QT != SSD_F16 : BF;                  // the first product's operands: the queries' type, which holds the codes exactly
    static constexpr int QN = CODES && QT == SSD_F32 ? 3 : 1;                // 16-bit values that a query is the exact sum of
    static constexpr int PN = QT == SSD_F32 ? 3 : 2;                         // those of a weight: of outputs of 16 bits two, which hold it 2^9 (half: 2^6) times as exactly; a third cost 49.3 -> 52.5 us (16 contexts of int8)
    // Weights are taken times a power of two: in half's upper range, or so that sums of 2^30 values at the end of fp32's range stay in it.  A factor, not a term of the
    // exponent: there it would take five bits of the difference to the maximum.
    static constexpr float UNIT = PT == SSD_F16 ? 0x1p15f : 0x1p-32f;
};

// Whole number in byte I of w as fp32.  (Written out because the compiler takes the bytes apart first.)
template <int I>
__device__ __forceinline__ float whole(uint32_t w) {
    float v;
    if constexpr (I == 0) asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_0" : "=v"(v) : "v"(w));
    else if constexpr (I == 1) asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_1" : "=v"(v) : "v"(w));
    else if constexpr (I == 2) asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_2" : "=v"(v) : "v"(w));
    else asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_3" : "=v"(v) : "v"(w));
    return v;
}

// Two codes to a pair of bfloat16 (BF) or half, exactly: bytes 2 HIGH and 2 HIGH + 1 of w.
template <int PT, bool BF, bool HIGH>
__device__ __forceinline__ uint32_t code_pair(uint32_t w) {
    if constexpr (PT == SSD_E4M3) {
        if constexpr (BF) return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, HIGH));
        else return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.f, HIGH));
    } else {
        const float lo = whole<2 * HIGH>(w), hi = whole<2 * HIGH + 1>(w);
        if constexpr (BF) return __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);
        else return pack16<false>(lo, hi);
    }
}

// Whole numbers in byte I of two words to a pair of bfloat16.
template <int I>
__device__ __forceinline__ uint32_t whole_pair(uint32_t lo, uint32_t hi) { return __builtin_amdgcn_perm(__float_as_uint(whole<I>(hi)), __float_as_uint(whole<I>(lo)), 0x07060302u); }

// The sign bits of the elements of a word that are not finite; the word with zeros for them.
template <int PT> __device__ __forceinline__ uint32_t not_finite(uint32_t w) {
    if constexpr (PT == SSD_I8) return 0u;
    else if constexpr (PT == SSD_E4M3) return ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
    else if constexpr (PT == SSD_F32) return ((w & 0x7fffffffu) + 0x00800000u) & 0x80000000u;
    else return beyond_of<PT == SSD_BF16>(w) & SIGNS;
}
template <int PT> __device__ __forceinline__ uint32_t finite(uint32_t w) {
    constexpr int BITS = PT == SSD_E4M3 || PT == SSD_I8 ? 8 : PT == SSD_F32 ? 32 : 16;
    return w & ~((not_finite<PT>(w) >> (BITS - 1)) * (BITS == 32 ? ~0u : (1u << BITS % 32) - 1u));
}

// Queries of a lane's column as operands of the first product: 16-bit values 8 of a step, or one fp32 value a step.
template <int QT, int PT, int HD> struct Queries {
    typedef Kind<QT, PT> T;
    f16x8_t x[T::QN][HD / 32];
    __device__ __forceinline__ void load(const void* q, int64_t at, int hd, int g) {
#pragma unroll
        for (int e = 0; e < HD / 32; ++e) {
            const int dim = T::CODES ? 64 * (e / 2) + 16 * g + 8 * (e % 2) : 32 * e + 8 * g;
            if constexpr (T::QN == 1) x[0][e] = as_f16x8(*reinterpret_cast<const uint4*>((const uint16_t*)q + at + dim));
            else {
                float v[8];
                const typename Elem<QT>::type* p = (const typename Elem<QT>::type*)q + at + dim;
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = Elem<QT>::get(p[i]);
#pragma unroll
                for (int n = 0; n < T::QN; ++n) {
                    uint32_t w[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        w[i] = pack16<true>(v[2 * i], v[2 * i + 1]);
                        v[2 * i] -= __uint_as_float(w[i] << 16);
                        v[2 * i + 1] -= __uint_as_float(w[i] & 0xffff0000u);
                    }
                    x[n][e] = as_f16x8(make_uint4(w[0], w[1], w[2], w[3]));
                }
            }
        }
    }
};
template <int HD> struct Queries<SSD_F32, SSD_F32, HD> {
    f32x4_t x[HD / 16];
    __device__ __forceinline__ void load(const void* q, int64_t at, int hd, int g) {
#pragma unroll
        for (int e = 0; e < HD / 16; ++e) {
            const int dim = 16 * e + 4 * g;
            x[e] = dim < hd ? *reinterpret_cast<const f32x4_t*>((const float*)q + at + dim) : (f32x4_t){0.f, 0.f, 0.f, 0.f};
        }
    }
};

__device__ __forceinline__ f32x4_t mfma_f32(float a, float b, const f32x4_t& c) { return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0); }

// Four values of a result, one store.  Means of 8-bit pages may lie beyond half's range, those of half pages do not.
template <int QT>
__device__ __forceinline__ void store4(typename Elem<QT>::type* out, f32x4_t v, bool codes, int32_t* flags) {
    if constexpr (QT == SSD_F32) *reinterpret_cast<f32x4_t*>(out) = v;
    else {
        if (QT == SSD_F16 && codes) {
            bool over = false;
#pragma unroll
            for (int e = 0; e < 4; ++e) over |= !(fabsf(v[e]) < F16_END);
            if (over) {
                raise_flag(flags, SSD_FLAG_ACT_OVERFLOW);
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = fabsf(v[e]) <= F32_MOST ? fminf(fmaxf(v[e], -F16_MAX), F16_MAX) : v[e];
            }
        }
        *reinterpret_cast<uint2*>(out) = make_uint2(pack16<QT == SSD_BF16>(v[0], v[1]), pack16<QT == SSD_BF16>(v[2], v[3]));
    }
}

// What a workgroup does: piece `part` of n of utterance b, rows from ..; index: the piece's number among all.
struct Piece { int b, part, n, index, len, given, from, rows; };

__device__ __forceinline__ int units(int rows) { return (rows + PAGED_UNIT - 1) / PAGED_UNIT; }
__device__ __forceinline__ int clamped(const PagesArgs& p, int len) { return min(max(len, 0), p.max_ctx); }

// Units of a shared piece for so many in all.
__device__ __forceinline__ int shared_units(const PagedAttnArgs& a, int total) { return max(1, (int)(((uint32_t)total + a.shared - 1) / (uint32_t)a.shared)); }

struct OpAdd { __device__ __forceinline__ int operator()(int x, int y) const { return x + y; } };
__device__ __forceinline__ int lanes_sum(int v) { return group_allreduce_i<64>(v, OpAdd()); }
// Sum of the lanes up to each: inside rows of 16, then over the rows before (their last lanes go to the rows behind).
__device__ __forceinline__ int lanes_scan(int v) {
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);      // row_shr 1, 2, 4, 8
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);      // row_bcast 15 to rows 1 and 3
    v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);      // row_bcast 31 to rows 2 and 3
    return v;
}

// The workgroup's piece; false: there is none.  Up to 64 utterances a wavefront finds it by itself, a lane an utterance.
__device__ __forceinline__ bool find_piece(const PagedAttnArgs& a, Piece& t) {
    const PagesArgs& p = a.p;
    const int lane = threadIdx.x % 64, x = blockIdx.x;
    int size;
    if (a.shared == 0) {
        t.b = blockIdx.z / a.tiles;
        t.part = x;
        t.given = p.ctx_len[t.b];
        t.len = clamped(p, t.given);
        size = PAGED_MOST;
        t.n = max(1, (units(t.len) + size - 1) / size);
        t.index = t.b * a.n_pieces + x;
        if (a.n_pieces > 1 && x >= t.n) return false;
    } else if (p.B <= 64) {
        const int given = lane < p.B ? p.ctx_len[lane] : 0, len = clamped(p, given), u = units(len);
        const int want = max(a.shared, p.B);
        int share = shared_units(a, lanes_sum(u)), n, pieces;
        // every utterance's last piece is a shorter one: so many more than wanted, and a second round of workgroups for them, until pieces are a little longer
        for (int turn = 0;; ++turn) {
            n = lane < p.B ? max(1, (int)((uint32_t)(u + share - 1) / (uint32_t)share)) : 0;
            pieces = lanes_sum(n);
            if (pieces <= want || turn == 8) break;
            share = max(share + 1, (int)((float)share * (float)pieces / (float)want));
        }
        const int sum = lanes_scan(n);
        const uint64_t behind = __ballot(sum > x);
        if (!behind) return false;
        t.b = __ffsll((unsigned long long)behind) - 1;
        t.n = __builtin_amdgcn_readlane(n, t.b);
        t.part = x - (__builtin_amdgcn_readlane(sum, t.b) - t.n);
        t.given = __builtin_amdgcn_readlane(given, t.b);
        t.len = __builtin_amdgcn_readlane(len, t.b);
        t.index = x;
    } else {
        constexpr int THREADS = 64 * WAVES, PER = PAGED_UTTS / THREADS;
        __shared__ int wave_s[WAVES], found_s[4];
        const int tid = threadIdx.x, wave = tid / 64;
        int given[PER], u = 0;
#pragma unroll
        for (int e = 0; e < PER; ++e) {
            given[e] = tid * PER + e < p.B ? p.ctx_len[tid * PER + e] : 0;
            u += units(clamped(p, given[e]));
        }
        u = lanes_sum(u);
        if (lane == 0) wave_s[wave] = u;
        __syncthreads();
        int total = 0;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) total += wave_s[w];
        const int share = shared_units(a, total);
        int n[PER], mine = 0;
#pragma unroll
        for (int e = 0; e < PER; ++e) mine += n[e] = tid * PER + e < p.B ? max(1, (int)((uint32_t)(units(clamped(p, given[e])) + share - 1) / (uint32_t)share)) : 0;
        int sum = lanes_scan(mine);
        __syncthreads();
        if (lane == 63) wave_s[wave] = sum;
        if (tid == 0) found_s[0] = -1;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < WAVES; ++w) sum += w < wave ? wave_s[w] : 0;
        int at = sum - mine;
#pragma unroll
        for (int e = 0; e < PER; ++e) {
            if (x >= at && x < at + n[e]) {
                found_s[0] = tid * PER + e;
                found_s[1] = n[e];
                found_s[2] = x - at;
                found_s[3] = given[e];
            }
            at += n[e];
        }
        __syncthreads();
        t.b = __builtin_amdgcn_readfirstlane(found_s[0]);
        if (t.b < 0) return false;
        t.n = __builtin_amdgcn_readfirstlane(found_s[1]);
        t.part = __builtin_amdgcn_readfirstlane(found_s[2]);
        t.given = __builtin_amdgcn_readfirstlane(found_s[3]);
        t.len = clamped(p, t.given);
        t.index = x;
    }
    if (a.shared) size = (int)((uint32_t)(units(t.len) + t.n - 1) / (uint32_t)t.n);     // equal pieces; (n - 1 of them are less than the context)
    t.rows = size * PAGED_UNIT;
    t.from = t.part * t.rows;
    return true;
}

template <int QT, int PT, int HD, int NT>
__global__ void __launch_bounds__(64 * WAVES, 2) paged_attn_kernel(PagedAttnArgs a) {
    typedef Kind<QT, PT> T;
    typedef Elem<QT> E;
    constexpr int KEYS = T::KEYS, TILES = T::TILES, DPL = HD / 16, DT = HD / 16, STEP = KEYS * WAVES, PITCH = HD + 4;
    constexpr int K_LOADS = HD * T::SIZE / 64, V_WORDS = DPL * T::SIZE / 4, KNOWN = 64 / TILES;
    __shared__ float o_s[WAVES][16][PITCH];
    __shared__ float2 ml_s[WAVES][16];
    const PagesArgs& p = a.p;
    const int lane = threadIdx.x % 64, g = lane / 16, dc = lane % 16, hd = T::F32 ? p.head_dim : HD;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int kvh = blockIdx.y, tile = a.shared ? blockIdx.z : blockIdx.z % a.tiles;
    Piece t;
    if (!find_piece(a, t)) return;
    const int b = t.b, len = t.len, from = t.from, to = min(len, from + t.rows);
    const bool only = t.n == 1;
    bool bad = t.given != len;

    // Pages of the wavefront's tiles, of KNOWN blocks at a time: lane i has those of tile i % TILES of the block i / TILES behind the first of them.
    const int first = from + wave * KEYS, blocks = (to - first + STEP - 1) / STEP;
    int pages = -1;
    auto find_pages = [&](int block, int lane) {
        const int key = first + (block + lane / TILES) * STEP + 16 * (lane % TILES);
        pages = key < min(from + t.rows, p.max_ctx) ? page_of(p, b, key) : -1;      // (the first ones without waiting for the length)
        bad |= key < to && pages < 0;
        if (key >= to) pages = -1;
    };
    find_pages(0, lane);
    const int rows = a.n_new * a.group, row0 = tile * 16 * NT;
    const int least = len - (a.n_new - 1 - min(row0, rows - 1) / a.group);      // what all columns see
    int limit[NT];                                           // the column's token sees the rows before it
    Queries<QT, PT, HD> q[NT];
#pragma unroll
    for (int u = 0; u < NT; ++u) {
        const int row = min(row0 + 16 * u + dc, rows - 1), token = row / a.group;
        limit[u] = len - (a.n_new - 1 - token);
        q[u].load(a.q, ((int64_t)b * a.n_new + token) * a.q_stride + (int64_t)(kvh * a.group + row % a.group) * hd, hd, g);
    }

    u32x4_t kr[TILES][K_LOADS];
    constexpr int WORDS = T::F32 ? 4 : V_WORDS, V_PARTS = V_WORDS / WORDS;
    typedef uint32_t words_t __attribute__((ext_vector_type(WORDS)));
    words_t vr[TILES][4][V_PARTS];
    f32x4_t ks[T::CODES ? TILES : 1], vs[T::CODES ? TILES : 1];
    auto row_of = [&](int block, int c) {                    // first row of a tile; of pages that are none, any
        const int page = __builtin_amdgcn_readlane(pages, block % KNOWN * TILES + c);
        return row_in_pages(p, max(page, 0), kvh, first + block * STEP + 16 * c);
    };
    auto load_keys = [&](int block) {
#pragma unroll
        for (int c = 0; c < TILES; ++c) {
            const int64_t r = row_of(block, c);
            const char* k = (const char*)p.k + r * hd * T::SIZE;
            if constexpr (T::CODES) ks[c] = *reinterpret_cast<const f32x4_t*>(p.k_scale + r + 4 * g);
#pragma unroll
            for (int e = 0; e < K_LOADS; ++e) {
                if constexpr (T::F32) {
                    const int dim = 16 * e + 4 * g;
                    kr[c][e] = *reinterpret_cast<const u32x4_t*>(k + (dc * hd + (dim < hd ? dim : 0)) * 4);
                } else kr[c][e] = *reinterpret_cast<const u32x4_t*>(k + (uint32_t)(dc * HD * T::SIZE + 64 * e + 16 * g));
            }
        }
    };
    auto load_values = [&](int block) {
#pragma unroll
        for (int c = 0; c < TILES; ++c) {
            const int64_t r = row_of(block, c);
            const char* v = (const char*)p.v + r * hd * T::SIZE;
            if constexpr (T::CODES) vs[c] = *reinterpret_cast<const f32x4_t*>(p.v_scale + r + 4 * g);
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int h = 0; h < V_PARTS; ++h) {
                    const int dim = T::F32 ? 64 * h + 4 * dc : DPL * dc;
                    vr[c][i][h] = *reinterpret_cast<const words_t*>(v + (uint32_t)(((4 * g + i) * hd + (T::F32 && dim >= hd ? 0 : dim)) * T::SIZE));
                }
        }
    };
    if (blocks > 0) {
        load_keys(0);
        load_values(0);
    }
    const float sc = a.scale * LOG2E;
    float m[NT], l[NT];
    f32x4_t o[NT][DT];
    uint32_t lost[NT];                                       // outputs 4 i + e of the lane that are NaN because of a row that only some columns see
#pragma unroll
    for (int u = 0; u < NT; ++u) {
        m[u] = -F32_MOST;
        l[u] = 0.f;
        lost[u] = 0;
#pragma unroll
        for (int i = 0; i < DT; ++i) o[u][i] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
    }
    bool whole = !__any(bad);
    auto add_block = [&](auto last_c, int block) __attribute__((always_inline)) {
        constexpr bool LAST = decltype(last_c)::value;
        const int k0 = first + block * STEP;
        const bool masked = !whole || k0 + KEYS > min(least, to);
        float s[NT][TILES][4];
#pragma unroll
        for (int c = 0; c < TILES; ++c) {
            f32x4_t x[NT];
#pragma unroll
            for (int u = 0; u < NT; ++u) x[u] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
            if constexpr (T::F32) {
#pragma unroll
                for (int e = 0; e < K_LOADS; ++e) {
                    const f32x4_t k = __builtin_bit_cast(f32x4_t, kr[c][e]);
                    const bool there = 16 * e + 4 * g < hd;
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int u = 0; u < NT; ++u) x[u] = mfma_f32(there ? k[i] : 0.f, q[u].x[e][i], x[u]);
                }
            } else {
#pragma unroll
                for (int e = 0; e < HD / 32; ++e) {
                    f16x8_t k;
                    if constexpr (T::CODES) {
                        const uint32_t lo = kr[c][e / 2][e % 2 * 2], hi = kr[c][e / 2][e % 2 * 2 + 1];
                        k = as_f16x8(make_uint4(code_pair<PT, T::QBF, false>(lo), code_pair<PT, T::QBF, true>(lo), code_pair<PT, T::QBF, false>(hi),
                                                code_pair<PT, T::QBF, true>(hi)));
                    } else k = __builtin_bit_cast(f16x8_t, kr[c][e]);
#pragma unroll
                    for (int n = 0; n < T::QN; ++n)
#pragma unroll
                        for (int u = 0; u < NT; ++u) x[u] = mfma_16x16x32<T::QBF>(k, q[u].x[n][e], x[u]);
                }
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const float scale = T::CODES ? ks[c][r] * sc : sc;
#pragma unroll
                for (int u = 0; u < NT; ++u) s[u][c][r] = x[u][r] * scale;
            }
        }
        // Keys of the lane that its columns see (bits 4 c + r), and that some column does.
        uint32_t mine[NT], some = ~0u;
#pragma unroll
        for (int u = 0; u < NT; ++u) mine[u] = ~0u;
        if (masked) {
            some = 0;
#pragma unroll
            for (int u = 0; u < NT; ++u) mine[u] = 0;
#pragma unroll
            for (int c = 0; c < TILES; ++c) {
                const bool here = __builtin_amdgcn_readlane(pages, block % KNOWN * TILES + c) >= 0;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int j = k0 + 16 * c + 4 * g + r;
                    some |= (uint32_t)(here && j < len) << (4 * c + r);
#pragma unroll
                    for (int u = 0; u < NT; ++u) {
                        mine[u] |= (uint32_t)(here && j < limit[u]) << (4 * c + r);
                        s[u][c][r] = mine[u] >> (4 * c + r) & 1 ? s[u][c][r] : -INFINITY;
                    }
                }
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (!LAST) {
            if ((block + 1) % KNOWN == 0) {
                uint32_t all = ~0u;
                asm volatile("" : "+s"(all));                // (the lane's number is counted again: kept, with what follows from it, it takes registers of every block)
                find_pages(block + 1, __builtin_amdgcn_mbcnt_hi(all, __builtin_amdgcn_mbcnt_lo(all, 0)));
                whole = !__any(bad);
            }
            load_keys(block + 1);
        }
        __builtin_amdgcn_sched_barrier(0);
        float top[NT];
        bool above = false;
#pragma unroll
        for (int u = 0; u < NT; ++u) {
            float x = s[u][0][0];
#pragma unroll
            for (int i = 1; i < 4 * TILES; ++i) x = fmaxf(x, s[u][i / 4][i % 4]);
            x = fmaxf(x, __shfl_xor(x, 16));
            top[u] = fmaxf(m[u], fmaxf(x, __shfl_xor(x, 32)));
            above |= top[u] > m[u];
        }
        if (__any(above)) {
#pragma unroll
            for (int u = 0; u < NT; ++u) {
                const float alpha = __builtin_amdgcn_exp2f(m[u] - top[u]);
                l[u] *= alpha;
#pragma unroll
                for (int i = 0; i < DT; ++i) o[u][i] *= alpha;
                m[u] = top[u];
            }
        }
#pragma unroll
        for (int u = 0; u < NT; ++u) {
#pragma unroll
            for (int c = 0; c < TILES; ++c)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    s[u][c][r] = __builtin_amdgcn_exp2f(s[u][c][r] - m[u]);
                    l[u] += s[u][c][r];
                    s[u][c][r] *= T::CODES ? vs[c][r] * T::UNIT : T::UNIT;
                }
        }
        if (masked) {
            // Weights of rows that the column does not see are zeros, whatever their scales hold; rows that no column sees become zeros, whatever they hold.
            bool odd = false;
#pragma unroll
            for (int c = 0; c < TILES; ++c)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    if (T::CODES)
#pragma unroll
                        for (int u = 0; u < NT; ++u) s[u][c][r] = mine[u] >> (4 * c + r) & 1 ? s[u][c][r] : 0.f;
#pragma unroll
                    for (int h = 0; h < V_PARTS; ++h) {
                        vr[c][r][h] = some >> (4 * c + r) & 1 ? vr[c][r][h] : (words_t)(0u);
#pragma unroll
                        for (int w = 0; w < WORDS; ++w) odd |= not_finite<PT>(vr[c][r][h][w]) != 0;
                    }
                }
            // What is not finite in a row that some columns see makes the outputs of those NaN, and counts as zero for all.
            if (__any(odd)) {
#pragma unroll
                for (int c = 0; c < TILES; ++c)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
#pragma unroll
                        for (int i = 0; i < DT; ++i) {
                            const uint32_t x = vr[c][r][T::F32 ? i / 4 : 0][T::F32 ? i % 4 : i * T::SIZE / 4];
                            const bool is = not_finite<PT>(x) >> (T::SIZE == 1 ? 8 * (i % 4) + 7 : T::SIZE == 2 ? 16 * (i % 2) + 15 : 31) & 1;
#pragma unroll
                            for (int u = 0; u < NT; ++u) {
                                const f32x4_t n = mfma_f32(is ? 1.f : 0.f, mine[u] >> (4 * c + r) & 1 ? 1.f : 0.f, (f32x4_t){0.f, 0.f, 0.f, 0.f});
#pragma unroll
                                for (int e = 0; e < 4; ++e) lost[u] |= (uint32_t)(n[e] > 0.f) << (4 * i + e);
                                asm volatile("" : "+v"(lost[u]));        // (one after the other: registers, not speed)
                            }
                        }
#pragma unroll
                        for (int h = 0; h < V_PARTS; ++h)
#pragma unroll
                            for (int w = 0; w < WORDS; ++w) vr[c][r][h][w] = finite<PT>(vr[c][r][h][w]);
                    }
            }
        }
        if constexpr (T::F32) {
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int i = 0; i < DT; ++i)
#pragma unroll
                    for (int u = 0; u < NT; ++u) o[u][i] = mfma_f32(__uint_as_float(vr[0][r][i / 4][i % 4]), s[u][0][r], o[u][i]);
        } else {
            static_assert(TILES == 2, "32 keys an operand");
            f16x8_t w[NT][T::PN];
#pragma unroll
            for (int u = 0; u < NT; ++u)
#pragma unroll
                for (int n = 0; n < T::PN; ++n) {
                    uint32_t x[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        float& lo = s[u][e / 2][e % 2 * 2];
                        float& hi = s[u][e / 2][e % 2 * 2 + 1];
                        x[e] = pack16<T::BF>(lo, hi);
                        const f16x2_t z = __builtin_bit_cast(f16x2_t, x[e]);
                        lo -= T::BF ? __uint_as_float(x[e] << 16) : (float)z.x;
                        hi -= T::BF ? __uint_as_float(x[e] & 0xffff0000u) : (float)z.y;
                    }
                    w[u][n] = as_f16x8(make_uint4(x[0], x[1], x[2], x[3]));
                }
            auto add = [&](int i, uint32_t x0, uint32_t x1, uint32_t x2, uint32_t x3) __attribute__((always_inline)) {
                const f16x8_t x = as_f16x8(make_uint4(x0, x1, x2, x3));
#pragma unroll
                for (int n = 0; n < T::PN; ++n)
#pragma unroll
                    for (int u = 0; u < NT; ++u) o[u][i] = mfma_16x16x32<T::BF>(x, w[u][n], o[u][i]);
            };
            const auto& v0 = vr[0];
            const auto& v1 = vr[1];
            if constexpr (PT == SSD_I8) {
#pragma unroll
                for (int i = 0; i < DT; i += 4) {            // byte i % 4 of two rows
                    const auto rows = [&](int r) { return r < 4 ? v0[r][0][i / 4] : v1[r - 4][0][i / 4]; };
                    add(i, whole_pair<0>(rows(0), rows(1)), whole_pair<0>(rows(2), rows(3)), whole_pair<0>(rows(4), rows(5)), whole_pair<0>(rows(6), rows(7)));
                    add(i + 1, whole_pair<1>(rows(0), rows(1)), whole_pair<1>(rows(2), rows(3)), whole_pair<1>(rows(4), rows(5)), whole_pair<1>(rows(6), rows(7)));
                    add(i + 2, whole_pair<2>(rows(0), rows(1)), whole_pair<2>(rows(2), rows(3)), whole_pair<2>(rows(4), rows(5)), whole_pair<2>(rows(6), rows(7)));
                    add(i + 3, whole_pair<3>(rows(0), rows(1)), whole_pair<3>(rows(2), rows(3)), whole_pair<3>(rows(4), rows(5)), whole_pair<3>(rows(6), rows(7)));
                }
            } else if constexpr (PT == SSD_E4M3) {
#pragma unroll
                for (int i = 0; i < DT; i += 2) {            // bytes i, i + 1 of two rows side by side
                    const uint32_t pick = i % 4 ? 0x07030602u : 0x05010400u;
                    uint32_t t[4];
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        t[e] = __builtin_amdgcn_perm(v0[2 * e + 1][0][i / 4], v0[2 * e][0][i / 4], pick);
                        t[2 + e] = __builtin_amdgcn_perm(v1[2 * e + 1][0][i / 4], v1[2 * e][0][i / 4], pick);
                    }
                    add(i, code_pair<PT, true, false>(t[0]), code_pair<PT, true, false>(t[1]), code_pair<PT, true, false>(t[2]), code_pair<PT, true, false>(t[3]));
                    add(i + 1, code_pair<PT, true, true>(t[0]), code_pair<PT, true, true>(t[1]), code_pair<PT, true, true>(t[2]), code_pair<PT, true, true>(t[3]));
                }
            } else {
#pragma unroll
                for (int i = 0; i < DT; ++i) {
                    const uint32_t pick = i % 2 ? 0x07060302u : 0x05040100u;
                    add(i, __builtin_amdgcn_perm(v0[1][0][i / 2], v0[0][0][i / 2], pick), __builtin_amdgcn_perm(v0[3][0][i / 2], v0[2][0][i / 2], pick),
                        __builtin_amdgcn_perm(v1[1][0][i / 2], v1[0][0][i / 2], pick), __builtin_amdgcn_perm(v1[3][0][i / 2], v1[2][0][i / 2], pick));
                }
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (!LAST) load_values(block + 1);
        __builtin_amdgcn_sched_barrier(0);
    };
    for (int block = 0; block < blocks - 1; ++block) add_block(std::false_type(), block);
    if (blocks > 0) add_block(std::true_type(), blocks - 1);

#pragma unroll
    for (int u = 0; u < NT; ++u) {
        if (u) __syncthreads();
        if (__any(lost[u] != 0)) {
#pragma unroll
            for (int i = 0; i < 4 * DT; ++i) o[u][i / 4][i % 4] = lost[u] >> i & 1 ? NAN : o[u][i / 4][i % 4];
        }
        l[u] += __shfl_xor(l[u], 16);
        l[u] += __shfl_xor(l[u], 32);
        const float inv = l[u] == 0.f ? 0.f : 1.f / (T::UNIT * l[u]);
        if (g == 0) ml_s[wave][dc] = make_float2(m[u], l[u]);
#pragma unroll
        for (int i = 0; i < DT; i += 4)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int dim = T::F32 ? 16 * i + 16 * g + 4 * r : DPL * (4 * g + r) + i;
                *reinterpret_cast<f32x4_t*>(&o_s[wave][dc][dim]) = (f32x4_t){o[u][i][r] * inv, o[u][i + 1][r] * inv, o[u][i + 2][r] * inv, o[u][i + 3][r] * inv};
            }
        __syncthreads();
        constexpr int PER = HD / 4;                              // threads of a row
        for (int i = threadIdx.x; i < 16 * PER; i += 64 * WAVES) {
            const int r = i / PER, dim = i % PER * 4, n = row0 + 16 * u + r;
            if (n >= rows || dim >= hd) continue;
            float mt = -F32_MOST, lt = 0.f, share[WAVES];
#pragma unroll
            for (int w = 0; w < WAVES; ++w) mt = fmaxf(mt, ml_s[w][r].x);
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                const float2 x = ml_s[w][r];
                share[w] = x.y == 0.f ? 0.f : x.y * __builtin_amdgcn_exp2f(x.x - mt);
                lt += share[w];
            }
            const float one = lt == 0.f ? 0.f : 1.f / lt;
            f32x4_t v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < WAVES; ++w) v += *reinterpret_cast<const f32x4_t*>(&o_s[w][r][dim]) * (share[w] * one);
            const int64_t at = ((int64_t)b * a.n_new + n / a.group) * a.n_q_heads + kvh * a.group + n % a.group;
            if (only) {
                store4<QT>((typename E::type*)a.out + at * hd + dim, v, T::CODES, p.flags);
                if (a.lse && dim == 0) a.lse[at] = lt == 0.f ? -INFINITY : (mt + __builtin_amdgcn_logf(lt)) * LN2;
            } else {
                const int64_t to_at = ((int64_t)t.index * p.n_kv_heads + kvh) * rows + n;
                *reinterpret_cast<f32x4_t*>(a.part_o + to_at * HD + dim) = v;
                if (dim == 0) a.part_ml[to_at] = make_float2(mt, lt);
            }
        }
    }
    if (a.n_pieces > 1 && t.part == 0 && kvh == 0 && tile == 0 && threadIdx.x == 0) a.first[b] = make_int2(t.index, t.n);
    if (bad) raise_flag(p.flags, SSD_FLAG_BAD_PAGE);
}

// The pieces of a context, a mean of values each, joined: a workgroup has a query row, groups of HD / 4 lanes take its pieces in turn and are joined by lane moves, the
// wavefronts through LDS.
template <int QT, int HD, int THREADS>
__global__ void __launch_bounds__(THREADS) paged_join_kernel(PagedAttnArgs a) {
    typedef Elem<QT> E;
    constexpr int LANES = HD / 4, GROUPS = THREADS / LANES, U = 4, JOIN_WAVES = THREADS / 64;
    __shared__ f32x4_t o_s[JOIN_WAVES][LANES];
    __shared__ float2 ml_s[JOIN_WAVES];
    const int64_t at = blockIdx.x;
    const int token = (int)(at / a.n_q_heads), head = (int)(at % a.n_q_heads), b = token / a.n_new;
    const int first = a.first[b].x, pieces = a.first[b].y;
    if (pieces <= 1) return;
    const int group = threadIdx.x / LANES, dim = threadIdx.x % LANES * 4;
    const int64_t rows = a.n_new * a.group, step = rows * a.p.n_kv_heads;
    const int64_t row0 = first * step + head / a.group * rows + token % a.n_new * a.group + head % a.group;
    float m = -F32_MOST, l = 0.f;
    f32x4_t v = {0.f, 0.f, 0.f, 0.f};
    for (int p0 = group; p0 < pieces; p0 += U * GROUPS) {
        float2 y[U];
        f32x4_t z[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t i = row0 + min(p0 + u * GROUPS, pieces - 1) * step;
            y[u] = a.part_ml[i];
            z[u] = *reinterpret_cast<const f32x4_t*>(a.part_o + i * HD + dim);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (p0 + u * GROUPS >= pieces || y[u].y == 0.f) continue;                      // (a piece whose rows the token does not see)
            const float top = fmaxf(m, y[u].x), old = l * __builtin_amdgcn_exp2f(m - top), now = y[u].y * __builtin_amdgcn_exp2f(y[u].x - top);
            m = top;
            l = old + now;
            const float inv = 1.f / l;
            v = v * (old * inv) + z[u] * (now * inv);
        }
    }
#pragma unroll
    for (int off = LANES; off < 64; off *= 2) {
        const float other_m = __shfl_xor(m, off), other_l = __shfl_xor(l, off);
        const f32x4_t other_v = {__shfl_xor(v[0], off), __shfl_xor(v[1], off), __shfl_xor(v[2], off), __shfl_xor(v[3], off)};
        const float top = fmaxf(m, other_m), old = l == 0.f ? 0.f : l * __builtin_amdgcn_exp2f(m - top);
        const float now = other_l == 0.f ? 0.f : other_l * __builtin_amdgcn_exp2f(other_m - top), sum = old + now, inv = sum == 0.f ? 0.f : 1.f / sum;
        m = top;
        l = sum;
        v = v * (old * inv) + other_v * (now * inv);
    }
    const int wave = threadIdx.x / 64;
    if (threadIdx.x % 64 < LANES) o_s[wave][dim / 4] = v;
    if (threadIdx.x % 64 == 0) ml_s[wave] = make_float2(m, l);
    __syncthreads();
    if (group || dim >= a.p.head_dim) return;
    float mt = -F32_MOST, lt = 0.f, f[JOIN_WAVES];
#pragma unroll
    for (int i = 0; i < JOIN_WAVES; ++i) mt = fmaxf(mt, ml_s[i].x);
#pragma unroll
    for (int i = 0; i < JOIN_WAVES; ++i) {
        const float2 y = ml_s[i];
        f[i] = y.y == 0.f ? 0.f : y.y * __builtin_amdgcn_exp2f(y.x - mt);
        lt += f[i];
    }
    const float inv = lt == 0.f ? 0.f : 1.f / lt;
    f32x4_t s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < JOIN_WAVES; ++i) s += o_s[i][dim / 4] * (f[i] * inv);
    store4<QT>((typename E::type*)a.out + at * a.p.head_dim + dim, s, a.codes, a.p.flags);
    if (a.lse && dim == 0) a.lse[at] = lt == 0.f ? -INFINITY : (mt + __builtin_amdgcn_logf(lt)) * LN2;
}

template <int QT, int PT, int HD>
void launch_rows(const PagedAttnArgs& a, hipStream_t st) {
    const dim3 grid(a.n_pieces, a.p.n_kv_heads, a.shared ? a.tiles : a.p.B * a.tiles);
    constexpr int used = WAVES * 16 * ((HD + 4) * 4 + 8);
    const int more = a.shared ? PAGED_CU_LDS / (paged_per_cu(a.p.head_dim, a.tile_rows) + 1) + 1024 - used : 0;
    if constexpr (Kind<QT, PT>::CODES && QT == SSD_F32) paged_attn_kernel<QT, PT, HD, 1><<<grid, 64 * WAVES, more, st>>>(a);
    else if (a.tile_rows == 16) paged_attn_kernel<QT, PT, HD, 1><<<grid, 64 * WAVES, more, st>>>(a);
    else paged_attn_kernel<QT, PT, HD, 2><<<grid, 64 * WAVES, more, st>>>(a);
    const unsigned n = (unsigned)((int64_t)a.p.B * a.n_new * a.n_q_heads);
    const int each = a.shared ? a.n_pieces / a.p.B : a.n_pieces;             // pieces of an utterance, about
    // 128, 256, 512 and 1024 threads, whole calls in a graph, by the pieces of a context and the query rows in all: 2 of 1288 16.6, 17.0, 18.4, 21.4 us;
    // 16 of 64 50.7, 50.0, 50.2, 50.6; 64 of 16 145.8, 144.1, 143.7, 144.2; 85 of 192 22.4, 20.7, 20.4, 20.1; 235 of 8 23.3, 17.0, 14.1, 13.0
    if (each > 128) paged_join_kernel<QT, HD, 1024><<<n, 1024, 0, st>>>(a);
    else if (each > 32) paged_join_kernel<QT, HD, 512><<<n, 512, 0, st>>>(a);
    else if (each > 8) paged_join_kernel<QT, HD, 256><<<n, 256, 0, st>>>(a);
    else if (a.n_pieces > 1) paged_join_kernel<QT, HD, 128><<<n, 128, 0, st>>>(a);
}
template <int QT, int PT>
void launch_dims(const PagedAttnArgs& a, hipStream_t st) {
    if (a.p.head_dim > 64) launch_rows<QT, PT, 128>(a, st);
    else launch_rows<QT, PT, 64>(a, st);
}
template <int QT>
void launch_type(const PagedAttnArgs& a, int pages_dtype, hipStream_t st) {
    if (pages_dtype == SSD_E4M3) launch_dims<QT, SSD_E4M3>(a, st);
    else if (pages_dtype == SSD_I8) launch_dims<QT, SSD_I8>(a, st);
    else launch_dims<QT, QT>(a, st);
}

}  // namespace

void launch_paged_attention(const PagedAttnArgs& a, int q_dtype, int pages_dtype, hipStream_t st) {
    if (q_dtype == SSD_F32) launch_type<SSD_F32>(a, pages_dtype, st);
    else if (q_dtype == SSD_BF16) launch_type<SSD_BF16>(a, pages_dtype, st);
    else launch_type<SSD_F16>(a, pages_dtype, st);
}

}  // namespace ssd
