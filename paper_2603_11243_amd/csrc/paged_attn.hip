// Attention of the newest tokens over the pages of their utterances:
//   s_j = scale q . k_j,  lse = log sum_j exp s_j,  o = sum_j exp(s_j - lse) v_j   over the rows j that the token sees.
//
// One pass over the rows with a running maximum and sum.  A workgroup has up to 16 query rows of a K/V head (tokens times heads of the group), a column each of
// the matrix instructions, and a piece of the context; its four wavefronts take blocks of KEYS rows in turn and are joined through LDS, the pieces of a context
// by a second kernel.  S^T = K Q^T, then O^T += V^T P^T:
//   first product   lane (dc = lane % 16, g = lane / 16) holds row dc of a tile of 16 keys, the dims that its loads of 16 bytes bring (queries in the same order)
//   its result      column dc, keys 4 g + r
//   second product  the same lane's keys: so the weights are operands where they are, and the values of rows 4 g + r, dims DPL dc .. are loaded into the lane that
//                   needs them: a byte permutation inside its registers makes operands of them.  No LDS, no exchange, no barrier in the loop.
// 16-bit pages and codes go through v_mfma_f32_16x16x32 (half pages: half; all else bfloat16, which holds the codes of both 8-bit types exactly), fp32 pages through
// v_mfma_f32_16x16x4_f32.  The scale of a key row multiplies its score, that of a value row its weight.
// What bounds it is memory: 16 rows are few for the matrix cores.
#include "pages.h"
#include "tree_attn.h"

namespace ssd {

namespace {

constexpr int WAVES = KEY_WAVES;

template <int QT, int PT> struct Kind {
    static constexpr bool CODES = PT == SSD_E4M3 || PT == SSD_I8, F32 = PT == SSD_F32, BF = PT != SSD_F16;
    static constexpr int SIZE = CODES ? 1 : F32 ? 4 : 2;                     // bytes of an element
    static constexpr int KEYS = CODES ? 32 : F32 ? 16 : 32, TILES = KEYS / 16;     // 64 registers a lane of keys and values in flight
    static constexpr int QN = !CODES || QT == SSD_BF16 ? 1 : QT == SSD_F16 ? 2 : 3;      // 16-bit values that a query is the exact sum of
    static constexpr int PN = QT == SSD_F32 ? 3 : 2;                         // those of a weight
    // weights are taken times 2^BIAS: in half's upper range, or so that sums of 2^30 values at the end of fp32's range stay in it
    static constexpr float BIAS = PT == SSD_F16 ? 15.f : -32.f;
};

// Two codes to a pair of bfloat16, exactly: bytes 2 H and 2 H + 1 of w.
template <int PT, bool HIGH>
__device__ __forceinline__ uint32_t code_pair(uint32_t w) {
    if constexpr (PT == SSD_E4M3) return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, HIGH));
    else {
        const float lo = (float)(int8_t)(w >> (HIGH ? 16 : 0)), hi = (float)(int8_t)(w >> (HIGH ? 24 : 8));
        return __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);
    }
}

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

struct Piece { int b, kvh, tile, from, to, len; };

template <int QT, int PT, int HD>
__global__ void __launch_bounds__(64 * WAVES, 2) paged_attn_kernel(PagedAttnArgs a) {
    typedef Kind<QT, PT> T;
    typedef Elem<QT> E;
    constexpr int KEYS = T::KEYS, TILES = T::TILES, DPL = HD / 16, DT = HD / 16, STEP = KEYS * WAVES, PITCH = HD + 4;
    constexpr int K_LOADS = HD * T::SIZE / 64, V_WORDS = DPL * T::SIZE / 4;
    __shared__ float o_s[WAVES][16][PITCH];
    __shared__ float2 ml_s[WAVES][16];
    const PagesArgs& p = a.p;
    const int lane = threadIdx.x % 64, g = lane / 16, dc = lane % 16, hd = T::F32 ? p.head_dim : HD;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int part = blockIdx.x, kvh = blockIdx.y, b = blockIdx.z / a.tiles, tile = blockIdx.z % a.tiles;
    const int given = p.ctx_len[b], len = min(max(given, 0), p.max_ctx);
    const int from = part * a.piece, to = min(len, from + a.piece);
    if (part > 0 && from >= len) return;                     // (the first piece answers for an empty context)
    const bool only = len <= a.piece;
    bool bad = given != len;

    // Pages of the wavefront's tiles: lane i has those of tile i % TILES of its block i / TILES.
    const int first = from + wave * KEYS, blocks = (to - first + STEP - 1) / STEP;
    int pages = -1;
    {
        const int key = first + lane / TILES * STEP + 16 * (lane % TILES);
        if (key < to) {
            pages = page_of(p, b, key);
            bad |= pages < 0;
        }
    }
    const int rows = a.n_new * a.group, row = min(tile * 16 + dc, rows - 1), token = row / a.group;
    const int limit = len - (a.n_new - 1 - token);           // the column's token sees the rows before it
    const int least = len - (a.n_new - 1 - min(tile * 16, rows - 1) / a.group);     // what all columns see
    Queries<QT, PT, HD> q;
    q.load(a.q, ((int64_t)b * a.n_new + token) * a.q_stride + (int64_t)(kvh * a.group + row % a.group) * hd, hd, g);

    u32x4_t kr[TILES][K_LOADS];
    constexpr int WORDS = T::F32 ? 4 : V_WORDS, V_PARTS = V_WORDS / WORDS;
    typedef uint32_t words_t __attribute__((ext_vector_type(WORDS)));
    words_t vr[TILES][4][V_PARTS];
    f32x4_t ks[T::CODES ? TILES : 1], vs[T::CODES ? TILES : 1];
    auto row_of = [&](int block, int c) {                    // first row of a tile; of pages that are none, any
        const int page = __builtin_amdgcn_readlane(pages, block * TILES + c);
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
    float m = -F32_MOST, l = 0.f;
    f32x4_t o[DT];
#pragma unroll
    for (int i = 0; i < DT; ++i) o[i] = (f32x4_t){0.f, 0.f, 0.f, 0.f};

    const bool whole = !__any(bad);
    for (int block = 0; block < blocks; ++block) {
        const int k0 = first + block * STEP;
        const bool masked = !whole || k0 + KEYS > min(least, to);
        float s[TILES][4];
#pragma unroll
        for (int c = 0; c < TILES; ++c) {
            f32x4_t x = {0.f, 0.f, 0.f, 0.f};
            if constexpr (T::F32) {
#pragma unroll
                for (int e = 0; e < K_LOADS; ++e) {
                    const f32x4_t k = __builtin_bit_cast(f32x4_t, kr[c][e]);
                    const bool there = 16 * e + 4 * g < hd;
#pragma unroll
                    for (int i = 0; i < 4; ++i) x = mfma_f32(there ? k[i] : 0.f, q.x[e][i], x);
                }
            } else if constexpr (T::CODES) {
#pragma unroll
                for (int e = 0; e < HD / 32; ++e) {
                    const uint32_t lo = kr[c][e / 2][e % 2 * 2], hi = kr[c][e / 2][e % 2 * 2 + 1];
                    const f16x8_t k = as_f16x8(make_uint4(code_pair<PT, false>(lo), code_pair<PT, true>(lo), code_pair<PT, false>(hi), code_pair<PT, true>(hi)));
#pragma unroll
                    for (int n = 0; n < T::QN; ++n) x = mfma_16x16x32<true>(k, q.x[n][e], x);
                }
            } else {
#pragma unroll
                for (int e = 0; e < HD / 32; ++e) x = mfma_16x16x32<T::BF>(__builtin_bit_cast(f16x8_t, kr[c][e]), q.x[0][e], x);
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) s[c][r] = x[r] * (T::CODES ? ks[c][r] * sc : sc);
        }
        // Keys of the lane that its column sees (bits 4 c + r), and that some column does.
        uint32_t mine = ~0u, some = ~0u;
        if (masked) {
            mine = some = 0;
#pragma unroll
            for (int c = 0; c < TILES; ++c) {
                const bool here = __builtin_amdgcn_readlane(pages, block * TILES + c) >= 0;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int j = k0 + 16 * c + 4 * g + r;
                    mine |= (uint32_t)(here && j < limit) << (4 * c + r);
                    some |= (uint32_t)(here && j < len) << (4 * c + r);
                    s[c][r] = mine >> (4 * c + r) & 1 ? s[c][r] : -INFINITY;
                }
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        const int next = min(block + 1, blocks - 1);         // (behind the last block: it again)
        load_keys(next);
        __builtin_amdgcn_sched_barrier(0);
        float top = s[0][0];
#pragma unroll
        for (int i = 1; i < 4 * TILES; ++i) top = fmaxf(top, s[i / 4][i % 4]);
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(m, fmaxf(top, __shfl_xor(top, 32)));
        if (__any(top > m)) {
            const float alpha = __builtin_amdgcn_exp2f(m - top);
            l *= alpha;
#pragma unroll
            for (int i = 0; i < DT; ++i) o[i] *= alpha;
            m = top;
        }
        const float base = T::BIAS - m;
#pragma unroll
        for (int c = 0; c < TILES; ++c)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                s[c][r] = __builtin_amdgcn_exp2f(s[c][r] + base);
                l += s[c][r];
                if (T::CODES) s[c][r] *= vs[c][r];
            }
        if (masked) {
            // Weights of rows that the column does not see are zeros, whatever their scales hold; rows that no column sees become zeros, whatever they hold.
            bool odd = false;
#pragma unroll
            for (int c = 0; c < TILES; ++c)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    if (T::CODES) s[c][r] = mine >> (4 * c + r) & 1 ? s[c][r] : 0.f;
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
                        const float seen = mine >> (4 * c + r) & 1 ? 1.f : 0.f;
#pragma unroll
                        for (int i = 0; i < DT; ++i) {
                            const uint32_t x = vr[c][r][T::F32 ? i / 4 : 0][T::F32 ? i % 4 : i * T::SIZE / 4];
                            const bool is = not_finite<PT>(x) >> (T::SIZE == 1 ? 8 * (i % 4) + 7 : T::SIZE == 2 ? 16 * (i % 2) + 15 : 31) & 1;
                            const f32x4_t n = mfma_f32(is ? 1.f : 0.f, seen, (f32x4_t){0.f, 0.f, 0.f, 0.f});
#pragma unroll
                            for (int e = 0; e < 4; ++e) o[i][e] += n[e] > 0.f ? NAN : 0.f;
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
                for (int i = 0; i < DT; ++i) o[i] = mfma_f32(__uint_as_float(vr[0][r][i / 4][i % 4]), s[0][r], o[i]);
        } else {
#pragma unroll
            for (int h = 0; h < TILES / 2; ++h) {            // 32 keys
                f16x8_t w[T::PN];
#pragma unroll
                for (int n = 0; n < T::PN; ++n) {
                    uint32_t x[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        float& lo = s[2 * h + e / 2][e % 2 * 2];
                        float& hi = s[2 * h + e / 2][e % 2 * 2 + 1];
                        x[e] = pack16<T::BF>(lo, hi);
                        const f16x2_t z = __builtin_bit_cast(f16x2_t, x[e]);
                        lo -= T::BF ? __uint_as_float(x[e] << 16) : (float)z.x;
                        hi -= T::BF ? __uint_as_float(x[e] & 0xffff0000u) : (float)z.y;
                    }
                    w[n] = as_f16x8(make_uint4(x[0], x[1], x[2], x[3]));
                }
                auto add = [&](int i, uint32_t x0, uint32_t x1, uint32_t x2, uint32_t x3) __attribute__((always_inline)) {
                    const f16x8_t x = as_f16x8(make_uint4(x0, x1, x2, x3));
#pragma unroll
                    for (int n = 0; n < T::PN; ++n) o[i] = mfma_16x16x32<T::BF>(x, w[n], o[i]);
                };
                const auto& v0 = vr[2 * h];
                const auto& v1 = vr[2 * h + 1];
                if constexpr (T::CODES) {
#pragma unroll
                    for (int i = 0; i < DT; i += 2) {        // bytes i, i + 1 of two rows side by side
                        const uint32_t pick = i % 4 ? 0x07030602u : 0x05010400u;
                        uint32_t t[4];
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            t[e] = __builtin_amdgcn_perm(v0[2 * e + 1][0][i / 4], v0[2 * e][0][i / 4], pick);
                            t[2 + e] = __builtin_amdgcn_perm(v1[2 * e + 1][0][i / 4], v1[2 * e][0][i / 4], pick);
                        }
                        add(i, code_pair<PT, false>(t[0]), code_pair<PT, false>(t[1]), code_pair<PT, false>(t[2]), code_pair<PT, false>(t[3]));
                        add(i + 1, code_pair<PT, true>(t[0]), code_pair<PT, true>(t[1]), code_pair<PT, true>(t[2]), code_pair<PT, true>(t[3]));
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
        }
        __builtin_amdgcn_sched_barrier(0);
        load_values(next);
        __builtin_amdgcn_sched_barrier(0);
    }

    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    const float inv = l == 0.f ? 0.f : 1.f / l;
    if (g == 0) ml_s[wave][dc] = make_float2(m, l);
#pragma unroll
    for (int i = 0; i < DT; i += 4)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int dim = T::F32 ? 16 * i + 16 * g + 4 * r : DPL * (4 * g + r) + i;
            *reinterpret_cast<f32x4_t*>(&o_s[wave][dc][dim]) = (f32x4_t){o[i][r] * inv, o[i + 1][r] * inv, o[i + 2][r] * inv, o[i + 3][r] * inv};
        }
    __syncthreads();
    constexpr int PER = HD / 4;                              // threads of a row
    for (int i = threadIdx.x; i < 16 * PER; i += 64 * WAVES) {
        const int r = i / PER, dim = i % PER * 4, n = tile * 16 + r;
        if (n >= rows || dim >= hd) continue;
        float mt = -F32_MOST, lt = 0.f, w[WAVES];
#pragma unroll
        for (int u = 0; u < WAVES; ++u) mt = fmaxf(mt, ml_s[u][r].x);
#pragma unroll
        for (int u = 0; u < WAVES; ++u) {
            const float2 x = ml_s[u][r];
            w[u] = x.y == 0.f ? 0.f : x.y * __builtin_amdgcn_exp2f(x.x - mt);
            lt += w[u];
        }
        const float share = lt == 0.f ? 0.f : 1.f / lt;
        f32x4_t v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int u = 0; u < WAVES; ++u) v += *reinterpret_cast<const f32x4_t*>(&o_s[u][r][dim]) * (w[u] * share);
        const int64_t at = ((int64_t)b * a.n_new + n / a.group) * a.n_q_heads + kvh * a.group + n % a.group;
        if (only) {
            typename E::type* out = (typename E::type*)a.out + at * hd + dim;
#pragma unroll
            for (int e = 0; e < 4; ++e) out[e] = E::put(v[e]);
            if (a.lse && dim == 0) a.lse[at] = lt == 0.f ? -INFINITY : (mt - T::BIAS + __builtin_amdgcn_logf(lt)) * LN2;
        } else {
            *reinterpret_cast<f32x4_t*>(a.part_o + (at * a.n_pieces + part) * HD + dim) = v;
            if (dim == 0) a.part_ml[at * a.n_pieces + part] = make_float2(mt - T::BIAS, lt);
        }
    }
    if (bad) raise_flag(p.flags, SSD_FLAG_BAD_PAGE);
}

// The pieces of a context, a mean of values each, joined: a workgroup has a query row, groups of HD / 4 lanes take its pieces in turn and are joined through LDS.
template <int QT, int HD>
__global__ void __launch_bounds__(256) paged_join_kernel(PagedAttnArgs a) {
    typedef Elem<QT> E;
    constexpr int LANES = HD / 4, GROUPS = 256 / LANES, U = 4;
    __shared__ f32x4_t o_s[GROUPS][LANES];
    __shared__ float2 ml_s[GROUPS];
    const int64_t at = blockIdx.x;
    const int b = (int)(at / ((int64_t)a.n_new * a.n_q_heads)), len = min(max(a.p.ctx_len[b], 0), a.p.max_ctx), pieces = (len + a.piece - 1) / a.piece;
    if (pieces <= 1) return;
    const int group = threadIdx.x / LANES, dim = threadIdx.x % LANES * 4;
    const float2* ml = a.part_ml + at * a.n_pieces;
    const float* po = a.part_o + at * a.n_pieces * HD + dim;
    float m = -F32_MOST, l = 0.f;
    f32x4_t v = {0.f, 0.f, 0.f, 0.f};
    for (int p0 = group; p0 < pieces; p0 += U * GROUPS) {
        float2 y[U];
        f32x4_t z[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t i = min(p0 + u * GROUPS, pieces - 1);
            y[u] = ml[i];
            z[u] = *reinterpret_cast<const f32x4_t*>(po + i * HD);
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
    o_s[group][dim / 4] = v;
    if (dim == 0) ml_s[group] = make_float2(m, l);
    __syncthreads();
    if (group || dim >= a.p.head_dim) return;
    float mt = -F32_MOST, lt = 0.f, f[GROUPS];
#pragma unroll
    for (int i = 0; i < GROUPS; ++i) mt = fmaxf(mt, ml_s[i].x);
#pragma unroll
    for (int i = 0; i < GROUPS; ++i) {
        const float2 y = ml_s[i];
        f[i] = y.y == 0.f ? 0.f : y.y * __builtin_amdgcn_exp2f(y.x - mt);
        lt += f[i];
    }
    const float inv = lt == 0.f ? 0.f : 1.f / lt;
    f32x4_t s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < GROUPS; ++i) s += o_s[i][dim / 4] * (f[i] * inv);
    typename E::type* out = (typename E::type*)a.out + at * a.p.head_dim + dim;
#pragma unroll
    for (int e = 0; e < 4; ++e) out[e] = E::put(s[e]);
    if (a.lse && dim == 0) a.lse[at] = lt == 0.f ? -INFINITY : (mt + __builtin_amdgcn_logf(lt)) * LN2;
}

template <int QT, int PT, int HD>
void launch_rows(const PagedAttnArgs& a, hipStream_t st) {
    paged_attn_kernel<QT, PT, HD><<<dim3(a.n_pieces, a.p.n_kv_heads, a.p.B * a.tiles), 64 * WAVES, 0, st>>>(a);
    if (a.n_pieces > 1) paged_join_kernel<QT, HD><<<(unsigned)((int64_t)a.p.B * a.n_new * a.n_q_heads), 256, 0, st>>>(a);
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
