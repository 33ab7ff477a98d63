// Rows of a slot cache to pages and back, as they are or by 8-bit codes with a scale per row and head (definitions in ssd.h).  A workgroup takes consecutive rows of
// an utterance (or of short ones side by side), HEADS heads of each: a thread finds its row's places once, requests the heads' values together and has 8 elements of each.
// Four heads, or one where that makes few workgroups (64 rows of 8 heads of 128, half to e4m3: 3.9 and 3.3 us; 24 layers of 6 utterances of 200 to 400 rows, half to int8, with two
// heads 81 us, four 59, eight 57; 2 layers of 65537 rows, bfloat16 to e4m3, 172, 157, 158; back from e4m3, 24 layers, 70, 58, 58).
// Every row is read and written once, 16 bytes a load, past the caches (with ordinary loads and stores 24 layers to int8 take 64 us for 59, as they are 78 for 70, fp32 146 for 129; long runs
// of rows 158 for 157): what bounds it is memory, at 4.7 TB/s for int8 and 5.2 for long runs of rows.
#include <algorithm>

#include "pages.h"
#include "tree_attn.h"

namespace ssd {

namespace {


// Work of a launch: blockIdx.x = ((slice * n_layers) + layer) * 2 + (0 keys, 1 values), blockIdx.y the utterance where rows of one fill a workgroup.
struct Slice { int layer, which, index, count; };
__device__ __forceinline__ Slice slice_of(const MoveArgs& a) {
    const int which = blockIdx.x % 2, rest = blockIdx.x / 2;
    return Slice{rest % a.n_layers, which, rest / a.n_layers, (int)(gridDim.x / 2 / a.n_layers)};
}
// Units of rows_at_once rows times HEADS heads.
template <int HEADS> __device__ __forceinline__ int head_units(const MoveArgs& a) { return (a.p.n_kv_heads + HEADS - 1) / HEADS; }
__device__ __forceinline__ int64_t row_units(const MoveArgs& a, int rows_at_once) {
    const int64_t rows = gridDim.y > 1 || a.p.B == 1 ? a.max_rows : (int64_t)a.p.B * a.max_rows;
    return (rows + rows_at_once - 1) / rows_at_once;
}

// Where a row lies on either side, head 0; false: there is none.  here: it is not left out (else both places are some row's: what lies there may be requested, as
// the row's values are while its page number is on the way).
struct Place { int64_t slot, row; bool here; };
__device__ __forceinline__ bool place_of(const MoveArgs& a, int64_t index, int layer, Place& at, bool& bad) {
    int b = blockIdx.y, i = (int)index;
    if (gridDim.y == 1 && a.p.B > 1) {                       // (fewer than 2^31 rows in all)
        b = (uint32_t)index / (uint32_t)a.max_rows;
        i = (int)index - b * a.max_rows;
    }
    if (b >= a.p.B || i >= a.max_rows) return false;
    const int given = a.n_rows ? a.n_rows[b] : a.max_rows, n = min(max(given, 0), a.max_rows), len = a.p.ctx_len[b];
    const int64_t slot = (a.start ? (int64_t)a.start[b] : (int64_t)b * a.max_rows) + i, j = (int64_t)len - n + i;
    bad |= given != n;
    if (i >= n) return false;
    const bool inside = slot >= 0 && slot < a.slots && j >= 0 && j < a.p.max_ctx;
    const int page = page_of(a.p, b, inside ? (int)j : 0);
    at.here = inside && page >= 0;
    at.slot = layer * a.layer_stride + (inside ? slot : 0) * a.slot_stride;
    at.row = layer * a.p.layer_rows + row_in_pages(a.p, max(page, 0), 0, inside ? (int)j : 0);
    bad |= !at.here;
    return true;
}

// Eight consecutive elements, 16 bytes at a time.
template <int DT> struct Eight { uint4 w[DT == SSD_F32 ? 2 : 1]; };
template <int DT>
__device__ __forceinline__ Eight<DT> load8(const typename Elem<DT>::type* p) {
    Eight<DT> x;
#pragma unroll
    for (int i = 0; i < (DT == SSD_F32 ? 2 : 1); ++i) x.w[i] = __builtin_bit_cast(uint4, __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(p) + i));
    return x;
}
template <int DT>
__device__ __forceinline__ void values_of(const Eight<DT>& x, float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint4& q = x.w[DT == SSD_F32 ? i / 4 : 0];
        const int k = DT == SSD_F32 ? i % 4 : i / 2;
        const uint32_t w = k == 0 ? q.x : k == 1 ? q.y : k == 2 ? q.z : q.w;
        if constexpr (DT == SSD_F32) v[i] = __uint_as_float(w);
        else v[i] = Elem<DT>::get((uint16_t)(i % 2 ? w >> 16 : w));
    }
}

// Largest magnitude (as bits, so that NaN is the largest) over the lanes of a row.
template <int LANES>
__device__ __forceinline__ uint32_t row_max(const float (&x)[8]) {
    int top = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) top = max(top, (int)(__float_as_uint(x[e]) & 0x7fffffffu));
    top = max(top, dpp_i<DPP_XOR1>(top));
    top = max(top, dpp_i<DPP_XOR2>(top));
    top = max(top, dpp_i<DPP_HALF_MIRROR>(top));
    if (LANES == 16) top = max(top, dpp_i<DPP_MIRROR>(top));
    return (uint32_t)top;
}

// e4m3: x / 2^k is exact, the conversion rounds to nearest even.
__device__ __forceinline__ uint2 e4m3_codes(float (&x)[8], uint32_t top, float& scale) {
    const int k = max((int)(top >> 23) - 127 - 8 + ((top & 0x7fffffu) > 0x600000u), -126);     // 448 = 1.75 * 2^8
    const float inverse = __uint_as_float((uint32_t)(127 - k) << 23);
    scale = __uint_as_float((uint32_t)(127 + k) << 23);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] *= inverse;
    if (k == 120) {                                          // (256 would be worth 2^128)
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = __builtin_amdgcn_fmed3f(x[e], -240.f, 240.f);
    }
    int w[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        w[h] = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * h], x[4 * h + 1], 0, false);
        w[h] = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * h + 2], x[4 * h + 3], w[h], true);
    }
    return make_uint2((uint32_t)w[0], (uint32_t)w[1]);
}

// int8: 127 x / a to the nearest whole number, halves to even.  Added to 1.5 * 2^23 the product of x and 127 / a, rounded once, is rounded to that and has it in its low
// byte.  It is off by less than 2^-15; where what was rounded away is that near to a half, the exact products decide: both sides have at most 32 bits.
constexpr float I8_MOST_SCALE = 0x1.020406p+121f;            // the largest of which 127 times is finite
__device__ __forceinline__ uint2 i8_codes(float (&x)[8], uint32_t top, float& scale) {
    float a = __uint_as_float(top);
    scale = fminf(a / 127.f, I8_MOST_SCALE);
    if (a < 0x1p-100f) {                                     // (127 / a would not be finite)
        a *= 0x1p100f;
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] *= 0x1p100f;
    }
    const float inverse = 127.f / a;
    constexpr float MAGIC = 12582912.f;
    float c[8], far = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        c[e] = fmaf(x[e], inverse, MAGIC);
        far = fmaxf(far, fabsf(fmaf(x[e], inverse, MAGIC - c[e])));
    }
    if (far > 0.5f - 0x1p-14f) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float t = x[e] * inverse, low = floorf(t);
            if (fabsf(t - low - 0.5f) < 0x1p-13f) {
                const double d = 254.0 * (double)x[e] - (2.0 * (double)low + 1.0) * (double)a;
                c[e] = low + MAGIC + (d > 0.0 ? 1.f : d < 0.0 ? 0.f : fabsf(fmodf(low, 2.f)));
            }
        }
    }
    uint32_t w[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint32_t lo = __builtin_amdgcn_perm(__float_as_uint(c[4 * h + 1]), __float_as_uint(c[4 * h]), 0x0c0c0400u);
        const uint32_t hi = __builtin_amdgcn_perm(__float_as_uint(c[4 * h + 3]), __float_as_uint(c[4 * h + 2]), 0x04000c0cu);
        w[h] = lo | hi;
    }
    return make_uint2(w[0], w[1]);
}

template <int DT, int PT, int HD, int HEADS>
__global__ void __launch_bounds__(256) write_pages_kernel(MoveArgs a) {
    constexpr int LANES = HD / 8, ROWS = 256 / LANES;
    typedef typename Elem<DT>::type T;
    const Slice s = slice_of(a);
    const int lane = threadIdx.x % LANES, H = a.p.n_kv_heads, heads = head_units<HEADS>(a);
    const int64_t units = row_units(a, ROWS) * heads;
    const T* from = (const T*)(s.which ? a.v : a.k) + lane * 8;
    uint8_t* codes = (uint8_t*)(s.which ? a.p.v : a.p.k) + lane * 8;
    float* scales = s.which ? a.p.v_scale : a.p.k_scale;
    bool bad = false, odd = false;
    for (int64_t u = s.index; u < units; u += s.count) {
        const int h0 = (int)(u % heads) * HEADS;
        Place at;
        if (!place_of(a, u / heads * ROWS + threadIdx.x / LANES, s.layer, at, bad)) continue;
        Eight<DT> raw[HEADS];
#pragma unroll
        for (int h = 0; h < HEADS; ++h) raw[h] = load8<DT>(from + at.slot + (int64_t)min(h0 + h, H - 1) * a.head_stride);
        if (!at.here) continue;
#pragma unroll
        for (int h = 0; h < HEADS; ++h) {
            if (h0 + h >= H) break;
            float x[8], scale = 0.f;
            values_of<DT>(raw[h], x);
            const uint32_t top = row_max<LANES>(x);
            uint2 w = make_uint2(0u, 0u);
            if (top >= 0x7f800000u) {
                odd = true;
                scale = __uint_as_float(0x7fc00000u);
            } else if (top) w = PT == SSD_E4M3 ? e4m3_codes(x, top, scale) : i8_codes(x, top, scale);
            const int64_t row = at.row + ((int64_t)(h0 + h) << a.p.row_bits);
            __builtin_nontemporal_store(__builtin_bit_cast(u32x2_t, w), reinterpret_cast<u32x2_t*>(codes + row * HD));
            if (lane == 0) scales[row] = scale;
        }
    }
    if (odd && lane == 0) raise_flag(a.p.flags, SSD_FLAG_ACT_OVERFLOW);
    if (bad && lane == 0) raise_flag(a.p.flags, SSD_FLAG_BAD_PAGE);
}

// Eight values to the slots' type, side by side (fp32: four, and four half a row on).
template <int DT, int HD>
__device__ __forceinline__ void store8(typename Elem<DT>::type* p, float (&x)[8], bool& odd) {
    if constexpr (DT == SSD_F32) {
#pragma unroll
        for (int h = 0; h < 2; ++h) __builtin_nontemporal_store((f32x4_t){x[4 * h], x[4 * h + 1], x[4 * h + 2], x[4 * h + 3]}, reinterpret_cast<f32x4_t*>(p + h * HD / 2));
    } else {
        if (DT == SSD_F16) {
            bool over = false;
#pragma unroll
            for (int e = 0; e < 8; ++e) over |= !(fabsf(x[e]) <= F16_MAX);
            if (over) {
                odd = true;
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = x[e] != x[e] ? x[e] : fminf(fmaxf(x[e], -F16_MAX), F16_MAX);
            }
        }
        constexpr bool BF = DT == SSD_BF16;
        __builtin_nontemporal_store((u32x4_t){pack16<BF>(x[0], x[1]), pack16<BF>(x[2], x[3]), pack16<BF>(x[4], x[5]), pack16<BF>(x[6], x[7])}, reinterpret_cast<u32x4_t*>(p));
    }
}

template <int DT, int PT, int HD, int HEADS>
__global__ void __launch_bounds__(256) read_pages_kernel(MoveArgs a) {
    constexpr int LANES = HD / 8, ROWS = 256 / LANES;
    typedef typename Elem<DT>::type T;
    const Slice s = slice_of(a);
    const int lane = threadIdx.x % LANES, H = a.p.n_kv_heads, heads = head_units<HEADS>(a);
    const int64_t units = row_units(a, ROWS) * heads;
    constexpr bool F32 = DT == SSD_F32;                      // four elements in either half of the row, so that a store of all lanes is one piece of memory (24 layers 110 -> 90 us)
    T* to = (T*)(s.which ? a.v : a.k) + lane * (F32 ? 4 : 8);
    const uint8_t* codes = (const uint8_t*)(s.which ? a.p.v : a.p.k) + lane * (F32 ? 4 : 8);
    const float* scales = s.which ? a.p.v_scale : a.p.k_scale;
    bool bad = false, odd = false;
    for (int64_t u = s.index; u < units; u += s.count) {
        const int h0 = (int)(u % heads) * HEADS;
        Place at;
        if (!place_of(a, u / heads * ROWS + threadIdx.x / LANES, s.layer, at, bad)) continue;
        uint2 raw[HEADS];
        float scale[HEADS];
#pragma unroll
        for (int h = 0; h < HEADS; ++h) {
            const int64_t row = at.row + ((int64_t)min(h0 + h, H - 1) << a.p.row_bits);
            if constexpr (F32) {
                raw[h].x = __builtin_nontemporal_load(reinterpret_cast<const uint32_t*>(codes + row * HD));
                raw[h].y = __builtin_nontemporal_load(reinterpret_cast<const uint32_t*>(codes + row * HD + HD / 2));
            } else raw[h] = __builtin_bit_cast(uint2, __builtin_nontemporal_load(reinterpret_cast<const u32x2_t*>(codes + row * HD)));
            scale[h] = scales[row];
        }
        if (!at.here) continue;
#pragma unroll
        for (int h = 0; h < HEADS; ++h) {
            if (h0 + h >= H) break;
            float x[8];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const uint32_t c = e ? raw[h].y : raw[h].x;
                if constexpr (PT == SSD_E4M3) {
                    const f32x2_t lo = __builtin_amdgcn_cvt_pk_f32_fp8(c, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(c, true);
                    x[4 * e] = lo.x; x[4 * e + 1] = lo.y; x[4 * e + 2] = hi.x; x[4 * e + 3] = hi.y;
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i) x[4 * e + i] = (float)(int8_t)(c >> (8 * i));
                }
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] *= scale[h];
            store8<DT, HD>(to + at.slot + (int64_t)(h0 + h) * a.head_stride, x, odd);
        }
    }
    if (odd) raise_flag(a.p.flags, SSD_FLAG_ACT_OVERFLOW);
    if (bad && lane == 0) raise_flag(a.p.flags, SSD_FLAG_BAD_PAGE);
}

// Rows as they are: `chunks` of 16 bytes, a thread each of 1 << bits (those behind the row's end idle).
template <bool WRITE, int HEADS>
__global__ void __launch_bounds__(256) copy_pages_kernel(MoveArgs a, int chunks, int bits, int size) {
    const Slice s = slice_of(a);
    const int lane = threadIdx.x & ((1 << bits) - 1), rows = 256 >> bits, H = a.p.n_kv_heads, heads = head_units<HEADS>(a);
    const int64_t units = row_units(a, rows) * heads;
    char* slots = (char*)(s.which ? a.v : a.k) + lane * 16;
    char* pages = (char*)(s.which ? a.p.v : a.p.k) + lane * 16;
    bool bad = false;
    for (int64_t u = s.index; u < units; u += s.count) {
        const int h0 = (int)(u % heads) * HEADS;
        Place at;
        if (!place_of(a, u / heads * rows + (threadIdx.x >> bits), s.layer, at, bad) || lane >= chunks) continue;
        u32x4_t x[HEADS];
        auto slot_at = [&](int h) { return reinterpret_cast<u32x4_t*>(slots + (at.slot + (int64_t)h * a.head_stride) * size); };
        auto page_at = [&](int h) { return reinterpret_cast<u32x4_t*>(pages + (at.row + ((int64_t)h << a.p.row_bits)) * a.p.head_dim * size); };
#pragma unroll
        for (int h = 0; h < HEADS; ++h) x[h] = __builtin_nontemporal_load(WRITE ? slot_at(min(h0 + h, H - 1)) : page_at(min(h0 + h, H - 1)));
        if (!at.here) continue;
#pragma unroll
        for (int h = 0; h < HEADS; ++h)
            if (h0 + h < H) __builtin_nontemporal_store(x[h], WRITE ? page_at(h0 + h) : slot_at(h0 + h));
    }
    if (bad && lane == 0) raise_flag(a.p.flags, SSD_FLAG_BAD_PAGE);
}

// rows: of a workgroup at a time.  Utterances of fewer lie side by side.
struct Launch { dim3 grid; bool one; };
Launch launch_of(const MoveArgs& a, int rows) {
    const bool beside = a.max_rows < rows;
    const int64_t all = beside ? (int64_t)a.p.B * a.max_rows : a.max_rows, utts = beside ? 1 : a.p.B, pairs = 2 * (int64_t)a.n_layers;
    const int64_t groups = (all + rows - 1) / rows;
    const bool one = groups * a.p.n_kv_heads * pairs * utts <= 512;
    const int64_t units = groups * (one ? a.p.n_kv_heads : (a.p.n_kv_heads + 3) / 4), slices = std::max<int64_t>(1, std::min(units, 32768 / (pairs * utts)));
    return Launch{dim3((unsigned)(slices * pairs), (unsigned)utts), one};
}

template <int DT, int PT, int HD>
void launch_codes(const MoveArgs& a, bool write, hipStream_t st) {
    const Launch l = launch_of(a, 256 / (HD / 8));
    if (write && l.one) write_pages_kernel<DT, PT, HD, 1><<<l.grid, 256, 0, st>>>(a);
    else if (write) write_pages_kernel<DT, PT, HD, 4><<<l.grid, 256, 0, st>>>(a);
    else if (l.one) read_pages_kernel<DT, PT, HD, 1><<<l.grid, 256, 0, st>>>(a);
    else read_pages_kernel<DT, PT, HD, 4><<<l.grid, 256, 0, st>>>(a);
}
template <int DT, int PT>
void launch_dims(const MoveArgs& a, bool write, hipStream_t st) {
    if (a.p.head_dim == 128) launch_codes<DT, PT, 128>(a, write, st);
    else launch_codes<DT, PT, 64>(a, write, st);
}
template <int PT>
void launch_type(const MoveArgs& a, int dtype, bool write, hipStream_t st) {
    if (dtype == SSD_F32) launch_dims<SSD_F32, PT>(a, write, st);
    else if (dtype == SSD_BF16) launch_dims<SSD_BF16, PT>(a, write, st);
    else launch_dims<SSD_F16, PT>(a, write, st);
}
void launch_move(const MoveArgs& a, int dtype, int pages_dtype, bool write, hipStream_t st) {
    if (pages_dtype == SSD_E4M3) return launch_type<SSD_E4M3>(a, dtype, write, st);
    if (pages_dtype == SSD_I8) return launch_type<SSD_I8>(a, dtype, write, st);
    const int size = dtype == SSD_F32 ? 4 : 2, chunks = a.p.head_dim * size / 16;
    int bits = 0;
    while (1 << bits < chunks) ++bits;
    const Launch l = launch_of(a, 256 >> bits);
    if (write && l.one) copy_pages_kernel<true, 1><<<l.grid, 256, 0, st>>>(a, chunks, bits, size);
    else if (write) copy_pages_kernel<true, 4><<<l.grid, 256, 0, st>>>(a, chunks, bits, size);
    else if (l.one) copy_pages_kernel<false, 1><<<l.grid, 256, 0, st>>>(a, chunks, bits, size);
    else copy_pages_kernel<false, 4><<<l.grid, 256, 0, st>>>(a, chunks, bits, size);
}

}  // namespace

void launch_write_pages(const MoveArgs& a, int dtype, int pages_dtype, hipStream_t st) { launch_move(a, dtype, pages_dtype, true, st); }
void launch_read_pages(const MoveArgs& a, int dtype, int pages_dtype, hipStream_t st) { launch_move(a, dtype, pages_dtype, false, st); }

}  // namespace ssd
