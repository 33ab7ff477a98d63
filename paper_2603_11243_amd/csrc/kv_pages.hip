// Rows of a slot cache to pages and back, as they are or by 8-bit codes with a scale per row and head (definitions in ssd.h).
#include <algorithm>

#include "pages.h"
#include "tree_attn.h"

namespace ssd {

namespace {

// The row of a thread's group of lanes: where it lies on either side, or that it is left out.
struct Place { int64_t slot, row; };
__device__ __forceinline__ bool place_of(const MoveArgs& a, int b, int i, int head, int layer, int n, Place& at, bool& bad) {
    const int64_t slot = (a.start ? (int64_t)a.start[b] : (int64_t)b * a.max_rows) + i;
    const int64_t j = (int64_t)a.p.ctx_len[b] - n + i;
    if (slot < 0 || slot >= a.slots || j < 0 || j >= a.p.max_ctx) { bad = true; return false; }
    const int page = page_of(a.p, b, (int)j);
    if (page < 0) { bad = true; return false; }
    at.slot = layer * a.layer_stride + slot * a.slot_stride + head * a.head_stride;
    at.row = layer * a.p.layer_rows + row_in_pages(a.p, page, head, (int)j);
    return true;
}
__device__ __forceinline__ int rows_of(const MoveArgs& a, int b, bool& bad) {
    const int n = a.n_rows ? a.n_rows[b] : a.max_rows;
    bad |= n < 0 || n > a.max_rows;
    return min(max(n, 0), a.max_rows);
}

// Eight consecutive elements as fp32.
template <int DT>
__device__ __forceinline__ void load8(const typename Elem<DT>::type* p, float (&x)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = Elem<DT>::get(p[e]);
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

// Scale 2^k of a row, its inverse, and the largest magnitude of what is rounded: code 256 of scale 2^120 would be worth 2^128.
__device__ __forceinline__ float e4m3_scale(uint32_t top, float& inverse, float& most) {
    const int k = max((int)(top >> 23) - 127 - 8 + ((top & 0x7fffffu) > 0x600000u), -126);     // 448 = 1.75 * 2^8
    inverse = __uint_as_float((uint32_t)(127 - k) << 23);
    most = k == 120 ? 240.f : 448.f;
    return __uint_as_float((uint32_t)(127 + k) << 23);
}

// 127 x / a to the nearest whole number, halves to even.  The fp32 product is off by less than 2^-15; where it lies that near to a half the exact products decide:
// both sides of the comparison have at most 32 bits.
__device__ __forceinline__ int i8_code(float x, float a, float inverse) {
    const float t = x * inverse, low = floorf(t), part = t - low;
    if (fabsf(part - 0.5f) > 0x1p-14f) return (int)rintf(t);
    const double d = 254.0 * (double)x - (2.0 * (double)low + 1.0) * (double)a;
    const int n = (int)low;
    return d > 0.0 ? n + 1 : d < 0.0 ? n : n + (n & 1);
}
constexpr float I8_MOST_SCALE = 0x1.020406p+121f;            // the largest of which 127 times is finite

template <int DT, int PT, int HD>
__global__ void __launch_bounds__(256) write_pages_kernel(MoveArgs a) {
    constexpr int LANES = HD / 8, GROUPS = 256 / LANES;
    const int b = blockIdx.y, which = blockIdx.x % 2, layer = blockIdx.x / 2 % a.n_layers, part = blockIdx.x / 2 / a.n_layers;
    const int parts = gridDim.x / 2 / a.n_layers, lane = threadIdx.x % LANES, H = a.p.n_kv_heads;
    bool bad = false, odd = false;
    const int n = rows_of(a, b, bad);
    typedef typename Elem<DT>::type T;
    const T* from = (const T*)(which ? a.v : a.k);
    uint8_t* codes = (uint8_t*)(which ? a.p.v : a.p.k);
    float* scales = which ? a.p.v_scale : a.p.k_scale;
    for (int64_t i = (int64_t)part * GROUPS + threadIdx.x / LANES; i < (int64_t)n * H; i += (int64_t)parts * GROUPS) {
        Place at;
        if (!place_of(a, b, (int)(i / H), (int)(i % H), layer, n, at, bad)) continue;
        float x[8];
        load8<DT>(from + at.slot + lane * 8, x);
        const uint32_t top = row_max<LANES>(x);
        uint32_t w[2] = {0, 0};
        float scale = 0.f;
        if (top >= 0x7f800000u) {
            odd = true;
            scale = __uint_as_float(0x7fc00000u);
        } else if (top) {
            if constexpr (PT == SSD_E4M3) {
                float inverse, most;
                scale = e4m3_scale(top, inverse, most);
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = __builtin_amdgcn_fmed3f(x[e] * inverse, -most, most);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    int v = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * h], x[4 * h + 1], 0, false);
                    w[h] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[4 * h + 2], x[4 * h + 3], v, true);
                }
            } else {
                const float most = __uint_as_float(top), lift = most < 0x1p-100f ? 0x1p100f : 1.f;     // (so that 127 / most is finite)
                scale = fminf(most / 127.f, I8_MOST_SCALE);
                const float inverse = 127.f / (most * lift);
#pragma unroll
                for (int e = 0; e < 8; ++e) w[e / 4] |= (uint32_t)(i8_code(x[e] * lift, most * lift, inverse) & 255) << (8 * (e % 4));
            }
        }
        *reinterpret_cast<uint2*>(codes + at.row * HD + lane * 8) = make_uint2(w[0], w[1]);
        if (lane == 0) scales[at.row] = scale;
    }
    if (odd && lane == 0) raise_flag(a.p.flags, SSD_FLAG_ACT_OVERFLOW);
    if (bad && lane == 0) raise_flag(a.p.flags, SSD_FLAG_BAD_PAGE);
}

// Eight values to the slots' type.
template <int DT>
__device__ __forceinline__ void store8(typename Elem<DT>::type* p, const float (&x)[8], bool& odd) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        float v = x[e];
        if (DT == SSD_F16) {
            odd |= !(fabsf(v) <= F16_MAX);
            v = v != v ? v : fminf(fmaxf(v, -F16_MAX), F16_MAX);
        }
        p[e] = Elem<DT>::put(v);
    }
}

template <int DT, int PT, int HD>
__global__ void __launch_bounds__(256) read_pages_kernel(MoveArgs a) {
    constexpr int LANES = HD / 8, GROUPS = 256 / LANES;
    const int b = blockIdx.y, which = blockIdx.x % 2, layer = blockIdx.x / 2 % a.n_layers, part = blockIdx.x / 2 / a.n_layers;
    const int parts = gridDim.x / 2 / a.n_layers, lane = threadIdx.x % LANES, H = a.p.n_kv_heads;
    bool bad = false, odd = false;
    const int n = rows_of(a, b, bad);
    typedef typename Elem<DT>::type T;
    T* to = (T*)(which ? a.v : a.k);
    const uint8_t* codes = (const uint8_t*)(which ? a.p.v : a.p.k);
    const float* scales = which ? a.p.v_scale : a.p.k_scale;
    for (int64_t i = (int64_t)part * GROUPS + threadIdx.x / LANES; i < (int64_t)n * H; i += (int64_t)parts * GROUPS) {
        Place at;
        if (!place_of(a, b, (int)(i / H), (int)(i % H), layer, n, at, bad)) continue;
        const uint2 w = *reinterpret_cast<const uint2*>(codes + at.row * HD + lane * 8);
        const float scale = scales[at.row];
        float x[8];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint32_t c = h ? w.y : w.x;
            if constexpr (PT == SSD_E4M3) {
                const f32x2_t lo = __builtin_amdgcn_cvt_pk_f32_fp8(c, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(c, true);
                x[4 * h] = lo.x * scale; x[4 * h + 1] = lo.y * scale; x[4 * h + 2] = hi.x * scale; x[4 * h + 3] = hi.y * scale;
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) x[4 * h + e] = (float)(int8_t)(c >> (8 * e)) * scale;
            }
        }
        store8<DT>(to + at.slot + lane * 8, x, odd);
    }
    if (odd) raise_flag(a.p.flags, SSD_FLAG_ACT_OVERFLOW);
    if (bad && lane == 0) raise_flag(a.p.flags, SSD_FLAG_BAD_PAGE);
}

// Rows as they are, 16 bytes a thread.
template <bool WRITE>
__global__ void __launch_bounds__(256) copy_pages_kernel(MoveArgs a, int chunks, int size) {
    const int b = blockIdx.y, which = blockIdx.x % 2, layer = blockIdx.x / 2 % a.n_layers, part = blockIdx.x / 2 / a.n_layers;
    const int parts = gridDim.x / 2 / a.n_layers, H = a.p.n_kv_heads;
    bool bad = false;
    const int n = rows_of(a, b, bad);
    char* slots = (char*)(which ? a.v : a.k);
    char* pages = (char*)(which ? a.p.v : a.p.k);
    const int64_t all = (int64_t)n * H * chunks;
    for (int64_t i = (int64_t)part * 256 + threadIdx.x; i < all; i += (int64_t)parts * 256) {
        const int chunk = (int)(i % chunks);
        const int64_t rh = i / chunks;
        Place at;
        if (!place_of(a, b, (int)(rh / H), (int)(rh % H), layer, n, at, bad)) continue;
        uint4* s = reinterpret_cast<uint4*>(slots + at.slot * size) + chunk;
        uint4* p = reinterpret_cast<uint4*>(pages + at.row * a.p.head_dim * size) + chunk;
        if (WRITE) *p = *s;
        else *s = *p;
    }
    if (bad) raise_flag(a.p.flags, SSD_FLAG_BAD_PAGE);
}

dim3 grid_of(const MoveArgs& a, int units) {
    const int64_t need = ((int64_t)a.max_rows * a.p.n_kv_heads + units - 1) / units, share = 16384 / ((int64_t)a.p.B * 2 * a.n_layers);
    const int64_t parts = std::max<int64_t>(1, std::min(need, share));
    return dim3((unsigned)(parts * 2 * a.n_layers), (unsigned)a.p.B);
}

template <int DT, int PT>
void launch_codes(const MoveArgs& a, bool write, hipStream_t st) {
    if (a.p.head_dim == 128) {
        if (write) write_pages_kernel<DT, PT, 128><<<grid_of(a, 16), 256, 0, st>>>(a);
        else read_pages_kernel<DT, PT, 128><<<grid_of(a, 16), 256, 0, st>>>(a);
    } else {
        if (write) write_pages_kernel<DT, PT, 64><<<grid_of(a, 32), 256, 0, st>>>(a);
        else read_pages_kernel<DT, PT, 64><<<grid_of(a, 32), 256, 0, st>>>(a);
    }
}
template <int PT>
void launch_type(const MoveArgs& a, int dtype, bool write, hipStream_t st) {
    if (dtype == SSD_F32) launch_codes<SSD_F32, PT>(a, write, st);
    else if (dtype == SSD_BF16) launch_codes<SSD_BF16, PT>(a, write, st);
    else launch_codes<SSD_F16, PT>(a, write, st);
}
void launch_move(const MoveArgs& a, int dtype, int pages_dtype, bool write, hipStream_t st) {
    if (pages_dtype == SSD_E4M3) return launch_type<SSD_E4M3>(a, dtype, write, st);
    if (pages_dtype == SSD_I8) return launch_type<SSD_I8>(a, dtype, write, st);
    const int size = dtype == SSD_F32 ? 4 : 2, chunks = a.p.head_dim * size / 16;
    const dim3 grid = grid_of(a, 256 / chunks > 0 ? 256 / chunks : 1);
    if (write) copy_pages_kernel<true><<<grid, 256, 0, st>>>(a, chunks, size);
    else copy_pages_kernel<false><<<grid, 256, 0, st>>>(a, chunks, size);
}

}  // namespace

void launch_write_pages(const MoveArgs& a, int dtype, int pages_dtype, hipStream_t st) { launch_move(a, dtype, pages_dtype, true, st); }
void launch_read_pages(const MoveArgs& a, int dtype, int pages_dtype, hipStream_t st) { launch_move(a, dtype, pages_dtype, false, st); }

}  // namespace ssd
