// K/V rows in pages: what the host layer hands to the kernels of kv_pages.hip and paged_attn.hip.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/ssd.h"

namespace ssd {

struct PagesArgs {
    void* k; void* v; float* k_scale; float* v_scale;
    int64_t layer_rows;                      // rows (of all heads) of a layer: pages * n_kv_heads * page_rows
    int32_t n_pages, row_bits, n_kv_heads, head_dim;      // page_rows = 1 << row_bits
    const int32_t* entries; int64_t stride; const int32_t* ctx_len;
    int32_t B, max_ctx;
    int32_t* flags;                          // NULL: none
};

// Page of row j of utterance b, or -1.  Only for 0 <= j < max_ctx.
__device__ __forceinline__ int page_of(const PagesArgs& p, int b, int j) {
    const int page = p.entries[b * p.stride + (j >> p.row_bits)];
    return page >= 0 && page < p.n_pages ? page : -1;
}
// Number of a row of a head among those of its layer.
__device__ __forceinline__ int64_t row_in_pages(const PagesArgs& p, int page, int head, int j) {
    return (((int64_t)page * p.n_kv_heads + head) << p.row_bits) + (j & ((1 << p.row_bits) - 1));
}

struct MoveArgs {
    PagesArgs p;
    void* k; void* v; int64_t slots, slot_stride, head_stride, layer_stride;      // strides in elements
    const int32_t* start; const int32_t* n_rows;
    int32_t max_rows, n_layers;
};
// dtype: of the slots; pages_dtype: the same, SSD_E4M3 or SSD_I8
void launch_write_pages(const MoveArgs& a, int dtype, int pages_dtype, hipStream_t st);
void launch_read_pages(const MoveArgs& a, int dtype, int pages_dtype, hipStream_t st);

struct PagedAttnArgs {
    PagesArgs p;
    const void* q; int64_t q_stride;
    void* out; float* lse;
    int32_t n_q_heads, group, n_new;         // group: query heads of a K/V head
    float scale;
    int32_t tiles;                           // of 16 query rows, tokens times group
    int32_t piece, n_pieces;                 // rows of a piece of a context, pieces of max_ctx rows
    float* part_o; float2* part_ml;          // [token][query head][piece] mean of values (64 or 128 dims), (maximum to base 2, sum); not used by contexts of one piece
};
constexpr int PAGED_LEAST_PIECE = 256, PAGED_MOST_PIECE = 4096;      // (a wavefront has the pages of at most 4096 rows of its workgroup)
inline int paged_dims(int head_dim) { return head_dim > 64 ? 128 : 64; }
// Rows of a piece.
inline int paged_piece(int64_t pairs, int64_t max_ctx) {
    const int64_t share = pairs * max_ctx / 1024;
    const int64_t rows = (share + 255) / 256 * 256;
    return (int)(rows < PAGED_LEAST_PIECE ? PAGED_LEAST_PIECE : rows > 1024 ? 1024 : rows);
}
void launch_paged_attention(const PagedAttnArgs& a, int q_dtype, int pages_dtype, hipStream_t st);

}  // namespace ssd
