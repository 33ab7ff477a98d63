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
    bool codes;                              // pages of an 8-bit type
    int32_t tile_rows, tiles;                // query rows of a K/V head, tokens times group, in tiles of 16 or 32
    // Contexts are cut into pieces of whole PAGED_UNITs of rows: shared 0, each by itself every PAGED_MOST units, n_pieces of max_ctx rows; else all of a K/V head
    // and tile into about `shared` equal ones, at most n_pieces.
    int32_t shared, n_pieces;
    float* part_o; float2* part_ml;          // [piece (of an utterance with shared 0: utterance, piece)][query row of tile and K/V head]: mean of 64 or 128 values; (maximum to base 2, sum)
    int2* first;                             // [utterance] first piece, pieces
};
constexpr int PAGED_UNIT = 128, PAGED_MOST = 32;             // a round of four wavefronts of 32 rows; units of an unshared piece: a wavefront has the page numbers of so many in a register
constexpr int64_t PAGED_QUERIES = 1 << 21;                   // of a call: workgroups of up to 1024 threads that join their pieces
constexpr int PAGED_UTTS = 1024;                             // utterances of a batch that shares
inline int paged_dims(int head_dim) { return head_dim > 64 ? 128 : 64; }
// Query rows of a workgroup.  32 read keys and values half as often as 16, which halves what long contexts cost, but are longer on their way through a block and fewer workgroups: by the
// units of rows that workgroups of 16 would take.  Half, 12 tokens of 16 heads on 8 of 128, 16 and 32: 4 contexts of 150 to 300 rows 7.8 and 9.8 us, 1250 to 2500 (1280 units) 17.3 and
// 17.9, 10000 to 20000 72 and 61; 40 of 30 to 60 (640) 10.3 and 9.6, 300 to 600 25 and 22, 2000 to 4000 195 and 115.  Codes of 64 dims, 7 tokens of 16 heads on 4: 40 contexts of 750
// to 1500 (3840) 16.0 and 17.8, 2000 to 4000 (10240) 25.9 and 23.7.  Of 128 dims, 12 tokens of 16 heads on 8, int8 and e4m3: 4 of 1250 to 2500 (1216) 14.5 and 16.1, 13.9 and 16.2; 8 of 500 to
// 1000 (1024) 14.0 and 15.6, 12.5 and 15.2; 10 of 1000 to 2000 (2400) 20.7 and 19.1, 19.2 and 18.4; 40 of 2000 to 4000 (19840) 103 and 74, 99 and 71.  The units are those that the launch
// is made for: one made for long contexts takes 32 over short ones too (40 of 30 to 60 rows 8.2 and 9.4, 9.4 and 9.2).  fp32 pages of 64 dims 20.5 and 22.5 (1600), 43 and 36 (3840), of 128 120 and 148 (7680), 375 and 281 (20480);
// fp32 queries over codes have no registers for 32 (101 and 140).
inline int paged_tile_rows(int64_t rows, int64_t B, int64_t n_kv_heads, int64_t max_ctx, int head_dim, int q_dtype, int pages_dtype) {
    const bool codes = pages_dtype == SSD_E4M3 || pages_dtype == SSD_I8, wide = paged_dims(head_dim) == 128;
    if (rows <= 16 || (codes && q_dtype == SSD_F32)) return 16;
    const int64_t from = q_dtype == SSD_F32 ? (wide ? 15000 : 3000) : codes && !wide ? 8000 : 2000;
    return B * n_kv_heads * ((rows + 15) / 16) * ((max_ctx + PAGED_UNIT - 1) / PAGED_UNIT) >= from ? 32 : 16;
}
// Workgroups of a CU whose registers fit; shared pieces are as many as run at once, and are held to so many a CU by the LDS they ask for.
inline int paged_per_cu(int head_dim, int tile_rows) { return paged_dims(head_dim) == 128 ? 2 : tile_rows == 16 ? 4 : 3; }
constexpr int PAGED_CUS = 256, PAGED_CU_LDS = 160 * 1024;
// Pieces of a batch are at least so many times its utterances: their last pieces are shorter ones, which counts where there are few (40 utterances of 2000 to 4000 rows, half,
// 8 heads: 108 us with 1, 97 with 2, 3 or 6; 90 of 1500 to 3000, e4m3: 98, 98, 101, 117).
constexpr int PAGED_EACH = 2;
// Units of the longest contexts that are not cut, by the workgroups there are without: the second launch and finding the piece cost 3 us.  In a graph, 8 heads, 64-row pages,
// half, cut and not: 1 utterance of 600 rows 8.7 and 9.4 us, 1000 8.8 and 13.0; 16 of 300 to 600 13.9 and 10.9, 500 to 1000 15.8 and 14.9, 750 to 1500 18.9 and 19.0;
// 40 of 1300 47.9 and 48.2 (e4m3 32.0 and 26.9), 2000 67.6 and 70.3 (43.2 and 38.7); 90 of 2000 136 and 125 (82 and 73); 200 of 375 to 1500 147 and 145 (106 and 82).
inline int paged_whole(int64_t workgroups) { return workgroups >= 1024 ? PAGED_MOST : workgroups >= 256 ? 16 : workgroups >= 128 ? 8 : 5; }
void launch_paged_attention(const PagedAttnArgs& a, int q_dtype, int pages_dtype, hipStream_t st);

}  // namespace ssd
