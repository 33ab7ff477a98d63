// Trees of drafted tokens over cached rows: what the host layer hands to the kernels of tree_attn.hip, tree_path.hip and kv_evict.hip.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/ssd.h"

namespace ssd {

constexpr int MAX_TREE_NODES = SSD_MAX_TREE_NODES;

// Host metadata of a call as 32-bit words: arguments of the launch where they are few (4 KB with the rest), else in the workspace.
struct MetaWords {
    static constexpr int WORDS = 940;
    int n;
    uint32_t word[WORDS];
    __device__ __forceinline__ uint32_t operator()(int i) const { return word[i]; }
};
struct MetaArray {
    const uint32_t* word;
    __device__ __forceinline__ uint32_t operator()(int i) const { return word[i]; }
};
void launch_write_words(const MetaWords& w, uint32_t* dst, hipStream_t st);
// n words of pinned host memory to dst (16-byte aligned both)
void launch_copy_words(const uint32_t* host, size_t n, uint32_t* dst, hipStream_t st);

// Attention of nodes.  Query rows of one K/V head are numbered node * G + head of the group; keys are the rows of the utterance, n_ctx cached ones, then
// the nodes.  The words: per item of work six, at a place known without another: first slot, n_ctx, first node, nodes | tile of tile_rows query rows << 11,
// first key and the one behind the last (the first n_parts items, pieces of cut contexts, leave partial results); from `utts` on per utterance first slot and n_ctx, from `cu` on the
// B + 1 prefix sums of the nodes; from `joins` on per tile of a cut utterance three: utterance | tile << 16, item of its first piece,
// pieces; from `mass_items` on per item of the weights one: utterance | piece of mass_step keys << 16; from `spans` on per node its place in
// depth-first order | end of its subtree << 16.
struct TreeAttnArgs {
    const void* q; int64_t q_stride;
    const void* k; const void* v; int64_t slot_stride, head_stride;
    void* out;
    float* lse;                              // [nodes, n_q_heads]; NULL: not wanted
    float* mass; int64_t mass_stride;        // [n_kv_heads, mass_stride]; NULL: not wanted
    float* part_o; float2* part_ml;          // [item][K/V head][tile_rows] outputs and (maximum, sum) of pieces
    int n_q_heads, n_kv_heads, head_dim, dtype;
    int group; uint32_t group_magic;         // n_q_heads / n_kv_heads; 2^32 / group rounded up, 0 for 1
    float scale;
    int tile_rows, mass_step, n_items, n_parts, n_joins, n_mass;
    int utts, cu, joins, mass_items, spans;
};
// words: host memory, n of them, to travel as arguments; or NULL, then they are in dev_words
void launch_tree_attention(const TreeAttnArgs& a, const uint32_t* words, int n, const uint32_t* dev_words, hipStream_t st);
constexpr int TREE_ITEMS = 65535;            // of a call: rows of a grid
constexpr int TREE_WORKGROUPS = 512;         // long contexts are cut into about as many pieces in all, times K/V heads
constexpr int TREE_SPLIT_KEYS = 512;         // a share has at least as many keys, a piece of a cut context from three quarters of that on (its last one fewer)
constexpr int TREE_MASS_KEYS = 128;          // and one of the weights a multiple of these

// Words: the B + 1 prefix sums of the nodes (at most MAX_TREE_NODES an utterance); from `parents` on the nodes' parents inside their utterance or -1, 16
// bits each.  words: host memory, n of them, to travel as arguments; or NULL, then they are in dev_words.
struct TreePathArgs {
    const float* logp;
    int B, most_nodes, parents;
    float ln_tau;
    bool roots_given;                        // nodes without a parent pass
    int32_t* accept_len; int32_t* accept_node; int32_t* path;
};
void launch_tree_path(const TreePathArgs& a, const uint32_t* words, int n, const uint32_t* dev_words, hipStream_t st);

// node_logp[i] = logp[i], 0 where parent[i] < 0; greedy_tok[i] = greedy[row_of[i]]
void launch_tree_scatter(const float* logp, const int32_t* greedy, const int32_t* row_of, const int16_t* parent, int n, float* node_logp,
                         int32_t* greedy_tok, hipStream_t st);
// K/V rows of the accepted path (and their entries of mass [n_layers, n_kv_heads, slots], unless NULL) to the slots behind the context; strides in
// 16-byte units, a slot's heads one behind the other, row_chunks units each
void launch_tree_commit(void* k, void* v, int64_t slot_stride, int64_t layer_stride, int n_layers, int n_kv_heads, int row_chunks, float* mass, int64_t slots,
                        const int32_t* kv_start, const int32_t* ctx_len, const int32_t* cu, const int32_t* accept_len, const int32_t* path, int B,
                        hipStream_t st);

struct Known;
struct EvictUtt { int32_t slot0, n_ctx, keep, out0, kept0; };     // kept0: kept rows of the utterances before
struct EvictArgs {
    const void* k; const void* v; int64_t slot_stride, head_stride, layer_stride;         // in 16-byte units
    void* k_out; void* v_out; int64_t out_slot_stride, out_head_stride, out_layer_stride;
    int n_layers, n_kv_heads, row_chunks;    // 16-byte units of a row
    const float* mass; int64_t mass_slots;
    float* mass_out; int64_t mass_out_slots; // mass_out NULL: not wanted
    int B, most_ctx;                         // most_ctx: rows of the longest context
    int n_first, n_recent, n_kept;           // n_kept: rows that all utterances keep
    int32_t* rows;                           // [n_layers, n_kv_heads, n_kept]
    // contexts of more than EVICT_PIECE rows: pieces of piece_rows; from word `pieces` on the utterance of each, from `firsts` on each utterance's first
    int n_pieces, piece_rows, pieces, firsts;
    uint16_t* counts; Known* known; int2* before;      // [layers * heads][pieces][2][bins], [layers * heads][B][2], [layers * heads][pieces]
};
constexpr int EVICT_PIECE = 8192;            // rows of a workgroup (counts are 16 bits wide: at most 65535 rows a piece)
constexpr int EVICT_PIECES = 64;             // longer contexts are cut into at most so many pieces, and one an utterance
constexpr int EVICT_BINS = 2048;
constexpr size_t EVICT_KNOWN_BYTES = 16;
// words: the B EvictUtt, then those of the pieces, n in all, in host memory, to travel as arguments; or NULL, then they are in dev_words
void launch_kv_evict(const EvictArgs& a, const uint32_t* words, int n, const uint32_t* dev_words, hipStream_t st);

}  // namespace ssd
