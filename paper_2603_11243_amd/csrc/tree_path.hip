// Accepted path of a tree of drafted tokens (Eq. 5 and the definition of j, Sec. 2.3, for more than one continuation): a node stands if
// its own likelihood and those of all its ancestors pass; the deepest node that stands wins, the lowest index among equally deep ones.
#include <string.h>

#include "device_utils.h"
#include "tree.h"

namespace ssd {

// One workgroup a tree, one thread a node (NT of them).  Pointer jumping: after round r a node knows whether the 2^r nodes on the way up
// from it pass, how many there are, and who comes next: ten rounds of LDS for 1024 nodes.  The accepted path is then written by one thread that walks it up, a read of
// LDS and a store a node (some ten of them in the cases timed; a chain of 1024 that passes is 1024).  24 nodes 2.9 us, 256
// trees of 64 to 1000 nodes 6.9: a launch; the calls take 9 and 37 us, of which the host checks, packs and hands over the parents.
template <int NT, class M>
__global__ void __launch_bounds__(NT) tree_path_kernel(const float* __restrict__ logp, M w, int parents, float ln_tau, bool roots_given, int32_t* __restrict__ accept_len,
                                                       int32_t* __restrict__ accept_node, int32_t* __restrict__ path) {
    __shared__ int up_s[NT], way_s[NT], best_s;              // way: nodes on the way, negative if one of them fails
    const int i = threadIdx.x, node0 = (int)w(blockIdx.x), n = (int)w(blockIdx.x + 1) - node0;
    int up = -1, way = -1;
    if (i < n) {
        up = (int16_t)(w(parents + (node0 + i) / 2) >> 16 * ((node0 + i) % 2));
        way = (up < 0 && roots_given) || logp[node0 + i] > ln_tau ? 1 : -0x10000;
        path[node0 + i] = -1;
    }
    const int first_up = up;
    if (i == 0) best_s = -1;
    for (int r = 1; r < NT; r *= 2) {
        up_s[i] = up;
        way_s[i] = way;
        __syncthreads();
        if (up >= 0) {
            way += way_s[up];
            if (way < 0) way = -0x10000;
            up = up_s[up];
        }
        __syncthreads();
    }
    if (i < n && way > 0) atomicMax(&best_s, way * NT + (NT - 1 - i));
    up_s[i] = first_up;
    __syncthreads();
    if (i == 0) {
        const int best = best_s < 0 ? -1 : NT - 1 - best_s % NT, len = best_s < 0 ? 0 : best_s / NT;
        accept_len[blockIdx.x] = len;
        accept_node[blockIdx.x] = best;
        int at = best;
        for (int d = len - 1; d >= 0; --d) {
            path[node0 + d] = at;
            at = up_s[at];
        }
    }
}

__global__ void __launch_bounds__(256) write_words_kernel(MetaWords w, uint32_t* __restrict__ dst) {
    for (int i = threadIdx.x; i < w.n; i += 256) dst[i] = w.word[i];
}
void launch_write_words(const MetaWords& w, uint32_t* dst, hipStream_t st) {
    hipLaunchKernelGGL(write_words_kernel, dim3(1), dim3(256), 0, st, w, dst);
}

// Metadata from pinned host memory.  All loads of a thread are requested before the first is used, one way over the bus: 26 KB 5.7 us, 275 KB 9.0; the copy
// engine takes 17 us between two kernels for 24 KB.
constexpr int COPY_UNITS = 4;                // of 16 bytes a thread
__global__ void __launch_bounds__(256) copy_words_kernel(const uint4* __restrict__ host, int units, uint4* __restrict__ dst) {
    const int at = (int)blockIdx.x * 256 * COPY_UNITS + threadIdx.x;
    uint4 x[COPY_UNITS];
#pragma unroll
    for (int u = 0; u < COPY_UNITS; ++u) x[u] = host[min(at + u * 256, units - 1)];
#pragma unroll
    for (int u = 0; u < COPY_UNITS; ++u)
        if (at + u * 256 < units) dst[at + u * 256] = x[u];
}
void launch_copy_words(const uint32_t* host, size_t n, uint32_t* dst, hipStream_t st) {
    const int units = (int)((n + 3) / 4);                    // (both ends are allocated in larger units)
    hipLaunchKernelGGL(copy_words_kernel, dim3((units + 256 * COPY_UNITS - 1) / (256 * COPY_UNITS)), dim3(256), 0, st, (const uint4*)host, units, (uint4*)dst);
}

__global__ void __launch_bounds__(256) tree_scatter_kernel(const float* __restrict__ logp, const int32_t* __restrict__ greedy, const int32_t* __restrict__ row_of,
                                                          const int16_t* __restrict__ parent, int n, float* __restrict__ node_logp,
                                                          int32_t* __restrict__ greedy_tok) {
    const int i = blockIdx.x * 256 + threadIdx.x;
    if (i >= n) return;
    node_logp[i] = parent[i] < 0 ? 0.f : logp[i];
    greedy_tok[i] = greedy[row_of[i]];
}
void launch_tree_scatter(const float* logp, const int32_t* greedy, const int32_t* row_of, const int16_t* parent, int n, float* node_logp,
                         int32_t* greedy_tok, hipStream_t st) {
    hipLaunchKernelGGL(tree_scatter_kernel, dim3((n + 255) / 256), dim3(256), 0, st, logp, greedy, row_of, parent, n, node_logp, greedy_tok);
}

// One thread a 16-byte column of an utterance's rows in a layer.  Step d moves row path[d] >= d to d, and path[d + 1] > path[d]: no row is written that a later step
// reads, whatever the order of loads and stores, and no other thread touches the column.  Rows go eight at a time through an array that the compiler keeps in private memory
// (144 bytes a lane).
template <typename T>
__device__ __forceinline__ void move_rows(T* col, int64_t stride, const int32_t* from, int n) {
    for (int d0 = 0; d0 < n; d0 += 8) {
        T x[8];
#pragma unroll
        for (int d = 0; d < 8; ++d) x[d] = col[from[min(d0 + d, n - 1)] * stride];
#pragma unroll
        for (int d = 0; d < 8; ++d)
            if (d0 + d < n) col[(d0 + d) * stride] = x[d];
    }
}

__global__ void __launch_bounds__(256) tree_commit_kernel(uint4* __restrict__ k, uint4* __restrict__ v, int64_t slot_stride, int64_t layer_stride, int n_kv_heads,
                                                         int cols, float* __restrict__ mass, int64_t slots, const int32_t* __restrict__ kv_start,
                                                         const int32_t* __restrict__ ctx_len, const int32_t* __restrict__ cu,
                                                         const int32_t* __restrict__ accept_len, const int32_t* __restrict__ path) {
    const int b = blockIdx.x, layer = blockIdx.y, n = accept_len[b];
    const int32_t* from = path + cu[b];
    if (n <= 0 || from[n - 1] == n - 1) return;              // (a path of the first nodes is in its place)
    const int64_t slot0 = (int64_t)kv_start[b] + ctx_len[b], base = layer * layer_stride + slot0 * slot_stride;
    for (int c = threadIdx.x; c < 2 * cols; c += 256) move_rows((c < cols ? k : v) + base + c % cols, slot_stride, from, n);
    if (mass)
        for (int h = threadIdx.x; h < n_kv_heads; h += 256) move_rows(mass + ((int64_t)layer * n_kv_heads + h) * slots + slot0, 1, from, n);
}
void launch_tree_commit(void* k, void* v, int64_t slot_stride, int64_t layer_stride, int n_layers, int n_kv_heads, int row_chunks, float* mass, int64_t slots,
                        const int32_t* kv_start, const int32_t* ctx_len, const int32_t* cu, const int32_t* accept_len, const int32_t* path, int B,
                        hipStream_t st) {
    hipLaunchKernelGGL(tree_commit_kernel, dim3(B, n_layers), dim3(256), 0, st, (uint4*)k, (uint4*)v, slot_stride, layer_stride, n_kv_heads, n_kv_heads * row_chunks,
                       mass, slots, kv_start, ctx_len, cu, accept_len, path);
}

template <class M>
static void launch(const TreePathArgs& a, const M& w, hipStream_t st) {
#define SSD_PATH(NT_) hipLaunchKernelGGL((tree_path_kernel<NT_, M>), dim3(a.B), dim3(NT_), 0, st, a.logp, w, a.parents, a.ln_tau, a.roots_given, a.accept_len, a.accept_node, a.path)
    if (a.most_nodes <= 64) SSD_PATH(64);
    else if (a.most_nodes <= 256) SSD_PATH(256);
    else SSD_PATH(MAX_TREE_NODES);
#undef SSD_PATH
}

void launch_tree_path(const TreePathArgs& a, const uint32_t* words, int n, const uint32_t* dev_words, hipStream_t st) {
    if (!words) { launch(a, MetaArray{dev_words}, st); return; }
    MetaWords w;
    w.n = n;
    memcpy(w.word, words, (size_t)n * 4);
    launch(a, w, st);
}

}  // namespace ssd
