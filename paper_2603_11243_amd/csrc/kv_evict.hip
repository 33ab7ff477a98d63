// Eviction of cached rows by the attention weight they have collected: per layer, utterance and K/V head the first n_first rows, the last
// n_recent and, of those between, the ones of the largest weight are copied to another cache in their order.  Rotated keys carry their
// position, and attention does not ask for the order of its rows, so each head may keep rows of its own.
#include <string.h>

#include "device_utils.h"
#include "tree.h"

namespace ssd {

// Whole numbers in the order of the weights: 0 for NaN, which goes first; both zeros alike.
__device__ __forceinline__ uint32_t ordered(float v) {
    if (v != v) return 0;
    const uint32_t u = __float_as_uint(v + 0.f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

template <class M>
__device__ __forceinline__ EvictUtt utt_of(const M& w, int b) {
    return EvictUtt{(int)w(5 * b), (int)w(5 * b + 1), (int)w(5 * b + 2), (int)w(5 * b + 3), (int)w(5 * b + 4)};
}

// Selection: the need-th largest weight is found digit by digit, 11, 11 and 10 bits from the top: a histogram of the rows that agree with the digits found,
// and of its bins the one in which the count from above reaches `need`; there is nothing left to find once it reaches it exactly.  COPIES
// counters a bin, by lane: attention weights share few exponents, and lanes on one counter take turns.  Then the kept rows in order: a ballot gives the
// marks of 64 consecutive rows, one scan over these words their places.
// Up to EVICT_PIECE rows one workgroup has a (layer, head, utterance), V weights a thread in registers (row e THREADS + t is thread t's weight e).
// Longer ones are cut into pieces of a workgroup each, which a launch a digit ties together.
constexpr int BINS = EVICT_BINS;

// Sums of v over the threads before this one (x), and over all (y).
template <int THREADS>
__device__ __forceinline__ int2 scan(int v, int* waves) {
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    int s = v;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int o = __shfl_up(s, d);
        if (lane >= d) s += o;
    }
    __syncthreads();
    if (lane == 63) waves[wave] = s;
    __syncthreads();
    int before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) {
        if (w < wave) before += waves[w];
        all += waves[w];
    }
    return make_int2(before + s - v, all);
}

// A digit: its bits are digit << shift.
struct Digit { int shift; uint32_t digit; };
__device__ __forceinline__ Digit digit_of(int round) { return round == 0 ? Digit{21, 2047u} : round == 1 ? Digit{10, 2047u} : Digit{0, 1023u}; }

// What is known of the need-th largest: its digits t in the bits of mask, and how many of the rows that agree with them stay.
struct Known { uint32_t t, mask; int need, done; };
static_assert(sizeof(Known) == EVICT_KNOWN_BYTES, "what the workspace holds");

// The digit whose bin (counts count(bin), the same for all threads that ask) reaches `need` from above: found = {bin, rows above it, rows of it}.
template <int THREADS, class F>
__device__ __forceinline__ void find_bin(const F& count, int need, int* waves, int* found) {
    constexpr int PER = BINS / THREADS;
    int mine[PER], sum = 0;                                  // from the top: thread t has bins BINS - 1 - t PER - e
#pragma unroll
    for (int e = 0; e < PER; ++e) sum += mine[e] = count(BINS - 1 - (int)threadIdx.x * PER - e);
    int above = scan<THREADS>(sum, waves).x;
#pragma unroll
    for (int e = 0; e < PER; ++e) {
        if (above < need && above + mine[e] >= need) {
            found[0] = BINS - 1 - threadIdx.x * PER - e;
            found[1] = above;
            found[2] = mine[e];
        }
        above += mine[e];
    }
    __syncthreads();
}

// Weights of rows c0 .. of an utterance, in order; behind the end copies of the last.
template <int THREADS, int V>
__device__ __forceinline__ void load_weights(uint32_t (&x)[V], const float* w, int c0, int n) {
#pragma unroll
    for (int e = 0; e < V; ++e) x[e] = __float_as_uint(w[min(c0 + e * THREADS + (int)threadIdx.x, n - 1)]);
#pragma unroll
    for (int e = 0; e < V; ++e) x[e] = ordered(__uint_as_float(x[e]));
}

template <int THREADS, int V, int COPIES>
__device__ __forceinline__ void count_rows(const uint32_t (&x)[V], int c0, int lo, int hi, const Known& k, Digit d, int* hist) {
#pragma unroll
    for (int e = 0; e < V; ++e) {
        const int i = c0 + e * THREADS + threadIdx.x;
        if (i >= lo && i < hi && ((x[e] ^ k.t) & k.mask) == 0) atomicAdd(&hist[(x[e] >> d.shift & d.digit) * COPIES + threadIdx.x % COPIES], 1);
    }
}

// The kept ones of rows c0 .. c0 + THREADS V - 1 (below `end`), behind `out` kept ones and `ties` rows that agree with k; both follow.
template <int THREADS, int V>
__device__ __forceinline__ void list_rows(const uint32_t (&x)[V], int c0, int end, int lo, int hi, const Known& k, int2* marks, int* waves, int32_t* rows, int& out, int& ties) {
    constexpr int WAVES = THREADS / 64, WORDS = WAVES * V;
    static_assert(WORDS <= THREADS, "a thread a word of marks");
    const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64;
    uint32_t sure_bits = 0, tie_bits = 0;
    static_assert(V <= 32, "marks of a thread");
#pragma unroll
    for (int e = 0; e < V; ++e) {
        const int i = c0 + e * THREADS + tid;
        const bool between = i >= lo && i < hi, in = i < end;
        const bool sure = in && (!between || (x[e] & k.mask) > k.t), tie = in && between && (x[e] & k.mask) == k.t;
        sure_bits |= (uint32_t)sure << e;
        tie_bits |= (uint32_t)tie << e;
        const int2 n = make_int2(__popcll(__ballot(sure)), __popcll(__ballot(tie)));
        if (lane == 0) marks[e * WAVES + wave] = n;
    }
    __syncthreads();
    const int2 n = tid < WORDS ? marks[tid] : make_int2(0, 0);
    const int2 s = scan<THREADS>(n.x, waves), r = scan<THREADS>(n.y, waves);
    if (tid < WORDS) marks[tid] = make_int2(s.x, r.x);
    __syncthreads();
    const uint64_t below = ((uint64_t)1 << lane) - 1;
    const int kept_ties = min(ties, k.need);
#pragma unroll
    for (int e = 0; e < V; ++e) {
        const bool sure = sure_bits >> e & 1, tie = tie_bits >> e & 1;
        const int2 before = marks[e * WAVES + wave];
        const int sures = before.x + __popcll(__ballot(sure) & below), tied = ties + before.y + __popcll(__ballot(tie) & below);
        if (sure || (tie && tied < k.need)) rows[out + sures + min(tied, k.need) - kept_ties] = c0 + e * THREADS + tid;
    }
    ties += r.y;
    out += s.y + min(ties, k.need) - kept_ties;
}

// Nothing between stays, or rows between are to be found: what is known at the beginning.
__device__ __forceinline__ Known known_at_first(const EvictArgs& a, const EvictUtt& u) {
    const int need = u.keep - a.n_first - a.n_recent;
    return need > 0 ? Known{0u, 0u, need, 0} : Known{~0u, ~0u, 0, 1};      // (all bits: no weight is above, and of those that agree none stays)
}

template <int THREADS, int V, int COPIES, class M>
__global__ void __launch_bounds__(THREADS) evict_select_kernel(EvictArgs a, M meta) {
    __shared__ int hist[BINS * COPIES];
    __shared__ int waves[THREADS / 64];
    __shared__ int found[3];
    __shared__ int2 marks[THREADS / 64 * V];
    const EvictUtt u = utt_of(meta, blockIdx.x);
    const int64_t lh = blockIdx.y;                           // layer * heads + head
    int32_t* rows = a.rows + lh * a.n_kept + u.kept0;
    if (u.keep >= u.n_ctx) {
        for (int i = threadIdx.x; i < u.n_ctx; i += THREADS) rows[i] = i;
        return;
    }
    const int lo = a.n_first, hi = u.n_ctx - a.n_recent;
    uint32_t x[V];
    load_weights<THREADS, V>(x, a.mass + lh * a.mass_slots + u.slot0, 0, u.n_ctx);
    Known k = known_at_first(a, u);
    for (int round = 0; round < 3 && !k.done; ++round) {
        const Digit d = digit_of(round);
        for (int i = threadIdx.x; i < BINS * COPIES; i += THREADS) hist[i] = 0;
        __syncthreads();
        count_rows<THREADS, V, COPIES>(x, 0, lo, hi, k, d, hist);
        __syncthreads();
        find_bin<THREADS>([&](int bin) {
            int n = 0;
#pragma unroll
            for (int c = 0; c < COPIES; ++c) n += hist[bin * COPIES + c];
            return n;
        }, k.need, waves, found);
        k.t |= (uint32_t)found[0] << d.shift;
        k.mask |= d.digit << d.shift;
        k.need -= found[1];
        k.done = found[2] == k.need;
        __syncthreads();
    }
    int out = 0, ties = 0;
    list_rows<THREADS, V>(x, 0, u.n_ctx, lo, hi, k, marks, waves, rows, out, ties);
}

// Round 0, 1, 2: a histogram of a piece's rows by the round's digit, after the digit of the round before has been found in the pieces' histograms; round
// 3: the last digit, and the piece's kept rows.  Every piece finds the same; what it needs of the pieces before it, it counts itself.
template <int ROUND, class M>
__global__ void __launch_bounds__(1024) evict_piece_kernel(EvictArgs a, M meta) {
    constexpr int THREADS = 1024, V = EVICT_PIECE / THREADS, COPIES = 4;
    __shared__ int hist[ROUND < 3 ? BINS * COPIES : 1];
    __shared__ int waves[THREADS / 64];
    __shared__ int found[3], tied;
    __shared__ int2 marks[ROUND == 3 ? THREADS / 64 * V : 1];
    const int piece = blockIdx.x, tid = threadIdx.x, b = (int)meta(a.pieces + piece), first = (int)meta(a.firsts + b);
    const EvictUtt u = utt_of(meta, b);
    const int64_t lh = blockIdx.y;
    const int64_t r0 = (int64_t)(piece - first) * a.piece_rows;
    const int end = (int)min((int64_t)u.n_ctx, r0 + a.piece_rows), lo = a.n_first, hi = u.n_ctx - a.n_recent;
    const int n_pieces = (int)(((int64_t)u.n_ctx + a.piece_rows - 1) / a.piece_rows);
    int32_t* rows = a.rows + lh * a.n_kept + u.kept0;
    if (u.keep >= u.n_ctx) {
        if (ROUND == 3)
            for (int i = (int)r0 + tid; i < end; i += THREADS) rows[i] = i;
        return;
    }
    uint16_t* counts = a.counts + (lh * a.n_pieces + first) * 2 * BINS;          // of the utterance's pieces, two buffers each
    Known* known = a.known + (lh * a.B + b) * 2;
    int2* before = a.before + lh * a.n_pieces + piece;       // rows above the digits, rows that agree with them, in the pieces before
    Known k = ROUND <= 1 ? known_at_first(a, u) : known[ROUND - 2];
    int2 prior = make_int2(0, 0);
    if (ROUND >= 2) prior = *before;
    if (ROUND && !k.done) {
        const Digit d = digit_of(ROUND - 1);
        // thread t: bins BINS - 1 - 2 t and the one below, of all pieces and of those before this one, eight pieces requested at once
        const uint32_t* c = reinterpret_cast<const uint32_t*>(counts + (ROUND - 1) % 2 * BINS) + BINS / 2 - 1 - tid;
        int all[2] = {0, 0}, earlier[2] = {0, 0};
        for (int p0 = 0; p0 < n_pieces; p0 += 8) {
            uint32_t n[8];
#pragma unroll
            for (int p = 0; p < 8; ++p) n[p] = c[(int64_t)min(p0 + p, n_pieces - 1) * BINS];
#pragma unroll
            for (int p = 0; p < 8; ++p)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int v = p0 + p < n_pieces ? (int)(e ? n[p] & 0xffffu : n[p] >> 16) : 0;
                    all[e] += v;
                    earlier[e] += p0 + p < piece - first ? v : 0;
                }
        }
        find_bin<THREADS>([&](int x) { return x & 1 ? all[0] : all[1]; }, k.need, waves, found);
        const int bin = found[0], top = BINS - 1 - 2 * tid;
        if (top == bin) tied = earlier[0];
        if (top - 1 == bin) tied = earlier[1];
        prior.x += scan<THREADS>((top > bin ? earlier[0] : 0) + (top - 1 > bin ? earlier[1] : 0), waves).y;      // (and its barriers: tied is written)
        prior.y = tied;
        k.t |= (uint32_t)bin << d.shift;
        k.mask |= d.digit << d.shift;
        k.need -= found[1];
        k.done = found[2] == k.need;
    }
    if (ROUND && ROUND < 3 && tid == 0) {
        *before = prior;
        if (piece == first) known[ROUND - 1] = k;
    }
    const float* w = a.mass + lh * a.mass_slots + u.slot0;
    uint32_t x[V];
    if constexpr (ROUND < 3) {
        if (k.done) return;
        for (int i = tid; i < BINS * COPIES; i += THREADS) hist[i] = 0;
        __syncthreads();
        for (int64_t c0 = r0; c0 < end; c0 += EVICT_PIECE) {
            load_weights<THREADS, V>(x, w, (int)c0, u.n_ctx);
            count_rows<THREADS, V, COPIES>(x, (int)c0, lo, min(hi, end), k, digit_of(ROUND), hist);
        }
        __syncthreads();
        uint16_t* mine = counts + ((int64_t)(piece - first) * 2 + ROUND % 2) * BINS;
        for (int i = tid; i < BINS; i += THREADS) mine[i] = (uint16_t)(hist[i * COPIES] + hist[i * COPIES + 1] + hist[i * COPIES + 2] + hist[i * COPIES + 3]);
    } else {
        int out = (int)(min(r0, (int64_t)lo) + max(r0 - hi, (int64_t)0)) + prior.x + min(prior.y, k.need), ties = prior.y;
        for (int64_t c0 = r0; c0 < end; c0 += EVICT_PIECE) {
            if (c0 > r0) __syncthreads();
            load_weights<THREADS, V>(x, w, (int)c0, u.n_ctx);
            list_rows<THREADS, V>(x, (int)c0, end, lo, hi, k, marks, waves, rows, out, ties);
        }
    }
}

// Row `blockIdx.x` of the kept ones in a layer, all heads.
template <class M>
__global__ void __launch_bounds__(256) evict_copy_kernel(EvictArgs a, M meta) {
    const int r = blockIdx.x;
    int b = 0, end = a.B;                                    // the utterance it belongs to: the last one that begins at or before it
    while (end - b > 1) {
        const int mid = (b + end) / 2;
        if ((int)meta(5 * mid + 4) <= r) b = mid;
        else end = mid;
    }
    const EvictUtt u = utt_of(meta, b);
    const int64_t dst = u.out0 + (r - u.kept0);
    const int per = a.row_chunks, n = a.n_kv_heads * per;
    const int layer = blockIdx.y;
    for (int i = threadIdx.x; i < n; i += 256) {
        const int h = i / per, c = i % per;
        const int64_t lh = (int64_t)layer * a.n_kv_heads + h;
        const int64_t src = u.slot0 + a.rows[lh * a.n_kept + r];
        const int64_t s = layer * a.layer_stride + h * a.head_stride + src * a.slot_stride + c;
        const int64_t d = layer * a.out_layer_stride + h * a.out_head_stride + dst * a.out_slot_stride + c;
        const uint4 k = ((const uint4*)a.k)[s], v = ((const uint4*)a.v)[s];
        ((uint4*)a.k_out)[d] = k;
        ((uint4*)a.v_out)[d] = v;
        if (a.mass_out && c == 0) a.mass_out[lh * a.mass_out_slots + dst] = a.mass[lh * a.mass_slots + src];
    }
}

// By the longest context.  Selection of 8 heads in one workgroup each: 1000 rows 7.7 us, 8192 rows 11.4 and, with the weights read again for every digit, 32768 rows
// 27, 65536 rows 77; in pieces 22 and 25 us for 32768 and 131072 rows: four launches of 4 to 11 us, the chain histogram, count, scan.  The copy
// of 768 kept rows in 24 layers of 8 heads of 128 (151 MB read and written) takes 32 us, of 8191 in 2 layers (134 MB) 30: 4.7 and 4.5 TB/s of a plain copy's 5.1.
template <class M>
static void launch(const EvictArgs& a, const M& w, hipStream_t st) {
    const int lh = a.n_layers * a.n_kv_heads;
    if (a.most_ctx <= 256 * 4) hipLaunchKernelGGL((evict_select_kernel<256, 4, 1, M>), dim3(a.B, lh), dim3(256), 0, st, a, w);
    else if (a.most_ctx <= EVICT_PIECE) hipLaunchKernelGGL((evict_select_kernel<1024, EVICT_PIECE / 1024, 2, M>), dim3(a.B, lh), dim3(1024), 0, st, a, w);
    else {
        const dim3 grid(a.n_pieces, lh);
        hipLaunchKernelGGL((evict_piece_kernel<0, M>), grid, dim3(1024), 0, st, a, w);
        hipLaunchKernelGGL((evict_piece_kernel<1, M>), grid, dim3(1024), 0, st, a, w);
        hipLaunchKernelGGL((evict_piece_kernel<2, M>), grid, dim3(1024), 0, st, a, w);
        hipLaunchKernelGGL((evict_piece_kernel<3, M>), grid, dim3(1024), 0, st, a, w);
    }
    hipLaunchKernelGGL((evict_copy_kernel<M>), dim3(a.n_kept, a.n_layers), dim3(256), 0, st, a, w);
}

void launch_kv_evict(const EvictArgs& a, const uint32_t* words, int n, const uint32_t* dev_words, hipStream_t st) {
    static_assert(sizeof(EvictArgs) + sizeof(MetaWords) + 16 <= 4096, "arguments of a launch");
    if (!words) { launch(a, MetaArray{dev_words}, st); return; }
    MetaWords w;
    w.n = n;
    memcpy(w.word, words, (size_t)n * 4);
    launch(a, w, st);
}

}  // namespace ssd
