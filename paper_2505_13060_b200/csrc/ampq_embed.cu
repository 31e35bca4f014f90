// Embedding lookup with scaling and its gradient (include/ampq.h:
// ampq_embed_forward, ampq_embed_backward).
//
// The gradient's rows are sums over the tokens that read them.  The tokens are
// sorted (by value, then by place), so that the rows of gy that belong together lie
// in one run of the order; runs are cut into pieces of a fixed number of tokens, and
// what a cut run leaves is joined in order by whoever comes last.  No atomics on
// values: the result depends on the inputs alone.
#include "ampq_decoder.h"

namespace ampq {
namespace {

constexpr int kThreads = 256;

// Threads that share a row: a chunk to each, whole warps, a CTA at most; wider rows
// are cut into slabs.
struct RowSplit {
    int threads;
    unsigned slabs;
    RowSplit(long long cols, int elems) {
        const long long chunks = (cols + elems - 1) / elems;
        threads = 32;
        while (threads < kThreads && threads < chunks) threads *= 2;
        slabs = (unsigned)((chunks + threads - 1) / threads);
    }
};

// A warp's block of a row: 32 chunks.  A lane has one of them where rows start on
// 16-byte boundaries.  Elsewhere (STRIDED) a chunk is not one access; there a lane has
// every 32nd element (fp32) or pair (bf16), so that a warp's accesses are neighbours.
template <typename T, bool STRIDED>
struct Block {
    static constexpr int E = Chunk<T>::kElems;
    static constexpr int kPer = 4 / (int)sizeof(T);  // elements of a word
    // Column of a lane's word i.
    __device__ static __forceinline__ int column(int c_block, int i) { return c_block + kPer * ((int)(threadIdx.x % 32) + 32 * i); }
    __device__ static __forceinline__ void load_words(const T* row, int c_block, int cols, unsigned (&w)[8]) {
        if constexpr (!STRIDED) {
            const int c0 = c_block + (int)(threadIdx.x % 32) * E;
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = 0;
            if (c0 < cols) Chunk<T>::load_words(row + c0, min(E, cols - c0), w);
        } else {
            const bool words = (reinterpret_cast<uintptr_t>(row) & 3) == 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int c = column(c_block, i);
                if constexpr (sizeof(T) == 4) {
                    w[i] = c < cols ? __ldg(reinterpret_cast<const unsigned*>(row) + c) : 0u;
                } else if (words && c + 1 < cols) {
                    w[i] = __ldg(reinterpret_cast<const unsigned*>(row + c));
                } else {
                    const unsigned short* h = reinterpret_cast<const unsigned short*>(row) + c;
                    const unsigned lo = c < cols ? __ldg(h) : 0u, hi = c + 1 < cols ? __ldg(h + 1) : 0u;
                    w[i] = lo | hi << 16;
                }
            }
        }
    }
    __device__ static __forceinline__ void store(T* row, int c_block, int cols, const Chunk<T>& k) {
        if constexpr (!STRIDED) {
            const int c0 = c_block + (int)(threadIdx.x % 32) * E;
            if (c0 < cols) k.store(row + c0, min(E, cols - c0));
        } else {
            unsigned w[8];
            k.to_words(w);
            const bool words = (reinterpret_cast<uintptr_t>(row) & 3) == 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int c = column(c_block, i);
                if constexpr (sizeof(T) == 4) {
                    if (c < cols) reinterpret_cast<unsigned*>(row)[c] = w[i];
                } else if (words && c + 1 < cols) {
                    *reinterpret_cast<unsigned*>(row + c) = w[i];
                } else {
                    unsigned short* h = reinterpret_cast<unsigned short*>(row) + c;
                    if (c < cols) h[0] = (unsigned short)w[i];
                    if (c + 1 < cols) h[1] = (unsigned short)(w[i] >> 16);
                }
            }
        }
    }
    // The block in fp32, in a row that starts on a 16-byte boundary and has whole chunks.
    __device__ static __forceinline__ void store_part(float* row, int c_block, int cols, const Chunk<T>& k) {
        if constexpr (!STRIDED) {
            const int c0 = c_block + (int)(threadIdx.x % 32) * E;
            if (c0 >= cols) return;
#pragma unroll
            for (int i = 0; i < E / 4; ++i)
                reinterpret_cast<float4*>(row + c0)[i] = make_float4(k.v[2 * i].x, k.v[2 * i].y, k.v[2 * i + 1].x, k.v[2 * i + 1].y);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int c = column(c_block, i);
                if (c >= cols) continue;
                if constexpr (kPer == 2)
                    *reinterpret_cast<float2*>(row + c) = k.v[i % (E / 2)];
                else
                    row[c] = i % 2 ? k.v[i / 2].y : k.v[i / 2].x;
            }
        }
    }
    __device__ static __forceinline__ void add_part(const float* row, int c_block, int cols, Chunk<T>& k) {
        if constexpr (!STRIDED) {
            const int c0 = c_block + (int)(threadIdx.x % 32) * E;
            if (c0 >= cols) return;
#pragma unroll
            for (int i = 0; i < E / 4; ++i) {
                const float4 f = __ldcg(reinterpret_cast<const float4*>(row + c0) + i);
                k.v[2 * i] = __fadd2_rn(k.v[2 * i], make_float2(f.x, f.y));
                k.v[2 * i + 1] = __fadd2_rn(k.v[2 * i + 1], make_float2(f.z, f.w));
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int c = column(c_block, i);
                if (c >= cols) continue;
                if constexpr (kPer == 2)
                    k.v[i % (E / 2)] = __fadd2_rn(k.v[i % (E / 2)], __ldcg(reinterpret_cast<const float2*>(row + c)));
                else
                    (i % 2 ? k.v[i / 2].y : k.v[i / 2].x) += __ldcg(row + c);
            }
        }
    }
};

// Zeros to a row, by `threads` threads: whole 32-byte vectors on their boundaries, and
// the elements before and behind them.
template <typename T>
__device__ __forceinline__ void zero_row(T* row, int cols, int t, int threads) {
    constexpr int E = 32 / (int)sizeof(T);
    const int over = (int)(reinterpret_cast<uintptr_t>(row) & 31) / (int)sizeof(T), head = min(over ? E - over : 0, cols);
    const int vectors = (cols - head) / E, tail = cols - head - vectors * E;
    for (int i = t; i < vectors; i += threads)
        asm volatile("st.global.v8.b32 [%0], {%1, %1, %1, %1, %1, %1, %1, %1};" ::"l"(row + head + (long long)i * E), "r"(0u) : "memory");
    if (t < head) store_elem(row + t, 0.0f);
    if (t < tail) store_elem(row + head + vectors * E + t, 0.0f);
}

// y[n] = scale * weight[token[n]]; bound by the reads and writes of rows (8192 of
// 128000 x 8192 bf16: 37 us, 5.4 TB/s).  A block takes a slab of one row, or whole rows.
template <typename T, bool STRIDED, int U>
__global__ void __launch_bounds__(kThreads) embed_forward_kernel(const void* __restrict__ tokens, bool wide, unsigned n, const T* __restrict__ weight,
                                                                 long long ld_w, long long vocab, int cols, float scale, T* __restrict__ y, long long ld_y,
                                                                 int row_threads, unsigned slabs) {
    using K = Chunk<T>;
    const unsigned group = blockIdx.x / slabs, slab = blockIdx.x - group * slabs;
    const unsigned row = group * (unsigned)(kThreads / row_threads) + threadIdx.x / (unsigned)row_threads;
    if (row >= n) return;
    const int c_first = ((int)slab * U * row_threads + (int)(threadIdx.x % (unsigned)row_threads) / 32 * 32) * K::kElems, c_step = row_threads * K::kElems;
    const long long token = load_index(tokens, row, wide);
    const bool known = token >= 0 && token < vocab;
    unsigned w[U][8];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (known && c_first + u * c_step < cols) {
            Block<T, STRIDED>::load_words(weight + token * ld_w, c_first + u * c_step, cols, w[u]);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) w[u][i] = 0xFFFFFFFFu;  // NaN in either type
        }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        K k;
        k.from_words(w[u]);
        k.scale(scale);
        if (c_first + u * c_step < cols) Block<T, STRIDED>::store(y + row * ld_y, c_first + u * c_step, cols, k);
    }
}

// ---------------------------------------------------------------------------
// sorting tokens: a radix sort that keeps the order of equal keys, eight bits a pass

constexpr int kBits = 8, kBins = 1 << kBits;
constexpr int kSortWarps = 8, kRounds = 8;
constexpr int kTile = 32 * kSortWarps * kRounds;

// The sort key of a token: itself, or `vocab` for one whose row gets no gradient
// (behind all others).
struct Keys {
    const void* tokens;
    long long vocab, padding;
    bool wide;
    __device__ __forceinline__ unsigned operator()(unsigned i) const {
        const long long t = load_index(tokens, i, wide);
        return t >= 0 && t < vocab && t != padding ? (unsigned)t : (unsigned)vocab;
    }
};

// Few tokens: a token's place is the number of those before it in the order, which is
// counted by comparing it with all.  Keys get the place they have now in their low
// bits, so that no two are alike.  A CTA takes 64 tokens, two to a lane, and each of
// its warps a part of the others: 16.8 million comparisons for 4096 tokens, bound by
// the comparisons' two instructions.  A whole gradient of 120000 rows of 64 fp32 takes
// 21 us with 4096 tokens and 25 us with 8192, with the other sort 51 us.
constexpr int kRankBits = 13, kRankTokens = 1 << kRankBits, kRankWarps = 32, kRankShare = 64;
constexpr long long kRankVocab = 1LL << (32 - kRankBits);  // keys below it, `vocab` itself among them

__device__ __forceinline__ void count_below(unsigned k, unsigned mine, unsigned& rank) {
    asm("{\n.reg .pred p;\nsetp.lt.u32 p, %1, %2;\n@p add.u32 %0, %0, 1;\n}" : "+r"(rank) : "r"(k), "r"(mine));
}

__global__ void __launch_bounds__(32 * kRankWarps) sort_few_kernel(const Keys key_of, unsigned n, unsigned* __restrict__ keys, unsigned* __restrict__ places,
                                                                   unsigned* __restrict__ some, unsigned* __restrict__ arrived, unsigned counters) {
    extern __shared__ uint4 s_all[];
    __shared__ unsigned s_rank[kRankWarps][kRankShare];
    unsigned* all = reinterpret_cast<unsigned*>(s_all);
    const unsigned padded = (n + 4 * kRankWarps - 1) / (4 * kRankWarps) * (4 * kRankWarps);
    for (unsigned i0 = threadIdx.x; i0 < padded; i0 += 8 * 32 * kRankWarps) {
        unsigned k[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) {  // eight loads in flight
            const unsigned i = i0 + u * 32 * kRankWarps;
            k[u] = i < n ? key_of(i) << kRankBits | i : 0xFFFFFFFFu;
        }
#pragma unroll
        for (int u = 0; u < 8; ++u)
            if (i0 + u * 32 * kRankWarps < padded) all[i0 + u * 32 * kRankWarps] = k[u];
    }
    for (unsigned i = blockIdx.x * 32 * kRankWarps + threadIdx.x; i < counters; i += gridDim.x * 32 * kRankWarps) arrived[i] = 0;
    __syncthreads();
    const unsigned warp = threadIdx.x / 32, lane = threadIdx.x % 32, base = blockIdx.x * kRankShare;
    const unsigned mine0 = base + lane < n ? all[base + lane] : 0u, mine1 = base + 32 + lane < n ? all[base + 32 + lane] : 0u;
    unsigned rank0 = 0, rank1 = 0;
    const unsigned quads = padded / (4 * kRankWarps);
#pragma unroll 4
    for (unsigned j = 0; j < quads; ++j) {
        const uint4 k = s_all[warp * quads + j];
        count_below(k.x, mine0, rank0);
        count_below(k.y, mine0, rank0);
        count_below(k.z, mine0, rank0);
        count_below(k.w, mine0, rank0);
        count_below(k.x, mine1, rank1);
        count_below(k.y, mine1, rank1);
        count_below(k.z, mine1, rank1);
        count_below(k.w, mine1, rank1);
    }
    s_rank[warp][lane] = rank0;
    s_rank[warp][32 + lane] = rank1;
    __syncthreads();
    const unsigned i = base + threadIdx.x;
    if (threadIdx.x < kRankShare && i < n) {
        unsigned rank = 0;
#pragma unroll
        for (int w = 0; w < kRankWarps; ++w) rank += s_rank[w][threadIdx.x];
        const unsigned key = all[i] >> kRankBits;
        keys[rank] = key;
        places[rank] = i;
        if (key != (unsigned)key_of.vocab) some[key] = rank;
    }
}

__global__ void __launch_bounds__(kThreads) token_keys_kernel(const Keys key_of, unsigned n, unsigned* __restrict__ keys, unsigned* __restrict__ arrived, unsigned counters) {
    const unsigned stride = gridDim.x * kThreads;
    for (unsigned i = blockIdx.x * kThreads + threadIdx.x; i < n; i += stride) keys[i] = key_of(i);
    for (unsigned i = blockIdx.x * kThreads + threadIdx.x; i < counters; i += stride) arrived[i] = 0;
}

__global__ void __launch_bounds__(kThreads) sort_count_kernel(const unsigned* __restrict__ keys, unsigned n, int shift, unsigned tiles, unsigned* __restrict__ counts) {
    __shared__ unsigned bins[kBins];
    bins[threadIdx.x] = 0;
    __syncthreads();
    for (int r = 0; r < kTile / kThreads; ++r) {
        const unsigned i = blockIdx.x * (unsigned)kTile + r * kThreads + threadIdx.x;
        if (i < n) atomicAdd(bins + (keys[i] >> shift & (kBins - 1)), 1u);
    }
    __syncthreads();
    counts[(size_t)threadIdx.x * tiles + blockIdx.x] = bins[threadIdx.x];
}

// Exclusive prefix sum over the threads of a CTA of kThreads; `total` is the sum.
__device__ __forceinline__ unsigned block_scan(unsigned v, unsigned* warps, unsigned* total) {
    unsigned s = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const unsigned u = __shfl_up_sync(0xFFFFFFFFu, s, o);
        if (threadIdx.x % 32 >= (unsigned)o) s += u;
    }
    __syncthreads();
    if (threadIdx.x % 32 == 31) warps[threadIdx.x / 32] = s;
    __syncthreads();
    unsigned before = 0, all = 0;
#pragma unroll
    for (unsigned w = 0; w < kThreads / 32; ++w) {
        if (w < threadIdx.x / 32) before += warps[w];
        all += warps[w];
    }
    *total = all;
    return before + s - v;
}

// One digit to a CTA: where each tile's keys of that digit begin among the digit's.
__global__ void __launch_bounds__(kThreads) sort_scan_kernel(unsigned* __restrict__ counts, unsigned tiles, unsigned* __restrict__ totals) {
    __shared__ unsigned warps[kThreads / 32];
    unsigned* row = counts + (size_t)blockIdx.x * tiles;
    unsigned before = 0;
    for (unsigned t0 = 0; t0 < tiles; t0 += kThreads) {
        const unsigned t = t0 + threadIdx.x, v = t < tiles ? row[t] : 0u;
        unsigned sum;
        const unsigned at = before + block_scan(v, warps, &sum);
        if (t < tiles) row[t] = at;
        before += sum;
    }
    if (threadIdx.x == 0) totals[blockIdx.x] = before;
}

// Puts a tile's keys in their places.  A warp takes 32 * kRounds neighbouring keys, 32 at
// a time, so that equal digits keep their order.  `places` is NULL in the first pass,
// `some` in all but the last.
__global__ void __launch_bounds__(kThreads) sort_scatter_kernel(const unsigned* __restrict__ keys, const unsigned* __restrict__ places, unsigned n, int shift,
                                                                unsigned tiles, const unsigned* __restrict__ counts, const unsigned* __restrict__ totals,
                                                                unsigned* __restrict__ keys_out, unsigned* __restrict__ places_out,
                                                                unsigned* __restrict__ some, unsigned none) {
    __shared__ unsigned warps[kThreads / 32];
    __shared__ unsigned at[kSortWarps][kBins];
    const unsigned warp = threadIdx.x / 32, lane = threadIdx.x % 32;
#pragma unroll
    for (int w = 0; w < kSortWarps; ++w) at[w][threadIdx.x] = 0;
    __syncthreads();
    const unsigned first = blockIdx.x * (unsigned)kTile + warp * 32 * kRounds;
    unsigned key[kRounds], rank[kRounds];
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
        const unsigned i = first + 32 * r + lane;
        const bool there = i < n;
        key[r] = there ? keys[i] : 0u;
        const unsigned digit = there ? key[r] >> shift & (kBins - 1) : kBins;
        const unsigned same = __match_any_sync(0xFFFFFFFFu, digit);
        const unsigned mine = same & ((1u << lane) - 1);
        unsigned base = 0;
        if (there) base = at[warp][digit];
        __syncwarp();
        if (there && mine == 0) at[warp][digit] = base + __popc(same);
        __syncwarp();
        rank[r] = base + __popc(mine);
    }
    __syncthreads();
    unsigned sum;
    unsigned begin = block_scan(totals[threadIdx.x], warps, &sum) + counts[(size_t)threadIdx.x * tiles + blockIdx.x];
#pragma unroll
    for (int w = 0; w < kSortWarps; ++w) {
        const unsigned c = at[w][threadIdx.x];
        at[w][threadIdx.x] = begin;
        begin += c;
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
        const unsigned i = first + 32 * r + lane;
        if (i >= n) continue;
        const unsigned to = at[warp][key[r] >> shift & (kBins - 1)] + rank[r];
        keys_out[to] = key[r];
        places_out[to] = places ? places[i] : i;
        if (some && key[r] != none) some[key[r]] = to;
    }
}

// ---------------------------------------------------------------------------
// sums over runs of equal tokens

struct GradArgs {
    const void* gy;
    const unsigned *keys, *places, *some;
    unsigned* arrived;
    float* part;
    void* gw;
    long long vocab, ld_gy, pitch;
    unsigned n, pieces, slabs, blocks;  // blocks: of 32 chunks, in a row
    int cols, piece, row_threads;
    unsigned sum_blocks, mix;
    float scale;
};

template <typename T, bool STRIDED>
__device__ __forceinline__ void store_scaled(const GradArgs& a, unsigned token, int c_block, Chunk<T> k) {
    k.scale(a.scale);
    Block<T, STRIDED>::store(static_cast<T*>(a.gw) + (long long)token * a.cols, c_block, a.cols, k);
}

// The first and the last entry of the run that entry `at` is in: the warp looks at the
// 32 neighbours on either side, and at 32 places spread over what is left where those
// are all of the run.
__device__ __forceinline__ void run_ends(const GradArgs& a, unsigned token, unsigned at, unsigned& first, unsigned& last) {
    const unsigned off = threadIdx.x % 32 + 1;
    const bool down = off <= at && __ldg(a.keys + (at - min(off, at))) == token;
    const bool up = off < a.n - at && __ldg(a.keys + min(at + off, a.n - 1)) == token;
    const unsigned many_down = __popc(__ballot_sync(0xFFFFFFFFu, down)), many_up = __popc(__ballot_sync(0xFFFFFFFFu, up));
    first = at - many_down;  // equal keys are neighbours: lanes from the first on
    last = at + many_up;
    if (many_down == 32) {
        unsigned gap = first + 1;  // entries from here down to the nearest one known not to be of the run (or none)
        while (gap > 1) {
            const unsigned step = (gap + 32) / 33;
            const unsigned many = __popc(__ballot_sync(0xFFFFFFFFu, step * off < gap && __ldg(a.keys + (first - min(step * off, first))) == token));
            first -= step * many;
            gap = min(gap - step * many, step);
        }
    }
    if (many_up == 32) {
        unsigned gap = a.n - last;
        while (gap > 1) {
            const unsigned step = (gap + 32) / 33;
            const unsigned many = __popc(__ballot_sync(0xFFFFFFFFu, step * off < gap && __ldg(a.keys + min(last + step * off, a.n - 1)) == token));
            last += step * many;
            gap = min(gap - step * many, step);
        }
    }
}

// Whether this warp is the last of `all` to come to a counter; what the others wrote
// before they came is then there to be read.
__device__ __forceinline__ bool last_to_come(unsigned* counter, unsigned all) {
    __threadfence();
    __syncwarp();
    unsigned come = 0;
    if (threadIdx.x % 32 == 0) come = atomicAdd(counter, 1u);
    come = __shfl_sync(0xFFFFFFFFu, come, 0);
    __threadfence();
    return come == all - 1;
}

// A partial sum of a run that was cut: the piece's first partial row for a run that
// began before it, its second for one that begins in it.  The last of the run's pieces
// to come (a warp of 32 chunks to a piece) adds them up in order.  Long runs are added
// up in groups of about the root of their pieces first, by the last of each group, and
// then the groups' sums by the last of these: 512 pieces took 90 us in one row.  One run in rows
// of 4096 bf16, the whole gradient at once and in groups: 8 pieces 12.6 and 13.3 us, 16 pieces 17.3 and 15.0 us.
constexpr unsigned kOneGroup = 8;

template <typename T, bool STRIDED>
__device__ void leave_part(const GradArgs& a, unsigned token, unsigned piece, bool before, int c_block, unsigned block, Chunk<T> k) {
    using B = Block<T, STRIDED>;
    const unsigned anchor = before ? piece * (unsigned)a.piece : min((piece + 1) * (unsigned)a.piece, a.n) - 1;
    unsigned first, last;
    run_ends(a, token, anchor, first, last);
    first /= (unsigned)a.piece;
    last /= (unsigned)a.piece;
    const unsigned count = last - first + 1, size = count <= kOneGroup ? count : (unsigned)ceilf(sqrtf((float)count));
    // a piece's row for this run; no two runs have the same
    auto row = [&](unsigned p) { return 2LL * p + (p == first ? 1 : 0); };
    B::store_part(a.part + row(piece) * a.pitch, c_block, a.cols, k);
    const unsigned head = first + (piece - first) / size * size, end = min(head + size - 1, last);
    if (!last_to_come(a.arrived + row(head) * a.blocks + block, end - head + 1)) return;
    k.zero();
#pragma unroll 4
    for (unsigned p = head; p <= end; ++p) B::add_part(a.part + row(p) * a.pitch, c_block, a.cols, k);
    if (size < count) {
        B::store_part(a.part + row(head) * a.pitch, c_block, a.cols, k);
        const unsigned groups = (count + size - 1) / size;
        if (!last_to_come(a.arrived + (2LL * a.pieces + first) * a.blocks + block, groups)) return;
        k.zero();
#pragma unroll 4
        for (unsigned g = 0; g < groups; ++g) B::add_part(a.part + row(first + g * size) * a.pitch, c_block, a.cols, k);
    }
    store_scaled<T, STRIDED>(a, token, c_block, k);
}

// Some blocks sum: `piece` sorted tokens and a slab of columns to a group of
// row_threads threads; a run inside a piece is stored at once.  The others write zeros
// to the rows of no token, those v for which keys[some[v]] is not v (`some` was written
// for the tokens that there are and holds anything elsewhere).  The sums wait for their
// loads, the zeros for the memory: one block in `mix` sums while there are any to do.
// 8192 tokens of 128000 x 8192 bf16 358 us with the sort (6.2 TB/s), bound by HBM; 8192
// of 1000 x 257 and the like by the chain of key, row, sum and join (8 us).
template <typename T, bool STRIDED>
__global__ void __launch_bounds__(kThreads, 2) embed_backward_kernel(const GradArgs a) {
    using K = Chunk<T>;
    const int group = threadIdx.x / a.row_threads, t = threadIdx.x % a.row_threads, groups = kThreads / a.row_threads;
    const unsigned lane = threadIdx.x % 32;
    const unsigned turn = blockIdx.x / a.mix, place = blockIdx.x - turn * a.mix;
    if (place != 0 || turn >= a.sum_blocks) {
        const unsigned fill = blockIdx.x - (turn >= a.sum_blocks ? a.sum_blocks : turn + 1);
        const long long v0 = ((long long)fill * groups + group) * 32;
        bool unused = v0 + lane < a.vocab;
        if (unused && a.n > 0) {
            const unsigned e = __ldg(a.some + v0 + lane);
            unused = e >= a.n || __ldg(a.keys + e) != (unsigned)(v0 + lane);
        }
        for (unsigned rows = __ballot_sync(0xFFFFFFFFu, unused); rows; rows &= rows - 1)
            zero_row(static_cast<T*>(a.gw) + (v0 + __ffs(rows) - 1) * a.cols, a.cols, t, a.row_threads);
        return;
    }
    const unsigned item = turn / a.slabs, slab = turn - item * a.slabs;
    const unsigned piece = item * (unsigned)groups + (unsigned)group;
    if (piece >= a.pieces) return;
    const unsigned block = (slab * (unsigned)a.row_threads + (unsigned)t) / 32;
    if (block >= a.blocks) return;  // a warp behind the last column
    const int c_block = (int)block * 32 * K::kElems;
    const unsigned begin = piece * (unsigned)a.piece, here = min((unsigned)a.piece, a.n - begin);  // at most 32
    const unsigned none = (unsigned)a.vocab;
    // a lane's entry of the piece, and the keys on its borders
    const unsigned my_key = lane < here ? __ldg(a.keys + begin + lane) : none, my_place = lane < here ? __ldg(a.places + begin + lane) : 0u;
    const unsigned key_before = begin > 0 ? __ldg(a.keys + begin - 1) : none, key_after = begin + here < a.n ? __ldg(a.keys + begin + here) : none;
    const unsigned count = __popc(__ballot_sync(0xFFFFFFFFu, my_key != none));  // those of no row are the last ones
    if (count == 0) return;
    unsigned token = __shfl_sync(0xFFFFFFFFu, my_key, 0);
    bool before = key_before == token;
    K sum;
    sum.zero();
    constexpr int kAhead = 4;
    for (unsigned e = 0; e < count; e += kAhead) {
        unsigned w[kAhead][8];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const unsigned from = __shfl_sync(0xFFFFFFFFu, my_place, (e + u) % 32);
            if (e + u < count) Block<T, STRIDED>::load_words(static_cast<const T*>(a.gy) + (long long)from * a.ld_gy, c_block, a.cols, w[u]);
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (e + u >= count) break;
            const unsigned key = __shfl_sync(0xFFFFFFFFu, my_key, e + u);
            if (key != token) {
                if (before)
                    leave_part<T, STRIDED>(a, token, piece, true, c_block, block, sum);
                else
                    store_scaled<T, STRIDED>(a, token, c_block, sum);
                token = key;
                before = false;
                sum.zero();
            }
            K k;
            k.from_words(w[u]);
#pragma unroll
            for (int i = 0; i < K::kElems / 2; ++i) sum.v[i] = __fadd2_rn(sum.v[i], k.v[i]);
        }
    }
    if (before || (count == here && key_after == token))
        leave_part<T, STRIDED>(a, token, piece, before, c_block, block, sum);
    else
        store_scaled<T, STRIDED>(a, token, c_block, sum);
}

// ---------------------------------------------------------------------------
// host side

constexpr long long kMaxBytes = 1LL << 52;

// Where everything lies in the workspace.
struct Plan {
    long long some, arrived, keys[2], places[2], counts, totals, part, bytes;
    long long pitch;
    unsigned tiles, pieces, blocks;
    int piece, passes;
    bool few;
    Plan(int dtype, long long n, long long vocab, long long cols, int sms) {
        const int elems = dtype == AMPQ_F32 ? 8 : 16;
        const RowSplit split(cols, elems);
        // longer pieces while there is enough to do for every SM; a lane has an entry
        piece = 16;
        while (piece < 32 && n * (long long)split.slabs / piece > 16LL * sms) piece *= 2;
        pieces = (unsigned)((n + piece - 1) / piece);
        tiles = (unsigned)((n + kTile - 1) / kTile);
        passes = 1;
        while (passes * kBits < 32 && vocab >> (passes * kBits)) ++passes;
        few = n <= kRankTokens && vocab < kRankVocab;
        blocks = (unsigned)(((cols + elems - 1) / elems + 31) / 32);
        pitch = (cols + 15) / 16 * 16;
        long long at = 0;
        auto take = [&at](long long size) {
            const long long here = at;
            at += (size + 255) / 256 * 256;
            return here;
        };
        some = take(vocab * 4);
        arrived = take(counters() * 4);
        for (int i = 0; i < (few ? 1 : 2); ++i) {
            keys[i] = take(n * 4);
            places[i] = take(n * 4);
        }
        counts = take(few ? 0 : (long long)tiles * kBins * 4);
        totals = take(few ? 0 : kBins * 4);
        part = take(2LL * pieces * pitch * 4);
        bytes = at;
    }
    long long counters() const { return 3LL * pieces * blocks; }  // of a piece's two partial rows, and of a run's groups
    bool fits() const { return bytes <= kMaxBytes && counters() <= 0x7FFFFFFFLL; }
};

int check_embed(int dtype, int index_type, const void* tokens, long long n, long long vocab, long long cols) {
    if (!known_dtype(dtype) || !known_index(index_type)) return AMPQ_ERR_INVALID;
    if (n < 0 || vocab < 0 || cols < 0 || (n > 0 && !tokens)) return AMPQ_ERR_INVALID;
    if (n > kMaxRows || vocab > kMaxRows || cols > kMaxCols) return AMPQ_ERR_TOO_LARGE;
    if (!aligned_to(tokens, index_bytes(index_type))) return AMPQ_ERR_ALIGN;
    return AMPQ_OK;
}

// From so many slabs of rows on a thread takes two chunks.  Rows of 8192 bf16, one chunk and
// two: 512 tokens (1024 slabs) 3.4 and 3.6 us, 1024 tokens 5.2 and 4.8, 2048 tokens 9.4 and 8.7, 4096 tokens 19.5
// and 16.8, 8192 tokens 37.3 and 36.3.
constexpr long long kManyBlocks = 4096;

template <typename T>
int launch_embed(const void* tokens, bool wide, long long n, const void* weight, long long ld_w, long long vocab, long long cols, float scale, void* y,
                 long long ld_y, cudaStream_t st) {
    RowSplit split(cols, Chunk<T>::kElems);
    constexpr int kType = sizeof(T) == 4 ? AMPQ_F32 : AMPQ_BF16;
    const bool aligned = rows_aligned(weight, ld_w, kType) && rows_aligned(y, ld_y, kType);
    const bool two = split.slabs > 1 && n * split.slabs >= kManyBlocks;
    if (two) split.slabs = (split.slabs + 1) / 2;
    auto kernel = aligned ? (two ? embed_forward_kernel<T, false, 2> : embed_forward_kernel<T, false, 1>)
                          : (two ? embed_forward_kernel<T, true, 2> : embed_forward_kernel<T, true, 1>);
    const long long rows = kThreads / split.threads, blocks = (n + rows - 1) / rows * split.slabs;
    if (blocks > 0x7FFFFFFFLL) return AMPQ_ERR_TOO_LARGE;
    kernel<<<(unsigned)blocks, kThreads, 0, st>>>(tokens, wide, (unsigned)n, static_cast<const T*>(weight), ld_w, vocab, (int)cols, scale, static_cast<T*>(y),
                                                  ld_y, split.threads, split.slabs);
    return launched();
}

template <typename T>
int launch_sums(GradArgs a, cudaStream_t st) {
    const RowSplit split(a.cols, Chunk<T>::kElems);
    a.row_threads = split.threads;
    a.slabs = split.slabs;
    const long long groups = kThreads / split.threads;
    const long long sums = (a.pieces + groups - 1) / groups * split.slabs;
    const long long fills = (a.vocab + 32 * groups - 1) / (32 * groups);
    if (sums + fills > 0x7FFFFFFFLL) return AMPQ_ERR_TOO_LARGE;
    a.sum_blocks = (unsigned)sums;
    a.mix = sums > 0 ? (unsigned)(fills / sums + 1) : 1u;
    constexpr int kType = sizeof(T) == 4 ? AMPQ_F32 : AMPQ_BF16;
    auto kernel = rows_aligned(a.gy, a.ld_gy, kType) && rows_aligned(a.gw, a.cols, kType) ? embed_backward_kernel<T, false> : embed_backward_kernel<T, true>;
    kernel<<<(unsigned)(sums + fills), kThreads, 0, st>>>(a);
    return launched();
}

}  // namespace
}  // namespace ampq

using namespace ampq;

extern "C" {
#pragma GCC visibility push(default)

int ampq_embed_forward(int device, void* cuda_stream, int dtype, int index_type, const void* tokens, long long n, const void* weight, long long ld_w,
                       long long vocab, long long cols, float scale, void* y, long long ld_y) {
    int rc = check_embed(dtype, index_type, tokens, n, vocab, cols);
    if (!rc) rc = check_matrix(weight, vocab, cols, ld_w, dtype);
    if (!rc) rc = check_matrix(y, n, cols, ld_y, dtype);
    if (rc) return rc;
    CkptDevice cur(device);
    if (cur.status) return cur.status;
    if (n == 0 || cols == 0) return AMPQ_OK;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
    const bool wide = index_type == AMPQ_I64;
    return dtype == AMPQ_F32 ? launch_embed<float>(tokens, wide, n, weight, ld_w, vocab, cols, scale, y, ld_y, st)
                             : launch_embed<__nv_bfloat16>(tokens, wide, n, weight, ld_w, vocab, cols, scale, y, ld_y, st);
}

int ampq_embed_backward_workspace(int device, int dtype, long long n, long long vocab, long long cols, long long* bytes) {
    if (!bytes) return AMPQ_ERR_INVALID;
    const int rc = check_embed(dtype, AMPQ_I32, nullptr, 0, vocab, cols);
    if (rc) return rc;
    if (n < 0) return AMPQ_ERR_INVALID;
    if (n > kMaxRows) return AMPQ_ERR_TOO_LARGE;
    CkptDevice cur(device);
    if (cur.status) return cur.status;
    const int sms = sm_count(device);
    if (sms < 1) return AMPQ_ERR_CUDA;
    const Plan plan(dtype, n, vocab, cols, sms);
    if (!plan.fits()) return AMPQ_ERR_TOO_LARGE;
    *bytes = plan.bytes;
    return AMPQ_OK;
}

int ampq_embed_backward(int device, void* cuda_stream, int dtype, int index_type, const void* tokens, long long n, const void* gy, long long ld_gy,
                        long long vocab, long long cols, float scale, long long padding, void* gw, void* workspace, long long workspace_bytes) {
    int rc = check_embed(dtype, index_type, tokens, n, vocab, cols);
    if (!rc) rc = check_matrix(gy, n, cols, ld_gy, dtype);
    if (!rc) rc = check_matrix(gw, vocab, cols, cols, dtype);
    if (rc) return rc;
    if (cols > 0 && vocab > kMaxBytes / (cols * (long long)elem_bytes(dtype))) return AMPQ_ERR_TOO_LARGE;
    if (!aligned_to(workspace, 256)) return AMPQ_ERR_ALIGN;
    CkptDevice cur(device);
    if (cur.status) return cur.status;
    if (vocab == 0 || cols == 0) return AMPQ_OK;
    const int sms = sm_count(device);
    if (sms < 1) return AMPQ_ERR_CUDA;
    const Plan plan(dtype, n, vocab, cols, sms);
    if (!plan.fits()) return AMPQ_ERR_TOO_LARGE;
    if (!workspace || workspace_bytes < plan.bytes) return AMPQ_ERR_INVALID;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
    unsigned char* ws = static_cast<unsigned char*>(workspace);
    auto words = [ws](long long at) { return reinterpret_cast<unsigned*>(ws + at); };
    unsigned *some = words(plan.some), *arrived = words(plan.arrived);
    const unsigned counters = (unsigned)plan.counters();
    int from = 0;
    if (n > 0) {
        const Keys key_of{tokens, vocab, padding, index_type == AMPQ_I64};
        if (plan.few) {
            sort_few_kernel<<<(unsigned)((n + kRankShare - 1) / kRankShare), 32 * kRankWarps, (size_t)((n + 4 * kRankWarps - 1) / (4 * kRankWarps) * (16 * kRankWarps)), st>>>(
                key_of, (unsigned)n, words(plan.keys[0]), words(plan.places[0]), some, arrived, counters);
        } else {
            token_keys_kernel<<<(unsigned)((n + kThreads - 1) / kThreads), kThreads, 0, st>>>(key_of, (unsigned)n, words(plan.keys[0]), arrived, counters);
            for (int pass = 0; pass < plan.passes; ++pass, from ^= 1) {
                const unsigned *keys = words(plan.keys[from]), *places = pass ? words(plan.places[from]) : nullptr;
                sort_count_kernel<<<plan.tiles, kThreads, 0, st>>>(keys, (unsigned)n, pass * kBits, plan.tiles, words(plan.counts));
                sort_scan_kernel<<<kBins, kThreads, 0, st>>>(words(plan.counts), plan.tiles, words(plan.totals));
                sort_scatter_kernel<<<plan.tiles, kThreads, 0, st>>>(keys, places, (unsigned)n, pass * kBits, plan.tiles, words(plan.counts), words(plan.totals),
                                                                     words(plan.keys[from ^ 1]), words(plan.places[from ^ 1]),
                                                                     pass + 1 == plan.passes ? some : nullptr, (unsigned)vocab);
            }
        }
        rc = launched();
        if (rc) return rc;
    }
    GradArgs a{};
    a.gy = gy; a.gw = gw;
    a.keys = words(plan.keys[from]); a.places = words(plan.places[from]); a.some = some; a.arrived = arrived;
    a.part = reinterpret_cast<float*>(ws + plan.part);
    a.vocab = vocab; a.ld_gy = ld_gy; a.pitch = plan.pitch;
    a.n = (unsigned)n; a.pieces = plan.pieces; a.blocks = plan.blocks;
    a.cols = (int)cols; a.piece = plan.piece;
    a.scale = scale;
    return dtype == AMPQ_F32 ? launch_sums<float>(a, st) : launch_sums<__nv_bfloat16>(a, st);
}

#pragma GCC visibility pop
}  // extern "C"
