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

// y[n] = scale * weight[token[n]]; bound by the reads and writes of rows.  A block
// takes a slab of one row, or whole rows.
template <typename T>
__global__ void __launch_bounds__(kThreads) embed_forward_kernel(const void* __restrict__ tokens, bool wide, unsigned n, const T* __restrict__ weight,
                                                                 long long ld_w, long long vocab, int cols, float scale, T* __restrict__ y, long long ld_y,
                                                                 int row_threads, unsigned slabs) {
    using K = Chunk<T>;
    const unsigned group = blockIdx.x / slabs, slab = blockIdx.x - group * slabs;
    const unsigned row = group * (unsigned)(kThreads / row_threads) + threadIdx.x / (unsigned)row_threads;
    if (row >= n) return;
    const int c0 = ((int)slab * row_threads + (int)(threadIdx.x % (unsigned)row_threads)) * K::kElems;
    if (c0 >= cols) return;
    const int m = min(K::kElems, cols - c0);
    const long long token = load_index(tokens, row, wide);
    K k;
    if (token >= 0 && token < vocab) {
        k.load(weight + token * ld_w + c0, m);
        k.scale(scale);
    } else {
#pragma unroll
        for (int i = 0; i < K::kElems / 2; ++i) k.v[i] = make_float2(NAN, NAN);
    }
    k.store(y + row * ld_y + c0, m);
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
// bits, so that no two are alike.  A CTA takes 32 tokens, one to a lane, and each of
// its warps a part of the others; 8192 tokens are 6 us, three passes of the other sort
// 45 us, and at 16384 the two meet.
constexpr int kRankBits = 13, kRankTokens = 1 << kRankBits, kRankWarps = 8;
constexpr long long kRankVocab = 1LL << (32 - kRankBits);  // keys below it, `vocab` itself among them

__global__ void __launch_bounds__(32 * kRankWarps) sort_few_kernel(const Keys key_of, unsigned n, unsigned* __restrict__ keys, unsigned* __restrict__ places,
                                                                   unsigned* __restrict__ some, unsigned* __restrict__ arrived, unsigned counters) {
    extern __shared__ uint4 s_all[];
    __shared__ unsigned s_rank[kRankWarps][32];
    unsigned* all = reinterpret_cast<unsigned*>(s_all);
    const unsigned padded = (n + 4 * kRankWarps - 1) / (4 * kRankWarps) * (4 * kRankWarps);
    for (unsigned i = threadIdx.x; i < padded; i += 32 * kRankWarps) all[i] = i < n ? key_of(i) << kRankBits | i : 0xFFFFFFFFu;
    for (unsigned i = blockIdx.x * 32 * kRankWarps + threadIdx.x; i < counters; i += gridDim.x * 32 * kRankWarps) arrived[i] = 0;
    __syncthreads();
    const unsigned warp = threadIdx.x / 32, lane = threadIdx.x % 32, i = blockIdx.x * 32 + lane;
    const unsigned mine = i < n ? all[i] : 0;
    unsigned rank = 0;
    const unsigned quads = padded / (4 * kRankWarps);
#pragma unroll 4
    for (unsigned j = 0; j < quads; ++j) {
        const uint4 k = s_all[warp * quads + j];
        rank += (k.x < mine) + (k.y < mine) + (k.z < mine) + (k.w < mine);
    }
    s_rank[warp][lane] = rank;
    __syncthreads();
    if (warp == 0 && i < n) {
        rank = 0;
#pragma unroll
        for (int w = 0; w < kRankWarps; ++w) rank += s_rank[w][lane];
        const unsigned key = mine >> kRankBits;
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
    int cols, piece, row_threads, fill_rows;
    unsigned sum_blocks;
    float scale;
};

template <typename T>
__device__ __forceinline__ void store_scaled(const GradArgs& a, unsigned token, int c0, Chunk<T> k) {
    k.scale(a.scale);
    if (c0 < a.cols) k.store(static_cast<T*>(a.gw) + (long long)token * a.cols + c0, min(Chunk<T>::kElems, a.cols - c0));
}

// The first (or, `last`, the last) entry with this key, of which entry `at` is one: the
// warp looks at 32 places at a time.
__device__ __forceinline__ unsigned run_end(const GradArgs& a, unsigned token, unsigned at, bool last) {
    const unsigned lane = threadIdx.x % 32;
    unsigned inside = at, outside = last ? a.n : 0xFFFFFFFFu;  // (one before the first entry)
    while ((last ? outside - inside : inside - outside) > 1) {
        const unsigned gap = last ? outside - inside : inside - outside, step = (gap + 32) / 33;
        const unsigned probe = last ? inside + step * (lane + 1) : inside - step * (lane + 1);
        const bool valid = step * (lane + 1) < gap;
        const unsigned same = __ballot_sync(0xFFFFFFFFu, valid && __ldg(a.keys + probe) == token);
        const unsigned many = __popc(same);  // equal keys are neighbours: a run of lanes from the first on
        const unsigned in = step * many, out = step * (many + 1);
        if (last) {
            outside = out < gap ? inside + out : outside;
            inside += in;
        } else {
            outside = out < gap ? inside - out : outside;
            inside -= in;
        }
    }
    return inside;
}

// A partial sum of a run that was cut: the piece's first partial row for a run that
// began before it, its second for one that begins in it.  The last of the run's pieces
// to come (a warp of 32 chunks to a piece) adds them up in order.
template <typename T>
__device__ void leave_part(const GradArgs& a, unsigned token, unsigned piece, bool before, int c0, unsigned block, Chunk<T> k) {
    constexpr int kVectors = Chunk<T>::kElems / 4;
    if (c0 < a.cols) {  // whole chunks fit into the pitch
        float4* p = reinterpret_cast<float4*>(a.part + (2LL * piece + (before ? 0 : 1)) * a.pitch + c0);
#pragma unroll
        for (int i = 0; i < kVectors; ++i) p[i] = make_float4(k.v[2 * i].x, k.v[2 * i].y, k.v[2 * i + 1].x, k.v[2 * i + 1].y);
    }
    const unsigned anchor = before ? piece * (unsigned)a.piece : min((piece + 1) * (unsigned)a.piece, a.n) - 1;
    const unsigned first = run_end(a, token, anchor, false) / (unsigned)a.piece, last = run_end(a, token, anchor, true) / (unsigned)a.piece;
    __threadfence();
    __syncwarp();
    unsigned come = 0;
    if (threadIdx.x % 32 == 0) come = atomicAdd(a.arrived + (size_t)first * a.blocks + block, 1u);
    come = __shfl_sync(0xFFFFFFFFu, come, 0);
    if (come != last - first) return;
    __threadfence();
    if (c0 >= a.cols) return;
    k.zero();
    constexpr int kAhead = 4;
    for (unsigned p = first; p <= last; p += kAhead) {
        float4 f[kAhead][kVectors];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const float4* from = reinterpret_cast<const float4*>(a.part + (2LL * (p + u) + (p + u == first ? 1 : 0)) * a.pitch + c0);
#pragma unroll
            for (int i = 0; i < kVectors; ++i) f[u][i] = p + u <= last ? __ldcg(from + i) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
            if (p + u <= last)
#pragma unroll
                for (int i = 0; i < kVectors; ++i) {
                    k.v[2 * i] = __fadd2_rn(k.v[2 * i], make_float2(f[u][i].x, f[u][i].y));
                    k.v[2 * i + 1] = __fadd2_rn(k.v[2 * i + 1], make_float2(f[u][i].z, f[u][i].w));
                }
    }
    store_scaled<T>(a, token, c0, k);
}

// The first blocks sum: `piece` sorted tokens and a slab of columns to a group of
// row_threads threads; a run inside a piece is stored at once.  The other blocks write
// zeros to the rows of no token, those v for which keys[some[v]] is not v (`some` was
// written for the tokens that there are and holds anything elsewhere).
template <typename T>
__global__ void __launch_bounds__(kThreads) embed_backward_kernel(const GradArgs a) {
    using K = Chunk<T>;
    const int group = threadIdx.x / a.row_threads, t = threadIdx.x % a.row_threads, groups = kThreads / a.row_threads;
    if (blockIdx.x >= a.sum_blocks) {
        const long long v0 = (long long)(blockIdx.x - a.sum_blocks) * a.fill_rows;
        K zero;
        zero.zero();
        for (long long v = v0 + group; v < v0 + a.fill_rows && v < a.vocab; v += groups) {
            const unsigned e = a.n > 0 ? __ldg(a.some + v) : 0u;
            if (e < a.n && __ldg(a.keys + e) == (unsigned)v) continue;
            T* row = static_cast<T*>(a.gw) + v * a.cols;
            for (int c0 = t * K::kElems; c0 < a.cols; c0 += a.row_threads * K::kElems) zero.store(row + c0, min(K::kElems, a.cols - c0));
        }
        return;
    }
    const unsigned item = blockIdx.x / a.slabs, slab = blockIdx.x - item * a.slabs;
    const unsigned piece = item * (unsigned)groups + (unsigned)group;
    if (piece >= a.pieces) return;
    const int chunk = (int)slab * a.row_threads + t, c0 = chunk * K::kElems;
    const unsigned block = (unsigned)chunk / 32;
    if (block >= a.blocks) return;  // a warp behind the last column
    const int m = min(K::kElems, a.cols - c0);
    const unsigned begin = piece * (unsigned)a.piece, end = min(begin + (unsigned)a.piece, a.n);
    const unsigned none = (unsigned)a.vocab;
    unsigned token = __ldg(a.keys + begin);
    bool before = begin > 0 && __ldg(a.keys + begin - 1) == token;
    K sum;
    sum.zero();
    constexpr int kAhead = 4;
    for (unsigned e = begin; e < end && token != none; e += kAhead) {
        unsigned key[kAhead];
        unsigned w[kAhead][8];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            key[u] = e + u < end ? __ldg(a.keys + e + u) : none;
#pragma unroll
            for (int i = 0; i < 8; ++i) w[u][i] = 0;
            if (key[u] != none && m > 0) K::load_words(static_cast<const T*>(a.gy) + (long long)__ldg(a.places + e + u) * a.ld_gy + c0, m, w[u]);
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (e + u >= end || token == none) break;
            if (key[u] != token) {
                if (before)
                    leave_part<T>(a, token, piece, true, c0, block, sum);
                else
                    store_scaled<T>(a, token, c0, sum);
                token = key[u];
                before = false;
                sum.zero();
            }
            K k;
            k.from_words(w[u]);
#pragma unroll
            for (int i = 0; i < K::kElems / 2; ++i) sum.v[i] = __fadd2_rn(sum.v[i], k.v[i]);
        }
    }
    if (token == none) return;
    const bool after = end < a.n && __ldg(a.keys + end) == token;
    if (before || after)
        leave_part<T>(a, token, piece, before, c0, block, sum);
    else
        store_scaled<T>(a, token, c0, sum);
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
        // longer pieces while there is enough to do for every SM
        piece = 8;
        while (piece < 64 && n * (long long)split.slabs / piece > 16LL * sms) piece *= 2;
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
        arrived = take((long long)pieces * blocks * 4);
        for (int i = 0; i < (few ? 1 : 2); ++i) {
            keys[i] = take(n * 4);
            places[i] = take(n * 4);
        }
        counts = take(few ? 0 : (long long)tiles * kBins * 4);
        totals = take(few ? 0 : kBins * 4);
        part = take(2LL * pieces * pitch * 4);
        bytes = at;
    }
    bool fits() const { return bytes <= kMaxBytes && (long long)pieces * blocks <= 0x7FFFFFFFLL; }
};

int check_embed(int dtype, int index_type, const void* tokens, long long n, long long vocab, long long cols) {
    if (!known_dtype(dtype) || !known_index(index_type)) return AMPQ_ERR_INVALID;
    if (n < 0 || vocab < 0 || cols < 0 || (n > 0 && !tokens)) return AMPQ_ERR_INVALID;
    if (n > kMaxRows || vocab > kMaxRows || cols > kMaxCols) return AMPQ_ERR_TOO_LARGE;
    if (!aligned_to(tokens, index_bytes(index_type))) return AMPQ_ERR_ALIGN;
    return AMPQ_OK;
}

template <typename T>
int launch_embed(const void* tokens, bool wide, long long n, const void* weight, long long ld_w, long long vocab, long long cols, float scale, void* y,
                 long long ld_y, cudaStream_t st) {
    const RowSplit split(cols, Chunk<T>::kElems);
    const long long rows = kThreads / split.threads, blocks = (n + rows - 1) / rows * split.slabs;
    if (blocks > 0x7FFFFFFFLL) return AMPQ_ERR_TOO_LARGE;
    embed_forward_kernel<T><<<(unsigned)blocks, kThreads, 0, st>>>(tokens, wide, (unsigned)n, static_cast<const T*>(weight), ld_w, vocab, (int)cols, scale,
                                                                   static_cast<T*>(y), ld_y, split.threads, split.slabs);
    return launched();
}

template <typename T>
int launch_sums(GradArgs a, cudaStream_t st) {
    const RowSplit split(a.cols, Chunk<T>::kElems);
    a.row_threads = split.threads;
    a.slabs = split.slabs;
    const long long groups = kThreads / split.threads;
    const long long sums = (a.pieces + groups - 1) / groups * split.slabs;
    a.fill_rows = (int)groups * 4;
    const long long fills = (a.vocab + a.fill_rows - 1) / a.fill_rows;
    if (sums + fills > 0x7FFFFFFFLL) return AMPQ_ERR_TOO_LARGE;
    a.sum_blocks = (unsigned)sums;
    embed_backward_kernel<T><<<(unsigned)(sums + fills), kThreads, 0, st>>>(a);
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
    const unsigned counters = plan.pieces * plan.blocks;
    int from = 0;
    if (n > 0) {
        const Keys key_of{tokens, vocab, padding, index_type == AMPQ_I64};
        if (plan.few) {
            sort_few_kernel<<<(unsigned)((n + 31) / 32), 32 * kRankWarps, (size_t)((n + 4 * kRankWarps - 1) / (4 * kRankWarps) * (16 * kRankWarps)), st>>>(
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
