// Layer norm and RMS norm, forward and backward (include/ampq.h:
// ampq_norm_forward, ampq_norm_backward), with the 8-bit checkpoint of the
// input written by the forward pass and read by the backward pass.
#include "ampq_ckpt.h"

#include <atomic>
#include <cmath>

namespace ampq {
namespace {

constexpr int kMaxNormCols = AMPQ_NORM_MAX_COLS;

// One thread holds 16 * WIDE elements of a row: so many chunks.
template <typename T, int WIDE>
constexpr int kChunks = 16 * WIDE / Chunk<T>::kElems;

// Sums N values over the WPR warps of a row group; every thread of the CTA calls
// it.  The order is fixed.
template <int WPR, int N>
__device__ __forceinline__ void row_sum(float (&s)[N], float* red, int warp) {
#pragma unroll
    for (int k = 0; k < N; ++k)
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) s[k] += __shfl_xor_sync(0xFFFFFFFFu, s[k], o);
    if (WPR == 1) return;
    if ((threadIdx.x & 31) == 0)
#pragma unroll
        for (int k = 0; k < N; ++k) red[warp * N + k] = s[k];
    __syncthreads();
    // every lane takes one of the group's sums and they are added up as before
    constexpr int kLanes = WPR <= 2 ? 2 : WPR <= 4 ? 4 : WPR <= 8 ? 8 : WPR <= 16 ? 16 : 32;
    const int from = threadIdx.x & (kLanes - 1);
#pragma unroll
    for (int k = 0; k < N; ++k) {
        s[k] = from < WPR ? red[(warp / WPR * WPR + from) * N + k] : 0.0f;
#pragma unroll
        for (int o = kLanes / 2; o > 0; o >>= 1) s[k] += __shfl_xor_sync(0xFFFFFFFFu, s[k], o);
    }
}

template <int WPR, int WIDE>
struct Shape {
    static constexpr int kWarps = WPR < 8 ? 8 : WPR;   // warps of a CTA
    static constexpr int kGroups = kWarps / WPR;       // rows a CTA works on at a time
    static constexpr int kThreads = 32 * kWarps;
};

// 16 elements of a parameter vector in fp32, as pairs.
template <typename T>
__device__ __forceinline__ void load_params(const void* p, bool bf16, int c0, int n, Chunk<T>& k) {
    constexpr int E = Chunk<T>::kElems;
    if (bf16 == (sizeof(T) == 2)) {
        k.load(static_cast<const T*>(p) + c0, n);
        return;
    }
#pragma unroll
    for (int i = 0; i < E / 2; ++i) {
        float2 f = make_float2(0.0f, 0.0f);
        if (bf16) {
            const __nv_bfloat16* q = static_cast<const __nv_bfloat16*>(p) + c0;
            if (2 * i < n) f.x = load_elem(q + 2 * i);
            if (2 * i + 1 < n) f.y = load_elem(q + 2 * i + 1);
        } else {
            const float* q = static_cast<const float*>(p) + c0;
            if (2 * i < n) f.x = load_elem(q + 2 * i);
            if (2 * i + 1 < n) f.y = load_elem(q + 2 * i + 1);
        }
        k.v[i] = f;
    }
}

// Whole rows come by bulk copies, whose bytes an mbarrier counts.
__device__ __forceinline__ void row_expect(unsigned bar, unsigned bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void row_copy(unsigned dst, const void* src, unsigned bytes, unsigned bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
template <unsigned HINT_NS>
__device__ __forceinline__ bool row_poll(unsigned bar, unsigned parity) {
    unsigned ok;
    asm volatile(
        "{\n"
        ".reg .pred p;\n"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n"
        "selp.u32 %0, 1, 0, p;\n"
        "}\n"
        : "=r"(ok)
        : "r"(bar), "r"(parity), "n"(HINT_NS)
        : "memory");
    return ok != 0;
}
// Polls of a row before a wait gives up.  A test build lets the rows' waits give up at
// once; the wait that drains copies in flight keeps the full limit.
constexpr unsigned kDrainPolls = 1u << 22;
#ifdef AMPQ_TEST_SHORT_WAITS
constexpr unsigned kRowPolls = 0u, kRowHintNs = 0u;
#else
constexpr unsigned kRowPolls = 1u << 22, kRowHintNs = 2000u;
#endif
// Waits for a row, with a limit; false when it runs out or the row group has given up
// (a row that is there is taken all the same).  A thread that missed a row takes none
// after it: what it would have written becomes NaN, and through the sums that its
// group shares so do the group's outputs of that row.  The thread that copies goes by
// its own rows: one that it has seen has left its place; once it missed one it starts
// no more copies and waits for those in flight.
__device__ __forceinline__ bool row_wait(unsigned bar, unsigned parity, volatile int* gave_up) {
    if (row_poll<kRowHintNs>(bar, parity)) return true;
    for (unsigned i = 0; i < kRowPolls; ++i) {
        if (*gave_up) return false;
        if (row_poll<kRowHintNs>(bar, parity)) return true;
    }
    *gave_up = 1;
    return false;
}
__device__ __forceinline__ bool row_drain(unsigned bar, unsigned parity) {
    for (unsigned i = 0; i < kDrainPolls; ++i)
        if (row_poll<2000u>(bar, parity)) return true;
    return false;
}
constexpr unsigned kNanBits = 0x7FC00000u;

__device__ __forceinline__ uint4 take16(unsigned src) {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(src) : "memory");
    return v;
}

// A chunk that lies in shared memory as it does in its row: the upper four of
// eight lanes read their second half first, so that the eight meet all 32 banks.
__device__ __forceinline__ void take_words(unsigned at, unsigned lane, unsigned (&w)[8]) {
    const unsigned swap = (lane >> 2) & 1;
    const uint4 p = take16(at + 16 * swap), q = take16(at + 16 * (1 - swap));
    const uint4 lo = swap ? q : p, hi = swap ? p : q;
    w[0] = lo.x; w[1] = lo.y; w[2] = lo.z; w[3] = lo.w;
    w[4] = hi.x; w[5] = hi.y; w[6] = hi.z; w[7] = hi.w;
}

// Stores a warp's piece of a row whose rows do not start on 16-byte boundaries: its
// chunks go through `scratch` (1040 bytes of shared memory), so that a store writes
// 32 neighbouring words instead of 32 places 32 bytes apart.  p: the piece's first
// element, n of them; all lanes call it.
template <typename T>
__device__ __forceinline__ void store_piece(T* p, int n, const Chunk<T>& k, unsigned scratch, unsigned lane) {
    unsigned w[8];
    k.to_words(w);
    __syncwarp();
    asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(scratch + 32 * lane), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]) : "memory");
    asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(scratch + 32 * lane + 16), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7]) : "memory");
    __syncwarp();
    const bool between = reinterpret_cast<uintptr_t>(p) & 2;  // bf16 rows that start between two words
    constexpr int kPer = 4 / (int)sizeof(T);
    unsigned* q = reinterpret_cast<unsigned*>(reinterpret_cast<uintptr_t>(p) + (between ? 2 : 0));
    const int words = (between ? n - 1 : n) / kPer;           // whole words of the row
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int j = 32 * i + (int)lane;
        unsigned a, b;
        asm volatile("ld.shared.u32 %0, [%1];" : "=r"(a) : "r"(scratch + 4 * j) : "memory");
        asm volatile("ld.shared.u32 %0, [%1];" : "=r"(b) : "r"(scratch + 4 * j + 4) : "memory");
        if (j < words) q[j] = between ? __funnelshift_r(a, b, 16) : a;
    }
    if (sizeof(T) == 2 && lane < 2) {  // what is left at the ends: half a word each
        const int at = lane ? n - 1 : 0;
        const bool alone = lane ? (between ? (n - 1) % 2 == 1 : n % 2 == 1) && (n > 1 || !between) : between;
        unsigned short h;
        asm volatile("ld.shared.u16 %0, [%1];" : "=h"(h) : "r"(scratch + 2 * at) : "memory");
        if (alone) reinterpret_cast<unsigned short*>(p)[at] = h;
    }
}

struct ForwardArgs {
    const void *x, *w, *b;
    void* y;
    float *mean, *rstd;
    unsigned char *codes, *scales;
    long long rows, ld_x, ld_y, ld_codes, ld_scales;
    int cols;
    float eps;
    bool param_bf16;
    bool whole;  // the last chunk of a row is a whole one
    bool e4m3;   // the checkpoint's format
    bool bulk;   // rows can be copied whole, and there are several to a group
};

// CTAs of the forward pass that share an SM, and the shared memory of one: two
// rows of each row group, the current one and the next.
template <typename T, int WPR, int WIDE>
struct ForwardRing {
    static constexpr int kRow = 512 * WPR * WIDE * (int)sizeof(T);
    static constexpr int kBytes = 2 * Shape<WPR, WIDE>::kGroups * kRow;
    static constexpr int kFit = 200 * 1024 / kBytes, kThreadFit = 1024 / Shape<WPR, WIDE>::kThreads;
    static constexpr int kCtas = kFit < kThreadFit ? kFit : kThreadFit;
};

// A row to a group of WPR warps, held in registers between the statistics (mean,
// then the sum of squared differences from it) and the output, so x is read once.
// Thread t of a group holds the chunks (j * threads + t): neighbouring lanes make
// the groups of the checkpoint.  Where there are several rows to a group and their
// layout allows it, the next row comes by a bulk copy meanwhile.  Bound by HBM and
// the two barriers of a row: RMS norm of 8192 x 8192 bf16 with its checkpoint 57 us
// (5.9 TB/s; 67 us without the copies ahead, 81 us with 16 elements to a thread).
template <typename T, bool KEPT, bool LAYER, int WPR, int WIDE>
__global__ void __launch_bounds__(Shape<WPR, WIDE>::kThreads, ForwardRing<T, WPR, WIDE>::kCtas) norm_forward_kernel(const ForwardArgs a) {
    using S = Shape<WPR, WIDE>;
    using K = Chunk<T>;
    using Ring = ForwardRing<T, WPR, WIDE>;
    constexpr int V = kChunks<T, WIDE>, E = K::kElems;
    extern __shared__ __align__(128) unsigned char rows_smem[];
    __shared__ float red[2][2][S::kWarps];
    __shared__ alignas(16) unsigned char s_scratch[S::kWarps][1040];
    __shared__ alignas(8) unsigned long long s_bars[2 * S::kGroups];
    __shared__ int s_gave_up[S::kGroups];
    const int warp = threadIdx.x / 32, group = warp / WPR;
    volatile int* gave_up = s_gave_up + group;
    const int t = threadIdx.x % (32 * WPR);
    const unsigned lane = threadIdx.x % 32;
    const long long stride = (long long)gridDim.x * S::kGroups, first = (long long)blockIdx.x * S::kGroups + group;
    const unsigned slots = (unsigned)__cvta_generic_to_shared(rows_smem) + 2 * group * Ring::kRow;
    const unsigned bars = (unsigned)__cvta_generic_to_shared(s_bars) + 16 * group;
    const unsigned row_bytes = (unsigned)a.cols * (unsigned)sizeof(T);
    auto begin_copy = [&](long long row, int slot) {
        row_expect(bars + 8 * slot, row_bytes);
        row_copy(slots + slot * Ring::kRow, static_cast<const T*>(a.x) + row * a.ld_x, row_bytes, bars + 8 * slot);
    };
    if (a.bulk) {
        if (t == 0) {
            asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(bars) : "memory");
            asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(bars + 8) : "memory");
            *gave_up = 0;
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        }
        __syncthreads();
        if (t == 0) {
            if (first < a.rows) begin_copy(first, 0);
            if (first + stride < a.rows) begin_copy(first + stride, 1);
        }
    }
    const float inv_cols = 1.0f / (float)a.cols;
    int taken = 0;  // rows of this group so far
    bool late = false;  // this thread missed a row
    for (long long row0 = (long long)blockIdx.x * S::kGroups; row0 < a.rows; row0 += stride, ++taken) {
        const long long row = row0 + group;
        const bool live = row < a.rows;
        const int slot = taken & 1;
        if (a.bulk && live && !late && !row_wait(bars + 8 * slot, (taken >> 1) & 1, gave_up)) {
            late = true;
            if (t == 0 && row_drain(bars + 8 * slot, (taken >> 1) & 1) && row + stride < a.rows) row_drain(bars + 8 * (slot ^ 1), ((taken + 1) >> 1) & 1);
        }
        K k[V];
        int n[V];
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const int c0 = (j * 32 * WPR + t) * E;
            n[j] = live ? min(E, a.cols - c0) : 0;
            k[j].zero();
            if (a.bulk) {
                unsigned w[8];
                take_words(slots + slot * Ring::kRow + (j * 32 * WPR + t) * 32, lane, w);
                if (n[j] > 0) k[j].from_words(w);
                if (late) k[j].v[0].x = __uint_as_float(kNanBits);  // and so the row's sums and the checkpoint's group
            } else if (n[j] > 0) {
                k[j].load(static_cast<const T*>(a.x) + row * a.ld_x + c0, n[j]);
            }
        }
        float mean = 0.0f;
        if (LAYER) {
            float2 s2 = make_float2(0.0f, 0.0f);
#pragma unroll
            for (int j = 0; j < V; ++j)
#pragma unroll
                for (int i = 0; i < E / 2; ++i) s2 = __fadd2_rn(s2, k[j].v[i]);
            float s[1] = {s2.x + s2.y};
            row_sum<WPR, 1>(s, red[slot][0], warp);
            mean = s[0] * inv_cols;
        }
        const float2 minus = make_float2(-mean, -mean);
        float2 q2 = make_float2(0.0f, 0.0f);
        if (!LAYER || a.whole) {
#pragma unroll
            for (int j = 0; j < V; ++j) {
                if (LAYER && n[j] <= 0) continue;
#pragma unroll
                for (int i = 0; i < E / 2; ++i) {
                    const float2 d = LAYER ? __fadd2_rn(k[j].v[i], minus) : k[j].v[i];
                    q2 = __ffma2_rn(d, d, q2);
                }
            }
        } else {
#pragma unroll
            for (int j = 0; j < V; ++j)
#pragma unroll
                for (int i = 0; i < E / 2; ++i) {
                    float2 d = __fadd2_rn(k[j].v[i], minus);
                    d = make_float2(2 * i < n[j] ? d.x : 0.0f, 2 * i + 1 < n[j] ? d.y : 0.0f);
                    q2 = __ffma2_rn(d, d, q2);
                }
        }
        float q[1] = {q2.x + q2.y};
        row_sum<WPR, 1>(q, red[slot][1], warp);
        // every thread of the group has read its part of the row: its place takes the row after the next
        if (WPR == 1) __syncwarp();
        if (a.bulk && t == 0 && !late && row + 2 * stride < a.rows) begin_copy(row + 2 * stride, slot);
        const float rstd = 1.0f / sqrtf(q[0] * inv_cols + a.eps);
        if (live && t == 0) {
            if (LAYER) a.mean[row] = mean;
            a.rstd[row] = rstd;
        }
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const int c0 = (j * 32 * WPR + t) * E;
            if (KEPT) {
                const unsigned amax = k[j].group_amax();
                const unsigned byte = a.e4m3 ? scale_byte<AMPQ_FMT_E4M3>(amax) : scale_byte<AMPQ_FMT_E5M2>(amax);
                if (live && (c0 & ~(kGroup - 1)) < a.cols) {  // whole groups: the columns behind the last are stored as 0
                    unsigned c[E / 4];
                    if (a.e4m3)
                        k[j].template encode<AMPQ_FMT_E4M3>(byte, c);
                    else
                        k[j].template encode<AMPQ_FMT_E5M2>(byte, c);
                    store_codes(a.codes + row * a.ld_codes + c0, c);
                    if (t % K::kLanes == 0) a.scales[row * a.ld_scales + c0 / kGroup] = (unsigned char)byte;
                }
            }
            T* y = static_cast<T*>(a.y) + row * a.ld_y;
            const bool straight = (reinterpret_cast<uintptr_t>(y) & 15) == 0;
            if (straight && n[j] <= 0) continue;
#pragma unroll
            for (int i = 0; i < E / 2; ++i) k[j].v[i] = __fmul2_rn(LAYER ? __fadd2_rn(k[j].v[i], minus) : k[j].v[i], make_float2(rstd, rstd));
            K p;
            if (a.w) {
                load_params(a.w, a.param_bf16, c0, max(n[j], 0), p);
#pragma unroll
                for (int i = 0; i < E / 2; ++i) k[j].v[i] = __fmul2_rn(k[j].v[i], p.v[i]);
            }
            if (LAYER && a.b) {
                load_params(a.b, a.param_bf16, c0, max(n[j], 0), p);
#pragma unroll
                for (int i = 0; i < E / 2; ++i) k[j].v[i] = __fadd2_rn(k[j].v[i], p.v[i]);
            }
            if (straight) {
                k[j].store(y + c0, n[j]);
            } else {
                const int at = c0 - (int)lane * E;
                if (live && at < a.cols)
                    store_piece(y + at, min(32 * E, a.cols - at), k[j], (unsigned)__cvta_generic_to_shared(s_scratch[warp]), lane);
            }
        }
    }
}

struct BackwardArgs {
    const void *gy, *x, *w;
    const unsigned char *codes, *scales;
    const float *mean, *rstd;
    void* gx;
    float* part;  // [2][CTAs][part_pitch]: sums of gy*h, then of gy
    long long part_pitch;
    long long rows, ld_gy, ld_x, ld_codes, ld_scales, ld_gx;
    int cols;
    bool param_bf16, sum_b;
    bool e4m3;               // the checkpoint's format
    bool aligned_gy, aligned_x;  // rows start on 16-byte boundaries
    bool whole;                  // rows can be copied whole
};

__device__ __forceinline__ void copy16(unsigned dst, const void* src, int bytes) {  // the first `bytes` of 16, zeros behind them
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy4(unsigned dst, const void* src) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}

// A warp's chunks of one row on their way: 1024 bytes, and a word for rows that
// start between two words, kept 16-byte aligned.
constexpr int kPiece = 1024 + 16;

// The columns of one warp (32 chunks from element `at` on, of `cols`) of row `row`,
// copied to shared memory.  16 bytes a lane where rows start on 16-byte boundaries,
// zeros behind the row's end.  Otherwise words from the one the piece starts in;
// what lies behind the row's end in the matrix is copied too, a word that the
// matrix holds only half of is put together by hand.
template <typename T>
__device__ __forceinline__ void copy_piece(unsigned to, const T* m, long long ld, long long rows, int cols, long long row, int at, bool aligned, unsigned lane) {
    const T* p = m + row * ld + at;
    if (aligned) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            constexpr int kPer = 16 / (int)sizeof(T);
            const int first = (32 * k + (int)lane) * kPer, bytes = min(16, (cols - at - first) * (int)sizeof(T));
            if (bytes > 0) copy16(to + 16 * (32 * k + lane), p + first, bytes);
        }
        return;
    }
    const uintptr_t a0 = reinterpret_cast<uintptr_t>(p), down = a0 & ~(uintptr_t)3;
    const int bytes = min(1024, (cols - at) * (int)sizeof(T));
    const int words = bytes > 0 ? ((int)(a0 - down) + bytes + 3) / 4 : 0;
    const uintptr_t begin = reinterpret_cast<uintptr_t>(m), end = reinterpret_cast<uintptr_t>(m + (rows - 1) * ld + cols);
    if (down >= begin && down + 4 * words <= end) {  // nearly all pieces
        const unsigned char* q = reinterpret_cast<const unsigned char*>(down) + 4 * lane;
#pragma unroll
        for (int k = 0; k < 9; ++k)
            if (32 * k + (int)lane < words) copy4(to + 4 * (32 * k + lane), q + 128 * k);
        return;
    }
#pragma unroll 1
    for (int k = 0; k < 9; ++k) {
        const int w = 32 * k + (int)lane;
        if (w >= words) break;
        const uintptr_t q = down + 4 * w;
        if (q >= begin && q + 4 <= end) {
            copy4(to + 4 * w, reinterpret_cast<const void*>(q));
        } else {
            const bool lower = q >= begin;  // the half that exists
            const unsigned half = __ldg(reinterpret_cast<const unsigned short*>(lower ? q : q + 2));
            asm volatile("st.shared.u32 [%0], %1;" ::"r"(to + 4 * w), "r"(lower ? half : half << 16) : "memory");
        }
    }
}

// The scale bytes of a warp's chunk of one row (groups g0 to g0 + count - 1 of
// `groups`), copied to shared memory by words from the one the first byte is in;
// words that the matrix holds only parts of are put together by hand.
__device__ __forceinline__ void copy_scales(unsigned to, const unsigned char* scales, long long ld, long long rows, int groups, long long row, int g0, int count,
                                            unsigned lane) {
    const uintptr_t p = reinterpret_cast<uintptr_t>(scales + row * ld + g0), down = p & ~(uintptr_t)3;
    const int n = min(count, groups - g0);
    const int words = n > 0 ? ((int)(p - down) + n + 3) / 4 : 0;
    if ((int)lane >= words) return;
    const uintptr_t begin = reinterpret_cast<uintptr_t>(scales), end = reinterpret_cast<uintptr_t>(scales + (rows - 1) * ld + groups);
    const uintptr_t q = down + 4 * lane;
    if (q >= begin && q + 4 <= end) {
        copy4(to + 4 * lane, reinterpret_cast<const void*>(q));
    } else {
        unsigned w = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (q + i >= begin && q + i < end) w |= (unsigned)__ldg(reinterpret_cast<const unsigned char*>(q + i)) << (8 * i);
        asm volatile("st.shared.u32 [%0], %1;" ::"r"(to + 4 * lane), "r"(w) : "memory");
    }
}

// This lane's chunk of a piece, zeros from element n on.  All lanes call it.
template <typename T>
__device__ __forceinline__ void take_chunk(unsigned from, const T* m, long long ld, long long row, int at, bool aligned, unsigned lane, int n, unsigned (&w)[8]) {
    take_words(from + 32 * lane, lane, w);
    if (aligned) {
        if (n * (int)sizeof(T) <= 16) w[4] = w[5] = w[6] = w[7] = 0;
        return;
    }
    if (reinterpret_cast<uintptr_t>(m + row * ld + at) & 2) {
        unsigned next = __shfl_down_sync(0xFFFFFFFFu, w[0], 1);
        if (lane == 31) asm volatile("ld.shared.u32 %0, [%1];" : "=r"(next) : "r"(from + 1024) : "memory");
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = __funnelshift_r(w[i], i < 7 ? w[i + 1] : next, 16);
    }
    if (__any_sync(0xFFFFFFFFu, n < Chunk<T>::kElems)) {  // a row's last warp
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (sizeof(T) == 4) {
                if (i >= n) w[i] = 0;
            } else {
                if (2 * i >= n) w[i] = 0;
                if (2 * i + 1 == n) w[i] &= 0xFFFFu;
            }
        }
    }
}

// Per warp: a row's mean and rstd, and the scale bytes of each chunk (at most five words).
template <typename T, int WIDE>
constexpr int kSmallPiece = 16 + 32 * kChunks<T, WIDE>;

// Shared memory of a CTA per row on its way: gy, x or its codes, the row's small
// values, and the scale bytes of rows that come whole.
template <typename T, bool KEPT, int WPR, int WIDE>
constexpr int kRowBytes = Shape<WPR, WIDE>::kWarps * (kChunks<T, WIDE> * kPiece + (KEPT ? 512 * WIDE : kChunks<T, WIDE> * kPiece) + kSmallPiece<T, WIDE> + (KEPT ? 16 * WIDE : 0));

// Rows on their way, the current one among them: four, or as many as leave room
// for the CTAs meant to be resident; 0 where not even two fit (fp32 rows of more
// than 8192 columns, kept in full) and rows are read as they come.
template <typename T, bool KEPT, int WPR, int WIDE>
struct Ring {
    static constexpr int kFit = (WPR <= 10 ? 104 : 208) * 1024 / kRowBytes<T, KEPT, WPR, WIDE>;
    static constexpr int kRows = kFit >= 4 ? 4 : kFit >= 2 ? kFit : 0;
    static constexpr int kBytes = kRows * kRowBytes<T, KEPT, WPR, WIDE>;
};

// Rows are dealt to the row groups of a persistent grid; a thread keeps the fp32
// sums of gy*h and gy of its columns in registers over all its rows.  Each warp
// copies its own parts of the next rows to shared memory while it works on one (no
// barrier: no other warp reads them), which keeps enough bytes on the way with the
// few threads that the sums' registers allow.  The groups of a CTA are joined in
// shared memory, the CTAs by join_columns_kernel, in a fixed order.
//
// Bound by the row's latency: sixteen warps go through one row in step with a barrier,
// and no other row fills the gap (issue slots and DRAM both half busy, a quarter of
// the warps).  RMS norm of 8192 x 8192 from 8 bits 76 us (4.4 TB/s), layer norm from
// bf16 87 us (4.6 TB/s).
// Holding a row back until the next row's sums are under way (103 us against 102 at
// that point) and two CTAs of half the warps (145 us) cost more in registers and
// repeated work than the barrier.  Rows off the 16-byte boundaries are copied and
// put together by words, and stored through shared memory: 2047 x 4099 bf16 33 us
// (47 us with each lane's words stored in place).
template <typename T, bool KEPT, bool LAYER, int WPR, int WIDE>
__global__ void __launch_bounds__(Shape<WPR, WIDE>::kThreads, Shape<WPR, WIDE>::kThreads <= 320 ? 2 : 1) norm_backward_kernel(const BackwardArgs a) {
    using S = Shape<WPR, WIDE>;
    using K = Chunk<T>;
    constexpr int V = kChunks<T, WIDE>, E = K::kElems, kThreads = S::kThreads, kSpan = 512 * WPR * WIDE;
    constexpr bool kTwice = kThreads > 256 && kThreads != 512;  // too few registers to hold (x - mean) * rstd for a row's output
    static_assert(!KEPT || Ring<T, KEPT, WPR, WIDE>::kRows > 0, "codes are read from the ring");
    constexpr int kAhead = Ring<T, KEPT, WPR, WIDE>::kRows;
    extern __shared__ __align__(16) unsigned char ring[];
    __shared__ float red[2][S::kWarps * 2];
    __shared__ alignas(8) unsigned long long s_bars[4 * S::kGroups];
    __shared__ int s_gave_up[S::kGroups];
    const int warp = threadIdx.x / 32;
    const int t = threadIdx.x % (32 * WPR);
    const int group = warp / WPR;
    const unsigned lane = threadIdx.x % 32;
    constexpr int kGyRow = S::kWarps * V * kPiece;  // bytes of a row's gy, in pieces by warp and chunk
    const unsigned ring_gy = (unsigned)__cvta_generic_to_shared(ring) + warp * V * kPiece;
    const unsigned ring_x = ring_gy + kAhead * kGyRow;
    const unsigned ring_codes = (unsigned)__cvta_generic_to_shared(ring) + kAhead * kGyRow + threadIdx.x * 16;
    constexpr int kSmall = kSmallPiece<T, WIDE>;
    const unsigned ring_small = (unsigned)__cvta_generic_to_shared(ring) + kAhead * (kRowBytes<T, KEPT, WPR, WIDE> - S::kWarps * (kSmall + (KEPT ? 16 * WIDE : 0))) + warp * kSmall;
    const int groups = (a.cols + kGroup - 1) / kGroup;
    float2 sum_w[V][E / 2], sum_b[V][E / 2];
#pragma unroll
    for (int j = 0; j < V; ++j)
#pragma unroll
        for (int i = 0; i < E / 2; ++i) sum_w[j][i] = sum_b[j][i] = make_float2(0.0f, 0.0f);
    const float inv_cols = 1.0f / (float)a.cols;
    const long long stride = (long long)gridDim.x * S::kGroups;
    // Rows on 16-byte boundaries come whole, by bulk copies that one thread of the
    // group starts (of the kernel's instructions, a fifth were copies by 16 bytes a
    // lane); they lie as in memory.
    const bool whole = kAhead > 0 && a.whole;
    const unsigned base = (unsigned)__cvta_generic_to_shared(ring);
    const unsigned row_gy = base + group * (WPR * V * 1024), row_x = row_gy + kAhead * kGyRow;
    const unsigned row_codes = base + kAhead * kGyRow + group * (WPR * 512 * WIDE);
    const unsigned row_scales = base + kAhead * (kRowBytes<T, KEPT, WPR, WIDE> - S::kWarps * 16 * WIDE) + group * (WPR * 16 * WIDE);
    const unsigned bars = (unsigned)__cvta_generic_to_shared(s_bars) + 8 * group;
    volatile int* gave_up = s_gave_up + group;
    bool late = false;  // this thread missed a row
    auto copy_whole = [&](long long row, int slot) {
        if (row < a.rows) {
            if (t == 0 && !late) {
                const unsigned bar = bars + 8 * S::kGroups * slot, bytes = (unsigned)a.cols * (unsigned)sizeof(T);
                row_expect(bar, KEPT ? bytes + (unsigned)groups * (kGroup + 1) : 2 * bytes);
                row_copy(row_gy + slot * kGyRow, static_cast<const T*>(a.gy) + row * a.ld_gy, bytes, bar);
                if (KEPT) {
                    row_copy(row_codes + slot * (kThreads * 16 * WIDE), a.codes + row * a.ld_codes, groups * kGroup, bar);
                    row_copy(row_scales + slot * (S::kWarps * 16 * WIDE), a.scales + row * a.ld_scales, groups, bar);
                } else {
                    row_copy(row_x + slot * kGyRow, static_cast<const T*>(a.x) + row * a.ld_x, bytes, bar);
                }
            }
            if (lane < 2 && (lane || LAYER)) copy4(ring_small + (unsigned)(slot * S::kWarps * kSmall) + 4 * lane, (lane ? a.rstd : a.mean) + row);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    auto copy_any = [&](long long row, int slot) {
        if (row < a.rows) {
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const int at = (j * 32 * WPR + t - (int)lane) * E, c0 = at + (int)lane * E;
                const unsigned piece = (unsigned)(slot * kGyRow + j * kPiece);
                copy_piece(ring_gy + piece, static_cast<const T*>(a.gy), a.ld_gy, a.rows, a.cols, row, at, a.aligned_gy, lane);
                if (!KEPT) copy_piece(ring_x + piece, static_cast<const T*>(a.x), a.ld_x, a.rows, a.cols, row, at, a.aligned_x, lane);
                if (KEPT) copy_scales(ring_small + (unsigned)(slot * S::kWarps * kSmall + 16 + 32 * j), a.scales, a.ld_scales, a.rows, groups, row, at / kGroup, E, lane);
                if (KEPT && c0 < a.cols) {
                    const unsigned char* p = a.codes + row * a.ld_codes + c0;
                    if (E == 16)
                        copy16(ring_codes + (unsigned)((slot * WIDE + j) * kThreads * 16), p, 16);
                    else
                        asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(ring_codes + (unsigned)((slot * WIDE + j / 2) * kThreads * 16) + 8 * (j & 1)), "l"(p) : "memory");
                }
            }
        }
        if (row < a.rows && lane < 2) {
            const float* p = lane ? a.rstd : a.mean;
            if (lane || LAYER) copy4(ring_small + (unsigned)(slot * S::kWarps * kSmall) + 4 * lane, p + row);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    const long long first = (long long)blockIdx.x * S::kGroups + group;
    if (whole) {
        if (t == 0) {
            for (int s = 0; s < kAhead; ++s) asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(bars + 8 * S::kGroups * s) : "memory");
            *gave_up = 0;
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        }
        __syncthreads();
#pragma unroll
        for (int s = 0; s < kAhead; ++s) copy_whole(first + s * stride, s);
    } else {
#pragma unroll
        for (int s = 0; s < kAhead - 1; ++s) copy_any(first + s * stride, s);
    }
    unsigned lap = 0;  // parity of the ring's turn
    int slot = 0;
    int phase = 0;
    K weight[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
        const int c0 = (j * 32 * WPR + t) * E;
        if (a.w && c0 < a.cols)
            load_params(a.w, a.param_bf16, c0, min(E, a.cols - c0), weight[j]);
        else
#pragma unroll
            for (int i = 0; i < E / 2; ++i) weight[j].v[i] = make_float2(1.0f, 1.0f);
    }
    for (long long row0 = (long long)blockIdx.x * S::kGroups; row0 < a.rows; row0 += stride) {
        const long long row = row0 + group;
        const bool live = row < a.rows;
        __syncwarp();  // the piece that is copied over has been read by all lanes
        if (kAhead > 0 && !whole) copy_any(row + (kAhead - 1) * stride, slot == 0 ? kAhead - 1 : slot - 1);
        asm volatile("cp.async.wait_group %0;" ::"n"(kAhead > 0 ? kAhead - 1 : 0) : "memory");
        __syncwarp();
        if (whole && live && !late && !row_wait(bars + 8 * S::kGroups * slot, lap, gave_up)) {
            late = true;
            for (int s = 0; t == 0 && s < kAhead && row + s * stride < a.rows; ++s) {  // the copies of this row and the next ones
                const bool wraps = slot + s >= kAhead;
                if (!row_drain(bars + 8 * S::kGroups * (slot + s - (wraps ? kAhead : 0)), wraps ? lap ^ 1 : lap)) break;
            }
        }
        float mean = 0.0f, rstd = 0.0f, p[V];
        if (live) {
            if (kAhead > 0) {
                const unsigned small = ring_small + (unsigned)(slot * S::kWarps * kSmall);
                asm volatile("ld.shared.f32 %0, [%1];" : "=f"(rstd) : "r"(small + 4) : "memory");
                if (LAYER) asm volatile("ld.shared.f32 %0, [%1];" : "=f"(mean) : "r"(small) : "memory");
                if (KEPT) {
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        unsigned at;
                        if (whole)
                            at = row_scales + (unsigned)(slot * (S::kWarps * 16 * WIDE) + (j * 32 * WPR + t) * E / kGroup);
                        else
                            at = small + 16 + 32 * j + (unsigned)(reinterpret_cast<uintptr_t>(a.scales + row * a.ld_scales + (j * 32 * WPR + t - (int)lane) * E / kGroup) & 3) + lane / K::kLanes;
                        unsigned byte;
                        asm volatile("ld.shared.u8 %0, [%1];" : "=r"(byte) : "r"(at) : "memory");
                        p[j] = scale_of(byte);
                    }
                }
            } else {
                rstd = __ldg(a.rstd + row);
                if (LAYER) mean = __ldg(a.mean + row);
            }
            if (late) rstd = __uint_as_float(kNanBits);
        }
        K g[V], h[kTwice ? 1 : V];                 // gy * weight; (x - mean) * rstd, or
        unsigned xr[V][KEPT ? E / 4 : 8];          // the codes or words of x to form it again
        // the scale of a kept x joins the subtraction
        auto normalized = [&](int j) {
            K k;
            if constexpr (KEPT) {
                if (a.e4m3)
                    k.template decode<AMPQ_FMT_E4M3>(xr[j]);
                else
                    k.template decode<AMPQ_FMT_E5M2>(xr[j]);
            } else {
                k.from_words(xr[j]);
            }
#pragma unroll
            for (int i = 0; i < E / 2; ++i) {
                float2 d = k.v[i];
                if (KEPT && LAYER) d = __ffma2_rn(d, make_float2(p[j], p[j]), make_float2(-mean, -mean));
                if (KEPT && !LAYER) d = __fmul2_rn(d, make_float2(p[j], p[j]));
                if (!KEPT && LAYER) d = __fadd2_rn(d, make_float2(-mean, -mean));
                k.v[i] = __fmul2_rn(d, make_float2(rstd, rstd));
            }
            return k;
        };
        float2 c2 = make_float2(0.0f, 0.0f), c1 = make_float2(0.0f, 0.0f);
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const int c0 = (j * 32 * WPR + t) * E;
            const int n = live ? min(E, a.cols - c0) : 0;
            unsigned w8[8];
            if (whole) {
                const unsigned at = (unsigned)(slot * kGyRow + (j * 32 * WPR + t) * 32);
                take_words(row_gy + at, lane, w8);
                if constexpr (!KEPT) take_words(row_x + at, lane, xr[j]);
            } else if constexpr (kAhead > 0) {
                const unsigned piece = (unsigned)(slot * kGyRow + j * kPiece);
                take_chunk(ring_gy + piece, static_cast<const T*>(a.gy), a.ld_gy, row, c0, a.aligned_gy, lane, n, w8);
                if constexpr (!KEPT) take_chunk(ring_x + piece, static_cast<const T*>(a.x), a.ld_x, row, c0, a.aligned_x, lane, n, xr[j]);
            } else if (n > 0) {
                K::load_words(static_cast<const T*>(a.gy) + row * a.ld_gy + c0, n, w8);
                if constexpr (!KEPT) K::load_words(static_cast<const T*>(a.x) + row * a.ld_x + c0, n, xr[j]);
            }
            if (n <= 0) continue;
            if constexpr (KEPT) {
                const unsigned at = whole ? row_codes + (unsigned)(slot * (kThreads * 16 * WIDE) + (j * 32 * WPR + t) * E)
                                          : ring_codes + (unsigned)((slot * WIDE + j * E / 16) * kThreads * 16 + j * E % 16);
                if (E == 16) {
                    const uint4 q = take16(at);
                    xr[j][0] = q.x; xr[j][1] = q.y; xr[j][2 % (E / 4)] = q.z; xr[j][3 % (E / 4)] = q.w;
                } else {
                    asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(xr[j][0]), "=r"(xr[j][1]) : "r"(at) : "memory");
                }
            }
            g[j].from_words(w8);
            const K k = normalized(j);  // behind the last column gy is 0, and this finite unless the row's sums are not
            if constexpr (!kTwice) h[j] = k;
#pragma unroll
            for (int i = 0; i < E / 2; ++i) {
                sum_w[j][i] = __ffma2_rn(g[j].v[i], k.v[i], sum_w[j][i]);
                if (LAYER) sum_b[j][i] = __fadd2_rn(sum_b[j][i], g[j].v[i]);
            }
#pragma unroll
            for (int i = 0; i < E / 2; ++i) g[j].v[i] = __fmul2_rn(g[j].v[i], weight[j].v[i]);
#pragma unroll
            for (int i = 0; i < E / 2; ++i) {
                c2 = __ffma2_rn(g[j].v[i], k.v[i], c2);
                if (LAYER) c1 = __fadd2_rn(c1, g[j].v[i]);
            }
        }
        float both[2] = {late ? __uint_as_float(kNanBits) : c2.x + c2.y, c1.x + c1.y};
        if (LAYER) {
            row_sum<WPR, 2>(both, red[phase], warp);
        } else {
            float one[1] = {both[0]};
            row_sum<WPR, 1>(one, red[phase], warp);
            both[0] = one[0];
        }
        phase ^= 1;
        // every thread of the group has read its part of the row: its place takes another one
        if (WPR == 1) __syncwarp();
        if (whole) copy_whole(row + kAhead * stride, slot);
        const float m2 = -both[0] * inv_cols, m1 = LAYER ? -both[1] * inv_cols : 0.0f;
        T* gx = static_cast<T*>(a.gx) + row * a.ld_gx;
        // the row's pieces of gy have been read: their place is free for gx on its way out
        const bool pieces = kAhead > 0 && !whole && (reinterpret_cast<uintptr_t>(gx) & 15) != 0;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const int c0 = (j * 32 * WPR + t) * E;
            const int n = live ? min(E, a.cols - c0) : 0;
            if (!pieces && n <= 0) continue;
            K k;
            if constexpr (kTwice)
                k = normalized(j);
            else
                k = h[j];
#pragma unroll
            for (int i = 0; i < E / 2; ++i) {
                float2 o = __ffma2_rn(k.v[i], make_float2(m2, m2), g[j].v[i]);
                if (LAYER) o = __fadd2_rn(o, make_float2(m1, m1));
                g[j].v[i] = __fmul2_rn(o, make_float2(rstd, rstd));
            }
            if (pieces) {
                const int at = c0 - (int)lane * E;
                if (live && at < a.cols) store_piece(gx + at, min(32 * E, a.cols - at), g[j], ring_gy + (unsigned)(slot * kGyRow + j * kPiece), lane);
            } else {
                g[j].store(gx + c0, n);
            }
        }
        if (++slot == kAhead) {
            slot = 0;
            lap ^= 1;
        }
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    if (!a.part) return;
    if (LAYER && late)  // sum_w is NaN already
#pragma unroll
        for (int j = 0; j < V; ++j)
#pragma unroll
            for (int i = 0; i < E / 2; ++i) sum_b[j][i] = make_float2(__uint_as_float(kNanBits), __uint_as_float(kNanBits));
    float* join = reinterpret_cast<float*>(ring);
    for (int k = 0; k < (LAYER && a.sum_b ? 2 : 1); ++k) {
        float* out = a.part + ((long long)k * gridDim.x + blockIdx.x) * a.part_pitch;
        if (S::kGroups == 1) {
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const int c0 = (j * 32 * WPR + t) * E;
                if (c0 >= a.cols) continue;  // whole chunks fit into the pitch
#pragma unroll
                for (int i = 0; i < E / 2; i += 2) {
                    const float2 f = k ? sum_b[j][i] : sum_w[j][i], h = k ? sum_b[j][i + 1] : sum_w[j][i + 1];
                    *reinterpret_cast<float4*>(out + c0 + 2 * i) = make_float4(f.x, f.y, h.x, h.y);
                }
            }
        } else {
            __syncthreads();
#pragma unroll
            for (int j = 0; j < V; ++j)
#pragma unroll
                for (int i = 0; i < E / 2; ++i)
                    *reinterpret_cast<float2*>(join + group * kSpan + (j * 32 * WPR + t) * E + 2 * i) = k ? sum_b[j][i] : sum_w[j][i];
            __syncthreads();
            for (int i = threadIdx.x; i < a.cols; i += kThreads) {
                float s = 0.0f;
#pragma unroll
                for (int g = 0; g < S::kGroups; ++g) s += join[g * kSpan + i];
                out[i] = s;
            }
        }
    }
}

// Warps of a row, a power of two: 512 columns each, 1024 above 4096 columns.
int warps_per_row(int cols) { return cols <= 512 ? 1 : cols <= 1024 ? 2 : cols <= 2048 ? 4 : cols <= 8192 ? 8 : 16; }
// of the backward pass: 512 columns each, and ten warps up to 5120
int backward_warps(int cols) { return cols <= 512 ? 1 : cols <= 1024 ? 2 : cols <= 2048 ? 4 : cols <= 4096 ? 8 : cols <= 5120 ? 10 : cols <= 8192 ? 16 : 32; }

// Columns of a partial row: whole chunks.
long long part_pitch(long long cols) { return (cols + 15) / 16 * 16; }

// CTAs of the backward pass: every row group gets a row before one gets two, and
// no more CTAs than are resident, so that the sums stay in registers.
int backward_ctas(long long rows, int cols, int sms) {
    const int wpr = backward_warps(cols), groups = wpr < 8 ? 8 / wpr : 1;
    const long long need = (rows + groups - 1) / groups;
    const long long most = (long long)sms * (wpr <= 10 ? 2 : 1);
    return (int)(need < most ? need : most);
}

constexpr int kMaxDevices = 64;

// Lets a kernel use `bytes` of dynamic shared memory, once per device.
template <class Kernel>
bool allow_smem(Kernel kernel, int bytes, std::atomic<bool>* prepared, int device) {
    if (device < kMaxDevices && prepared[device].load(std::memory_order_acquire)) return true;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess) {
        cudaGetLastError();
        return false;
    }
    if (device < kMaxDevices) prepared[device].store(true, std::memory_order_release);
    return true;
}

template <typename T, bool KEPT, bool LAYER, int WPR, int WIDE>
int start_forward(ForwardArgs a, int device, int sms, cudaStream_t st) {
    using S = Shape<WPR, WIDE>;
    using Ring = ForwardRing<T, WPR, WIDE>;
    static std::atomic<bool> prepared[kMaxDevices];
    const long long need = (a.rows + S::kGroups - 1) / S::kGroups, most = (long long)sms * Ring::kCtas;
    a.bulk = a.bulk && need > most;  // fewer rows are all read at once
    if (a.bulk && !allow_smem(norm_forward_kernel<T, KEPT, LAYER, WPR, WIDE>, Ring::kBytes, prepared, device)) return AMPQ_ERR_CUDA;
    norm_forward_kernel<T, KEPT, LAYER, WPR, WIDE><<<(unsigned)(a.bulk ? most : need), S::kThreads, a.bulk ? Ring::kBytes : 0, st>>>(a);
    return launched();
}

template <typename T, bool KEPT, bool LAYER>
int launch_forward(const ForwardArgs& a, int device, int sms, cudaStream_t st) {
    if (a.cols > 4096) return a.cols <= 8192 ? start_forward<T, KEPT, LAYER, 8, 2>(a, device, sms, st) : start_forward<T, KEPT, LAYER, 16, 2>(a, device, sms, st);
    switch (warps_per_row(a.cols)) {
        case 1: return start_forward<T, KEPT, LAYER, 1, 1>(a, device, sms, st);
        case 2: return start_forward<T, KEPT, LAYER, 2, 1>(a, device, sms, st);
        case 4: return start_forward<T, KEPT, LAYER, 4, 1>(a, device, sms, st);
        default: return start_forward<T, KEPT, LAYER, 8, 1>(a, device, sms, st);
    }
}

template <typename T, bool KEPT, bool LAYER, int WPR, int WIDE>
int start_backward(const BackwardArgs& a, int device, int ctas, cudaStream_t st) {
    static std::atomic<bool> prepared[kMaxDevices];  // the kernel may use its shared memory on that device
    using S = Shape<WPR, WIDE>;
    constexpr int kJoin = S::kGroups > 1 ? S::kGroups * 512 * WPR * WIDE * 4 : 0;
    constexpr int kBytes = Ring<T, KEPT, WPR, WIDE>::kBytes > kJoin ? Ring<T, KEPT, WPR, WIDE>::kBytes : kJoin;
    if (!allow_smem(norm_backward_kernel<T, KEPT, LAYER, WPR, WIDE>, kBytes, prepared, device)) return AMPQ_ERR_CUDA;
    norm_backward_kernel<T, KEPT, LAYER, WPR, WIDE><<<(unsigned)ctas, S::kThreads, kBytes, st>>>(a);
    return launched();
}

template <typename T, bool KEPT, bool LAYER>
int launch_backward(const BackwardArgs& a, int device, int ctas, cudaStream_t st) {
    switch (backward_warps(a.cols)) {
        case 1: return start_backward<T, KEPT, LAYER, 1, 1>(a, device, ctas, st);
        case 2: return start_backward<T, KEPT, LAYER, 2, 1>(a, device, ctas, st);
        case 4: return start_backward<T, KEPT, LAYER, 4, 1>(a, device, ctas, st);
        case 8: return start_backward<T, KEPT, LAYER, 8, 1>(a, device, ctas, st);
        case 10: return start_backward<T, KEPT, LAYER, 10, 1>(a, device, ctas, st);
        case 16: return start_backward<T, KEPT, LAYER, 16, 1>(a, device, ctas, st);
        default: return start_backward<T, KEPT, LAYER, 32, 1>(a, device, ctas, st);
    }
}

template <typename T>
int dispatch_forward(bool kept, bool layer, const ForwardArgs& a, int device, int sms, cudaStream_t st) {
    if (kept) return layer ? launch_forward<T, true, true>(a, device, sms, st) : launch_forward<T, true, false>(a, device, sms, st);
    return layer ? launch_forward<T, false, true>(a, device, sms, st) : launch_forward<T, false, false>(a, device, sms, st);
}

template <typename T>
int dispatch_backward(bool kept, bool layer, const BackwardArgs& a, int device, int ctas, cudaStream_t st) {
    if (kept) return layer ? launch_backward<T, true, true>(a, device, ctas, st) : launch_backward<T, true, false>(a, device, ctas, st);
    return layer ? launch_backward<T, false, true>(a, device, ctas, st) : launch_backward<T, false, false>(a, device, ctas, st);
}

int check_norm(int kind, int dtype, int param_dtype, int fmt, long long cols) {
    if (kind != AMPQ_NORM_LAYER && kind != AMPQ_NORM_RMS) return AMPQ_ERR_INVALID;
    if (!known_dtype(dtype) || !known_dtype(param_dtype)) return AMPQ_ERR_INVALID;
    if (fmt != AMPQ_FMT_BASE && !known_fp8(fmt)) return AMPQ_ERR_INVALID;
    if (cols > kMaxNormCols) return AMPQ_ERR_TOO_LARGE;
    return AMPQ_OK;
}

}  // namespace
}  // namespace ampq

using namespace ampq;

extern "C" {
#pragma GCC visibility push(default)

int ampq_norm_forward(int device, void* cuda_stream, int kind, int dtype, int param_dtype, int fmt, const void* x, long long ld_x,
                      long long rows, long long cols, const void* weight, const void* bias, float eps, void* y, long long ld_y,
                      float* mean, float* rstd, unsigned char* codes, long long ld_codes, unsigned char* scales, long long ld_scales) {
    int rc = check_norm(kind, dtype, param_dtype, fmt, cols);
    if (!rc) rc = check_matrix(x, rows, cols, ld_x, dtype);
    if (!rc) rc = check_matrix(y, rows, cols, ld_y, dtype);
    if (!rc && fmt != AMPQ_FMT_BASE) rc = check_ckpt(codes, ld_codes, scales, ld_scales, rows, cols);
    if (rc) return rc;
    if (!(eps >= 0.0f) || std::isinf(eps)) return AMPQ_ERR_INVALID;
    const bool layer = kind == AMPQ_NORM_LAYER;
    if (rows > 0 && cols > 0 && (!rstd || (layer && !mean))) return AMPQ_ERR_INVALID;
    if (!layer && bias) return AMPQ_ERR_INVALID;
    if (!aligned_to(weight, elem_bytes(param_dtype)) || !aligned_to(bias, elem_bytes(param_dtype)) || !aligned_to(mean, 4) || !aligned_to(rstd, 4))
        return AMPQ_ERR_ALIGN;
    CkptDevice cur(device);
    if (cur.status) return cur.status;
    if (rows == 0) return AMPQ_OK;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
    if (cols == 0) {  // the mean of nothing: NaN, all bits set
        for (float* p : {layer ? mean : nullptr, rstd})
            if (p && cudaMemsetAsync(p, 0xFF, (size_t)rows * sizeof(float), st) != cudaSuccess) {
                cudaGetLastError();
                return AMPQ_ERR_CUDA;
            }
        return AMPQ_OK;
    }
    const int sms = sm_count(device);
    if (sms < 1) return AMPQ_ERR_CUDA;
    ForwardArgs a;
    a.x = x; a.w = weight; a.b = bias; a.y = y;
    a.mean = mean; a.rstd = rstd;
    a.codes = codes; a.scales = scales;
    a.rows = rows; a.ld_x = ld_x; a.ld_y = ld_y; a.ld_codes = ld_codes; a.ld_scales = ld_scales;
    a.cols = (int)cols;
    a.eps = eps;
    a.e4m3 = fmt == AMPQ_FMT_E4M3;
    a.whole = cols % (dtype == AMPQ_F32 ? 8 : 16) == 0;
    a.bulk = rows_aligned(x, ld_x, dtype) && a.whole;
    a.param_bf16 = param_dtype == AMPQ_BF16;
    const bool kept = fmt != AMPQ_FMT_BASE;
    return dtype == AMPQ_F32 ? dispatch_forward<float>(kept, layer, a, device, sms, st) : dispatch_forward<__nv_bfloat16>(kept, layer, a, device, sms, st);
}

int ampq_norm_backward_workspace(int device, long long rows, long long cols, long long* bytes) {
    if (!bytes || rows < 0 || cols < 0) return AMPQ_ERR_INVALID;
    if (cols > kMaxNormCols || rows > kMaxRows) return AMPQ_ERR_TOO_LARGE;
    CkptDevice cur(device);
    if (cur.status) return cur.status;
    const int sms = sm_count(device);
    if (sms < 1) return AMPQ_ERR_CUDA;
    *bytes = 2LL * backward_ctas(rows, (int)cols, sms) * part_pitch(cols) * (long long)sizeof(float);
    return AMPQ_OK;
}

int ampq_norm_backward(int device, void* cuda_stream, int kind, int dtype, int param_dtype, int fmt, const void* gy, long long ld_gy,
                       const void* x, long long ld_x, const unsigned char* codes, long long ld_codes, const unsigned char* scales,
                       long long ld_scales, long long rows, long long cols, const float* mean, const float* rstd, const void* weight,
                       void* gx, long long ld_gx, void* gweight, void* gbias, void* workspace, long long workspace_bytes) {
    int rc = check_norm(kind, dtype, param_dtype, fmt, cols);
    if (!rc) rc = check_matrix(gy, rows, cols, ld_gy, dtype);
    if (!rc) rc = check_matrix(gx, rows, cols, ld_gx, dtype);
    if (!rc) rc = fmt == AMPQ_FMT_BASE ? check_matrix(x, rows, cols, ld_x, dtype) : check_ckpt(codes, ld_codes, scales, ld_scales, rows, cols);
    if (rc) return rc;
    const bool layer = kind == AMPQ_NORM_LAYER;
    if (rows > 0 && cols > 0 && (!rstd || (layer && !mean))) return AMPQ_ERR_INVALID;
    if (gbias && (!layer || !gweight)) return AMPQ_ERR_INVALID;
    if (!aligned_to(weight, elem_bytes(param_dtype)) || !aligned_to(gweight, elem_bytes(param_dtype)) ||
        !aligned_to(gbias, elem_bytes(param_dtype)) || !aligned_to(mean, 4) || !aligned_to(rstd, 4) || !aligned_to(workspace, 16))
        return AMPQ_ERR_ALIGN;
    CkptDevice cur(device);
    if (cur.status) return cur.status;
    if (cols == 0) return AMPQ_OK;
    const int sms = sm_count(device);
    if (sms < 1) return AMPQ_ERR_CUDA;
    const int ctas = backward_ctas(rows, (int)cols, sms);
    const bool sums = gweight != nullptr;
    if (sums && ctas > 0 && (!workspace || workspace_bytes < 2LL * ctas * part_pitch(cols) * (long long)sizeof(float))) return AMPQ_ERR_INVALID;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
    if (rows > 0) {
        BackwardArgs a;
        a.gy = gy; a.x = x; a.w = weight;
        a.codes = codes; a.scales = scales;
        a.mean = mean; a.rstd = rstd;
        a.gx = gx;
        a.part = sums ? static_cast<float*>(workspace) : nullptr;
        a.part_pitch = part_pitch(cols);
        a.rows = rows; a.ld_gy = ld_gy; a.ld_x = ld_x; a.ld_codes = ld_codes; a.ld_scales = ld_scales; a.ld_gx = ld_gx;
        a.cols = (int)cols;
        a.param_bf16 = param_dtype == AMPQ_BF16;
        a.sum_b = gbias != nullptr;
        a.e4m3 = fmt == AMPQ_FMT_E4M3;
        a.aligned_gy = rows_aligned(gy, ld_gy, dtype);
        a.aligned_x = rows_aligned(x, ld_x, dtype);
        const long long groups = cols / kGroup;
        a.whole = a.aligned_gy && cols % (dtype == AMPQ_F32 ? 8 : 16) == 0 &&
                  (fmt == AMPQ_FMT_BASE ? a.aligned_x : cols % kGroup == 0 && groups % 16 == 0 && ld_scales % 16 == 0 && aligned_to(scales, 16));
        const bool kept = fmt != AMPQ_FMT_BASE;
        rc = dtype == AMPQ_F32 ? dispatch_backward<float>(kept, layer, a, device, ctas, st) : dispatch_backward<__nv_bfloat16>(kept, layer, a, device, ctas, st);
        if (rc) return rc;
    }
    if (!sums) return AMPQ_OK;
    return launch_join_columns(static_cast<const float*>(workspace), gbias ? 2 : 1, ctas, cols, part_pitch(cols), gweight, gbias, param_dtype, st);
}

#pragma GCC visibility pop
}  // extern "C"
