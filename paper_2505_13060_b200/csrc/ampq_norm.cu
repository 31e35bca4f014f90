// Layer norm and RMS norm, forward and backward (include/ampq.h:
// ampq_norm_forward, ampq_norm_backward), with the 8-bit checkpoint of the
// input written by the forward pass and read by the backward pass.
#include "ampq_ckpt.h"

#include <atomic>
#include <cmath>

namespace ampq {
namespace {

constexpr int kMaxNormCols = AMPQ_NORM_MAX_COLS;

// One thread holds 16 elements of a row: one chunk of bf16 or two of fp32.
template <typename T>
constexpr int kChunks = 16 / Chunk<T>::kElems;

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
    // 32 lanes take one warp's sum each and add them up as before
    const int first = warp / WPR * WPR, lane = threadIdx.x & 31;
#pragma unroll
    for (int k = 0; k < N; ++k) {
        float t = lane < WPR ? red[(first + lane) * N + k] : 0.0f;
#pragma unroll
        for (int o = WPR / 2; o > 0; o >>= 1) t += __shfl_xor_sync(0xFFFFFFFFu, t, o);
        s[k] = __shfl_sync(0xFFFFFFFFu, t, 0);
    }
}

template <int WPR>
struct Shape {
    static constexpr int kWarps = WPR < 8 ? 8 : WPR;   // warps of a CTA
    static constexpr int kGroups = kWarps / WPR;       // rows a CTA works on at a time
    static constexpr int kThreads = 32 * kWarps;
    static constexpr int kSpan = 512 * WPR;            // most columns of a row
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

struct ForwardArgs {
    const void *x, *w, *b;
    void* y;
    float *mean, *rstd;
    unsigned char *codes, *scales;
    long long rows, ld_x, ld_y, ld_codes, ld_scales;
    int cols;
    float eps;
    bool layer, param_bf16;
};

// One row per group of WPR warps, held in registers between the statistics (mean,
// then the sum of squared differences from it) and the output, so x is read once.
// Thread t of a group holds the chunks (j * threads + t): loads are contiguous
// and neighbouring lanes make the groups of the checkpoint.
template <typename T, int FMT, int WPR>
__global__ void __launch_bounds__(Shape<WPR>::kThreads, 2048 / Shape<WPR>::kThreads > 4 ? 4 : 1) norm_forward_kernel(const ForwardArgs a) {
    using S = Shape<WPR>;
    using K = Chunk<T>;
    constexpr int V = kChunks<T>, E = K::kElems;
    __shared__ float red[2][S::kWarps];
    const int warp = threadIdx.x / 32;
    const int t = threadIdx.x % (32 * WPR);
    const long long row = (long long)blockIdx.x * S::kGroups + warp / WPR;
    const bool live = row < a.rows;
    const T* x = static_cast<const T*>(a.x) + row * a.ld_x;
    K k[V];
    int n[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
        const int c0 = (j * 32 * WPR + t) * E;
        n[j] = live ? min(E, a.cols - c0) : 0;
        k[j].zero();
        if (n[j] > 0) k[j].load(x + c0, n[j]);
    }
    const float inv_cols = 1.0f / (float)a.cols;
    float mean = 0.0f;
    if (a.layer) {
        float2 s2 = make_float2(0.0f, 0.0f);
#pragma unroll
        for (int j = 0; j < V; ++j)
#pragma unroll
            for (int i = 0; i < E / 2; ++i) s2 = __fadd2_rn(s2, k[j].v[i]);
        float s[1] = {s2.x + s2.y};
        row_sum<WPR, 1>(s, red[0], warp);
        mean = s[0] * inv_cols;
    }
    const float2 minus = make_float2(-mean, -mean);
    float2 q2 = make_float2(0.0f, 0.0f);
#pragma unroll
    for (int j = 0; j < V; ++j) {
#pragma unroll
        for (int i = 0; i < E / 2; ++i) {
            float2 d = __fadd2_rn(k[j].v[i], minus);
            if (n[j] < E) d = make_float2(2 * i < n[j] ? d.x : 0.0f, 2 * i + 1 < n[j] ? d.y : 0.0f);
            q2 = __ffma2_rn(d, d, q2);
        }
    }
    float q[1] = {q2.x + q2.y};
    row_sum<WPR, 1>(q, red[1], warp);
    const float rstd = 1.0f / sqrtf(q[0] * inv_cols + a.eps);
    if (live && t == 0) {
        if (a.layer) a.mean[row] = mean;
        a.rstd[row] = rstd;
    }
#pragma unroll
    for (int j = 0; j < V; ++j) {
        const int c0 = (j * 32 * WPR + t) * E;
        if (FMT != AMPQ_FMT_BASE) {
            constexpr int F = FMT == AMPQ_FMT_BASE ? AMPQ_FMT_E4M3 : FMT;
            const unsigned byte = scale_byte<F>(k[j].group_amax());
            if (live && (c0 & ~(kGroup - 1)) < a.cols) {  // whole groups: the columns behind the last are stored as 0
                unsigned c[E / 4];
                k[j].template encode<F>(byte, c);
                store_codes(a.codes + row * a.ld_codes + c0, c);
                if (t % K::kLanes == 0) a.scales[row * a.ld_scales + c0 / kGroup] = (unsigned char)byte;
            }
        }
        if (n[j] <= 0) continue;
#pragma unroll
        for (int i = 0; i < E / 2; ++i) k[j].v[i] = __fmul2_rn(__fadd2_rn(k[j].v[i], minus), make_float2(rstd, rstd));
        K p;
        if (a.w) {
            load_params(a.w, a.param_bf16, c0, n[j], p);
#pragma unroll
            for (int i = 0; i < E / 2; ++i) k[j].v[i] = __fmul2_rn(k[j].v[i], p.v[i]);
        }
        if (a.b) {
            load_params(a.b, a.param_bf16, c0, n[j], p);
#pragma unroll
            for (int i = 0; i < E / 2; ++i) k[j].v[i] = __fadd2_rn(k[j].v[i], p.v[i]);
        }
        k[j].store(static_cast<T*>(a.y) + row * a.ld_y + c0, n[j]);
    }
}

struct BackwardArgs {
    const void *gy, *x, *w;
    const unsigned char *codes, *scales;
    const float *mean, *rstd;
    void* gx;
    float* part;  // [2][CTAs][cols]: sums of gy*h, then of gy
    long long rows, ld_gy, ld_x, ld_codes, ld_scales, ld_gx;
    int cols;
    bool param_bf16, sum_b;
    bool async_gy, async_x;  // rows start on 16-byte boundaries: copied to shared memory ahead of time
};

__device__ __forceinline__ void copy16(unsigned dst, const void* src, int bytes) {  // the first `bytes` of 16, zeros behind them
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ uint4 take16(unsigned src) {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(src) : "memory");
    return v;
}

// Shared memory of a CTA per row on its way: 32 bytes of gy and of x (or its
// codes, 16) for each chunk of each thread.
template <typename T, int FMT, int WPR>
constexpr int kRowBytes = Shape<WPR>::kThreads * (kChunks<T> * 32 + (FMT == AMPQ_FMT_BASE ? kChunks<T> * 32 : 16));

// Rows on their way, the current one among them: four, or as many as leave room
// for the CTAs meant to be resident; 0 where not even two fit (fp32 rows of more
// than 8192 columns, kept in full) and rows are read as they come.
template <typename T, int FMT, int WPR>
struct Ring {
    static constexpr int kFit = (WPR <= 8 ? 104 : 208) * 1024 / kRowBytes<T, FMT, WPR>;
    static constexpr int kRows = kFit >= 4 ? 4 : kFit >= 2 ? kFit : 0;
    static constexpr int kBytes = kRows * kRowBytes<T, FMT, WPR>;
};

// Rows are dealt to the row groups of a persistent grid; a thread keeps the fp32
// sums of gy*h and gy of its 16 columns in registers over all its rows.  Each
// thread copies its own parts of the next rows to shared memory while it works on
// one (no barrier: nobody else reads them), which keeps enough bytes on the way
// with the few threads that the sums' registers allow.  The groups of a CTA are
// joined in shared memory, the CTAs by join_columns_kernel, in a fixed order.
template <typename T, int FMT, bool LAYER, int WPR>
__global__ void __launch_bounds__(Shape<WPR>::kThreads) norm_backward_kernel(const BackwardArgs a) {
    using S = Shape<WPR>;
    using K = Chunk<T>;
    constexpr int V = kChunks<T>, E = K::kElems, kThreads = S::kThreads;
    constexpr bool kKept = FMT != AMPQ_FMT_BASE;
    static_assert(!kKept || Ring<T, FMT, WPR>::kRows > 0, "codes are read from the ring");
    constexpr int kAhead = Ring<T, FMT, WPR>::kRows;
    extern __shared__ __align__(16) unsigned char ring[];
    __shared__ float red[2][S::kWarps * 2];
    const int warp = threadIdx.x / 32;
    const int t = threadIdx.x % (32 * WPR);
    const int group = warp / WPR;
    const unsigned ring_gy = (unsigned)__cvta_generic_to_shared(ring) + threadIdx.x * 16;
    const unsigned ring_x = ring_gy + kAhead * kThreads * 32 * V;
    float2 sum_w[V][E / 2], sum_b[V][E / 2];
#pragma unroll
    for (int j = 0; j < V; ++j)
#pragma unroll
        for (int i = 0; i < E / 2; ++i) sum_w[j][i] = sum_b[j][i] = make_float2(0.0f, 0.0f);
    const float inv_cols = 1.0f / (float)a.cols;
    const long long stride = (long long)gridDim.x * S::kGroups;
    const bool async_gy = kAhead > 0 && a.async_gy, async_x = kAhead > 0 && a.async_x;
    auto begin_copy = [&](long long row, int slot) {
        if (row < a.rows) {
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const int c0 = (j * 32 * WPR + t) * E, n = min(E, a.cols - c0);
                if (n <= 0) continue;
                const int bytes = n * (int)sizeof(T);
                const unsigned to = (unsigned)((slot * V + j) * 2 * kThreads * 16);
                if (async_gy) {
                    const unsigned char* p = reinterpret_cast<const unsigned char*>(static_cast<const T*>(a.gy) + row * a.ld_gy + c0);
                    copy16(ring_gy + to, p, min(16, bytes));
                    if (bytes > 16) copy16(ring_gy + to + kThreads * 16, p + 16, bytes - 16);
                }
                if (!kKept && async_x) {
                    const unsigned char* p = reinterpret_cast<const unsigned char*>(static_cast<const T*>(a.x) + row * a.ld_x + c0);
                    copy16(ring_x + to, p, min(16, bytes));
                    if (bytes > 16) copy16(ring_x + to + kThreads * 16, p + 16, bytes - 16);
                }
                if (kKept && kAhead > 0) {
                    const unsigned char* p = a.codes + row * a.ld_codes + c0;
                    if (E == 16)
                        copy16(ring_x + (unsigned)(slot * kThreads * 16), p, 16);
                    else
                        asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(ring_x + (unsigned)(slot * kThreads * 16) + 8 * j), "l"(p) : "memory");
                }
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    auto words_of = [&](unsigned from, int slot, int j, unsigned(&w)[8], int n) {
        const unsigned at = from + (unsigned)((slot * V + j) * 2 * kThreads * 16);
        const uint4 p = take16(at), q = n * (int)sizeof(T) > 16 ? take16(at + kThreads * 16) : make_uint4(0, 0, 0, 0);
        w[0] = p.x; w[1] = p.y; w[2] = p.z; w[3] = p.w;
        w[4] = q.x; w[5] = q.y; w[6] = q.z; w[7] = q.w;
    };
    const long long first = (long long)blockIdx.x * S::kGroups + group;
#pragma unroll
    for (int s = 0; s < kAhead - 1; ++s) begin_copy(first + s * stride, s);
    int slot = 0;
    int phase = 0;
    // the statistics and scale bytes of the next row are loaded one row ahead
    float next_mean = 0.0f, next_rstd = 0.0f;
    unsigned next_byte[V];
    auto fetch_small = [&](long long row) {
        if (row >= a.rows) return;
        next_rstd = __ldg(a.rstd + row);
        if (LAYER) next_mean = __ldg(a.mean + row);
        if (kKept) {
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const int c0 = (j * 32 * WPR + t) * E;
                next_byte[j] = c0 < a.cols ? __ldg(a.scales + row * a.ld_scales + c0 / kGroup) : 127u;
            }
        }
    };
    fetch_small(first);
    for (long long row0 = (long long)blockIdx.x * S::kGroups; row0 < a.rows; row0 += stride) {
        const long long row = row0 + group;
        const bool live = row < a.rows;
        if (kAhead > 0) begin_copy(row + (kAhead - 1) * stride, slot == 0 ? kAhead - 1 : slot - 1);
        const float mean = next_mean, rstd = live ? next_rstd : 0.0f;
        float p[V];
        if (kKept) {
#pragma unroll
            for (int j = 0; j < V; ++j) p[j] = scale_of(next_byte[j]);
        }
        fetch_small(row + stride);
        asm volatile("cp.async.wait_group %0;" ::"n"(kAhead > 0 ? kAhead - 1 : 0) : "memory");
        K h[V], g[V];
        float2 c2 = make_float2(0.0f, 0.0f), c1 = make_float2(0.0f, 0.0f);
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const int c0 = (j * 32 * WPR + t) * E;
            const int n = live ? min(E, a.cols - c0) : 0;
            h[j].zero();
            g[j].zero();
            if (n <= 0) continue;
            unsigned w8[8];
            if (async_gy)
                words_of(ring_gy, slot, j, w8, n);
            else
                K::load_words(static_cast<const T*>(a.gy) + row * a.ld_gy + c0, n, w8);
            g[j].from_words(w8);
            if (kKept) {
                constexpr int F = kKept ? FMT : AMPQ_FMT_E4M3;
                const uint4 q = take16(ring_x + (unsigned)(slot * kThreads * 16));
                unsigned c[E / 4];
                if (E == 16) {
                    c[0] = q.x; c[1] = q.y; c[2 % (E / 4)] = q.z; c[3 % (E / 4)] = q.w;
                } else {
                    c[0] = j ? q.z : q.x;
                    c[1] = j ? q.w : q.y;
                }
                h[j].template decode<F>(c);
            } else {
                if (async_x)
                    words_of(ring_x, slot, j, w8, n);
                else
                    K::load_words(static_cast<const T*>(a.x) + row * a.ld_x + c0, n, w8);
                h[j].from_words(w8);
            }
            K w;
            if (a.w) load_params(a.w, a.param_bf16, c0, n, w);
#pragma unroll
            for (int i = 0; i < E / 2; ++i) {
                // (x - mean) * rstd; the scale of a kept x joins the subtraction
                const float2 d = kKept ? __ffma2_rn(h[j].v[i], make_float2(p[j], p[j]), make_float2(-mean, -mean)) : __fadd2_rn(h[j].v[i], make_float2(-mean, -mean));
                float2 hh = __fmul2_rn(d, make_float2(rstd, rstd));
                if (n < E) hh = make_float2(2 * i < n ? hh.x : 0.0f, 2 * i + 1 < n ? hh.y : 0.0f);
                h[j].v[i] = hh;
                sum_w[j][i] = __ffma2_rn(g[j].v[i], hh, sum_w[j][i]);
                if (LAYER) sum_b[j][i] = __fadd2_rn(sum_b[j][i], g[j].v[i]);
                if (a.w) g[j].v[i] = __fmul2_rn(g[j].v[i], w.v[i]);
                c2 = __ffma2_rn(g[j].v[i], hh, c2);
                if (LAYER) c1 = __fadd2_rn(c1, g[j].v[i]);
            }
        }
        float both[2] = {c2.x + c2.y, c1.x + c1.y};
        if (LAYER) {
            row_sum<WPR, 2>(both, red[phase], warp);
        } else {
            float one[1] = {both[0]};
            row_sum<WPR, 1>(one, red[phase], warp);
            both[0] = one[0];
        }
        phase ^= 1;
        const float m2 = -both[0] * inv_cols, m1 = LAYER ? -both[1] * inv_cols : 0.0f;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const int c0 = (j * 32 * WPR + t) * E;
            const int n = live ? min(E, a.cols - c0) : 0;
            if (n <= 0) continue;
#pragma unroll
            for (int i = 0; i < E / 2; ++i) {
                float2 o = __ffma2_rn(h[j].v[i], make_float2(m2, m2), g[j].v[i]);
                if (LAYER) o = __fadd2_rn(o, make_float2(m1, m1));
                g[j].v[i] = __fmul2_rn(o, make_float2(rstd, rstd));
            }
            g[j].store(static_cast<T*>(a.gx) + row * a.ld_gx + c0, n);
        }
        if (++slot == kAhead) slot = 0;
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    if (!a.part) return;
    float* join = reinterpret_cast<float*>(ring);
    for (int k = 0; k < (LAYER && a.sum_b ? 2 : 1); ++k) {
        float* out = a.part + ((long long)k * gridDim.x + blockIdx.x) * a.cols;
        if (S::kGroups == 1) {
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const int c0 = (j * 32 * WPR + t) * E;
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    const float2 f = k ? sum_b[j][i / 2] : sum_w[j][i / 2];
                    if (c0 + i < a.cols) out[c0 + i] = i & 1 ? f.y : f.x;
                }
            }
        } else {
            __syncthreads();
#pragma unroll
            for (int j = 0; j < V; ++j)
#pragma unroll
                for (int i = 0; i < E / 2; ++i)
                    *reinterpret_cast<float2*>(join + group * S::kSpan + (j * 32 * WPR + t) * E + 2 * i) = k ? sum_b[j][i] : sum_w[j][i];
            __syncthreads();
            for (int i = threadIdx.x; i < a.cols; i += kThreads) {
                float s = 0.0f;
#pragma unroll
                for (int g = 0; g < S::kGroups; ++g) s += join[g * S::kSpan + i];
                out[i] = s;
            }
        }
    }
}

// Warps of a row: 512 columns each, a power of two.
int warps_per_row(int cols) { return cols <= 512 ? 1 : cols <= 1024 ? 2 : cols <= 2048 ? 4 : cols <= 4096 ? 8 : cols <= 8192 ? 16 : 32; }

// CTAs of the backward pass: every row group gets a row before one gets two, and
// no more CTAs than are resident, so that the sums stay in registers.
int backward_ctas(long long rows, int cols, int sms) {
    const int wpr = warps_per_row(cols), groups = wpr < 8 ? 8 / wpr : 1;
    const long long need = (rows + groups - 1) / groups;
    const long long most = (long long)sms * (wpr <= 8 ? 2 : 1);
    return (int)(need < most ? need : most);
}

template <typename T, int FMT, int WPR>
void start_forward(const ForwardArgs& a, cudaStream_t st) {
    const long long blocks = (a.rows + Shape<WPR>::kGroups - 1) / Shape<WPR>::kGroups;
    norm_forward_kernel<T, FMT, WPR><<<(unsigned)blocks, Shape<WPR>::kThreads, 0, st>>>(a);
}

template <typename T, int FMT>
int launch_forward(const ForwardArgs& a, cudaStream_t st) {
    switch (warps_per_row(a.cols)) {
        case 1: start_forward<T, FMT, 1>(a, st); break;
        case 2: start_forward<T, FMT, 2>(a, st); break;
        case 4: start_forward<T, FMT, 4>(a, st); break;
        case 8: start_forward<T, FMT, 8>(a, st); break;
        case 16: start_forward<T, FMT, 16>(a, st); break;
        default: start_forward<T, FMT, 32>(a, st);
    }
    return launched();
}

constexpr int kMaxDevices = 64;

template <typename T, int FMT, bool LAYER, int WPR>
int start_backward(const BackwardArgs& a, int device, int ctas, cudaStream_t st) {
    static std::atomic<bool> prepared[kMaxDevices];  // the kernel may use its shared memory on that device
    constexpr int kJoin = Shape<WPR>::kGroups > 1 ? Shape<WPR>::kGroups * Shape<WPR>::kSpan * 4 : 0;
    constexpr int kBytes = Ring<T, FMT, WPR>::kBytes > kJoin ? Ring<T, FMT, WPR>::kBytes : kJoin;
    if (kBytes > 32 * 1024 && (device >= kMaxDevices || !prepared[device].load(std::memory_order_acquire))) {
        if (cudaFuncSetAttribute(norm_backward_kernel<T, FMT, LAYER, WPR>, cudaFuncAttributeMaxDynamicSharedMemorySize, kBytes) != cudaSuccess) {
            cudaGetLastError();
            return AMPQ_ERR_CUDA;
        }
        if (device < kMaxDevices) prepared[device].store(true, std::memory_order_release);
    }
    norm_backward_kernel<T, FMT, LAYER, WPR><<<(unsigned)ctas, Shape<WPR>::kThreads, kBytes, st>>>(a);
    return launched();
}

template <typename T, int FMT, bool LAYER>
int launch_backward(const BackwardArgs& a, int device, int ctas, cudaStream_t st) {
    switch (warps_per_row(a.cols)) {
        case 1: return start_backward<T, FMT, LAYER, 1>(a, device, ctas, st);
        case 2: return start_backward<T, FMT, LAYER, 2>(a, device, ctas, st);
        case 4: return start_backward<T, FMT, LAYER, 4>(a, device, ctas, st);
        case 8: return start_backward<T, FMT, LAYER, 8>(a, device, ctas, st);
        case 16: return start_backward<T, FMT, LAYER, 16>(a, device, ctas, st);
        default: return start_backward<T, FMT, LAYER, 32>(a, device, ctas, st);
    }
}

template <typename T>
int dispatch_forward(int fmt, const ForwardArgs& a, cudaStream_t st) {
    if (fmt == AMPQ_FMT_E4M3) return launch_forward<T, AMPQ_FMT_E4M3>(a, st);
    if (fmt == AMPQ_FMT_E5M2) return launch_forward<T, AMPQ_FMT_E5M2>(a, st);
    return launch_forward<T, AMPQ_FMT_BASE>(a, st);
}

template <typename T, bool LAYER>
int dispatch_backward(int fmt, const BackwardArgs& a, int device, int ctas, cudaStream_t st) {
    if (fmt == AMPQ_FMT_E4M3) return launch_backward<T, AMPQ_FMT_E4M3, LAYER>(a, device, ctas, st);
    if (fmt == AMPQ_FMT_E5M2) return launch_backward<T, AMPQ_FMT_E5M2, LAYER>(a, device, ctas, st);
    return launch_backward<T, AMPQ_FMT_BASE, LAYER>(a, device, ctas, st);
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
    if (rows == 0 || cols == 0) return AMPQ_OK;
    ForwardArgs a;
    a.x = x; a.w = weight; a.b = bias; a.y = y;
    a.mean = mean; a.rstd = rstd;
    a.codes = codes; a.scales = scales;
    a.rows = rows; a.ld_x = ld_x; a.ld_y = ld_y; a.ld_codes = ld_codes; a.ld_scales = ld_scales;
    a.cols = (int)cols;
    a.eps = eps;
    a.layer = layer;
    a.param_bf16 = param_dtype == AMPQ_BF16;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
    return dtype == AMPQ_F32 ? dispatch_forward<float>(fmt, a, st) : dispatch_forward<__nv_bfloat16>(fmt, a, st);
}

int ampq_norm_backward_workspace(int device, long long rows, long long cols, long long* bytes) {
    if (!bytes || rows < 0 || cols < 0) return AMPQ_ERR_INVALID;
    if (cols > kMaxNormCols || rows > kMaxRows) return AMPQ_ERR_TOO_LARGE;
    CkptDevice cur(device);
    if (cur.status) return cur.status;
    const int sms = sm_count(device);
    if (sms < 1) return AMPQ_ERR_CUDA;
    *bytes = 2LL * backward_ctas(rows, (int)cols, sms) * cols * (long long)sizeof(float);
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
    if (sums && ctas > 0 && (!workspace || workspace_bytes < 2LL * ctas * cols * (long long)sizeof(float))) return AMPQ_ERR_INVALID;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
    if (rows > 0) {
        BackwardArgs a;
        a.gy = gy; a.x = x; a.w = weight;
        a.codes = codes; a.scales = scales;
        a.mean = mean; a.rstd = rstd;
        a.gx = gx;
        a.part = sums ? static_cast<float*>(workspace) : nullptr;
        a.rows = rows; a.ld_gy = ld_gy; a.ld_x = ld_x; a.ld_codes = ld_codes; a.ld_scales = ld_scales; a.ld_gx = ld_gx;
        a.cols = (int)cols;
        a.param_bf16 = param_dtype == AMPQ_BF16;
        a.sum_b = gbias != nullptr;
        a.async_gy = rows_aligned(gy, ld_gy, dtype);
        a.async_x = rows_aligned(x, ld_x, dtype);
        if (dtype == AMPQ_F32)
            rc = layer ? dispatch_backward<float, true>(fmt, a, device, ctas, st) : dispatch_backward<float, false>(fmt, a, device, ctas, st);
        else
            rc = layer ? dispatch_backward<__nv_bfloat16, true>(fmt, a, device, ctas, st) : dispatch_backward<__nv_bfloat16, false>(fmt, a, device, ctas, st);
        if (rc) return rc;
    }
    if (!sums) return AMPQ_OK;
    return launch_join_columns(static_cast<const float*>(workspace), gbias ? 2 : 1, ctas, cols, gweight, gbias, param_dtype, st);
}

#pragma GCC visibility pop
}  // extern "C"
