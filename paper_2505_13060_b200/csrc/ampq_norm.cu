// Layer norm and RMS norm, forward and backward (include/ampq.h:
// ampq_norm_forward, ampq_norm_backward), with the 8-bit checkpoint of the
// input written by the forward pass and read by the backward pass.
#include "ampq_ckpt.h"

#include <cmath>

namespace ampq {
namespace {

constexpr int kMaxNormCols = AMPQ_NORM_MAX_COLS;

// Eight elements of a parameter vector, in fp32.  p: float or bf16 by `bf16`;
// vec: 16-byte aligned.
__device__ __forceinline__ void load_param8(const void* p, bool bf16, bool vec, int c0, int n, float (&v)[8]) {
    if (bf16) {
        Raw8<__nv_bfloat16> r;
        if (vec)
            load8<true>(r, static_cast<const __nv_bfloat16*>(p) + c0, n);
        else
            load8<false>(r, static_cast<const __nv_bfloat16*>(p) + c0, n);
        r.values(v);
    } else {
        Raw8<float> r;
        if (vec)
            load8<true>(r, static_cast<const float*>(p) + c0, n);
        else
            load8<false>(r, static_cast<const float*>(p) + c0, n);
        r.values(v);
    }
}

// Sum of one value (two) over the WPR warps of a row group; every thread of the
// CTA calls it.  The order is fixed.
template <int WPR, int N>
__device__ __forceinline__ void row_sum(float (&s)[N], float* red, int warp) {
#pragma unroll
    for (int k = 0; k < N; ++k)
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) s[k] += __shfl_xor_sync(0xFFFFFFFFu, s[k], o);
    if (WPR == 1) return;
    __syncthreads();  // red is free again
    if ((threadIdx.x & 31) == 0)
#pragma unroll
        for (int k = 0; k < N; ++k) red[warp * N + k] = s[k];
    __syncthreads();
    const int first = warp / WPR * WPR;
#pragma unroll
    for (int k = 0; k < N; ++k) {
        float t = 0.0f;
#pragma unroll
        for (int i = 0; i < WPR; ++i) t += red[(first + i) * N + k];
        s[k] = t;
    }
}

template <int WPR>
struct Shape {
    static constexpr int kWarps = WPR < 8 ? 8 : WPR;   // warps of a CTA
    static constexpr int kGroups = kWarps / WPR;       // rows a CTA works on at a time
    static constexpr int kThreads = 32 * kWarps;
};

struct ForwardArgs {
    const void *x, *w, *b;
    void* y;
    float *mean, *rstd;
    unsigned char *codes, *scales;
    long long rows, ld_x, ld_y, ld_codes, ld_scales;
    int cols;
    float eps;
    bool layer, param_bf16, vec_x, vec_y, vec_p;
};

// One row per group of WPR warps, held in registers between the statistics (two
// passes over the registers: mean, then the sum of squared differences) and the
// output, so x is read once.  Lane l of the group holds columns
// (j * threads + l) * 8 .. + 7: loads are contiguous and four neighbouring lanes
// make one group of the checkpoint.
template <typename T, int FMT, int WPR, int V>
__global__ void __launch_bounds__(Shape<WPR>::kThreads) norm_forward_kernel(const ForwardArgs a) {
    using S = Shape<WPR>;
    __shared__ float red[S::kWarps];
    const int warp = threadIdx.x / 32;
    const int t = threadIdx.x % (32 * WPR);
    const long long row = (long long)blockIdx.x * S::kGroups + warp / WPR;
    const bool live = row < a.rows;
    const T* x = static_cast<const T*>(a.x) + row * a.ld_x;
    Raw8<T> raw[V];
    int n[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
        const int c0 = (j * 32 * WPR + t) * 8;
        n[j] = live ? max(0, min(8, a.cols - c0)) : 0;
        if (n[j] <= 0)
            raw[j].zero();
        else if (a.vec_x)
            load8<true>(raw[j], x + c0, n[j]);
        else
            load8<false>(raw[j], x + c0, n[j]);
    }
    const float cols = (float)a.cols;
    float mean = 0.0f;
    if (a.layer) {
        float s[1] = {0.0f};
#pragma unroll
        for (int j = 0; j < V; ++j) {
            float v[8];
            raw[j].values(v);
#pragma unroll
            for (int i = 0; i < 8; ++i) s[0] += v[i];
        }
        row_sum<WPR, 1>(s, red, warp);
        mean = s[0] / cols;
    }
    float q[1] = {0.0f};
#pragma unroll
    for (int j = 0; j < V; ++j) {
        float v[8];
        raw[j].values(v);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float d = i < n[j] ? v[i] - mean : 0.0f;
            q[0] = fmaf(d, d, q[0]);
        }
    }
    row_sum<WPR, 1>(q, red, warp);
    const float rstd = 1.0f / sqrtf(q[0] / cols + a.eps);
    if (live && t == 0) {
        if (a.layer) a.mean[row] = mean;
        a.rstd[row] = rstd;
    }
#pragma unroll
    for (int j = 0; j < V; ++j) {
        const int c0 = (j * 32 * WPR + t) * 8;
        float v[8];
        raw[j].values(v);
        if (FMT != AMPQ_FMT_BASE) {
            constexpr int F = FMT == AMPQ_FMT_BASE ? AMPQ_FMT_E4M3 : FMT;
            unsigned m = amax_bits8(v);
            m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, 1));
            m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, 2));
            const unsigned byte = scale_byte<F>(m);
            const uint2 c = encode_group8<F>(v, byte);
            if (live && (c0 & ~(kGroup - 1)) < a.cols) {  // whole groups: the columns behind the last are stored as 0
                *reinterpret_cast<uint2*>(a.codes + row * a.ld_codes + c0) = c;
                if ((t & 3) == 0) a.scales[row * a.ld_scales + c0 / kGroup] = (unsigned char)byte;
            }
        }
        if (n[j] <= 0) continue;
        float w[8], b[8];
        if (a.w) load_param8(a.w, a.param_bf16, a.vec_p, c0, n[j], w);
        if (a.b) load_param8(a.b, a.param_bf16, a.vec_p, c0, n[j], b);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float h = (v[i] - mean) * rstd;
            if (a.w) h *= w[i];
            if (a.b) h += b[i];
            v[i] = h;
        }
        Raw8<T> out;
        out.set(v);
        T* y = static_cast<T*>(a.y) + row * a.ld_y + c0;
        if (a.vec_y)
            store8<true>(out, y, n[j]);
        else
            store8<false>(out, y, n[j]);
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
    bool param_bf16, vec_gy, vec_x, vec_gx, vec_p, sum_b;
};

// Rows are dealt to the row groups of a persistent grid; a thread keeps the
// fp32 sums of gy*h and gy of its columns in registers over all its rows.  The
// groups of a CTA are joined in shared memory, the CTAs by join_columns_kernel,
// both in a fixed order.
template <typename T, int FMT, bool LAYER, int WPR, int V>
__global__ void __launch_bounds__(Shape<WPR>::kThreads) norm_backward_kernel(const BackwardArgs a) {
    using S = Shape<WPR>;
    __shared__ float red[S::kWarps * 2];
    __shared__ float join[S::kGroups > 1 ? S::kGroups * WPR * 256 * V : 1];
    const int warp = threadIdx.x / 32;
    const int t = threadIdx.x % (32 * WPR);
    const int group = warp / WPR;
    float sum_w[V][8], sum_b[V][8];
#pragma unroll
    for (int j = 0; j < V; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i) sum_w[j][i] = sum_b[j][i] = 0.0f;
    const float inv_cols = 1.0f / (float)a.cols;
    for (long long row0 = (long long)blockIdx.x * S::kGroups; row0 < a.rows; row0 += (long long)gridDim.x * S::kGroups) {
        const long long row = row0 + group;
        const bool live = row < a.rows;
        const float mean = LAYER && live ? __ldg(a.mean + row) : 0.0f;
        const float rstd = live ? __ldg(a.rstd + row) : 0.0f;
        float h[V][8], g[V][8];
        float c[2] = {0.0f, 0.0f};
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const int c0 = (j * 32 * WPR + t) * 8;
            const int n = live ? max(0, min(8, a.cols - c0)) : 0;
            if (n <= 0) {
#pragma unroll
                for (int i = 0; i < 8; ++i) h[j][i] = g[j][i] = 0.0f;
                continue;
            }
            Raw8<T> r;
            const T* gy = static_cast<const T*>(a.gy) + row * a.ld_gy + c0;
            if (a.vec_gy)
                load8<true>(r, gy, n);
            else
                load8<false>(r, gy, n);
            r.values(g[j]);
            if (FMT != AMPQ_FMT_BASE) {
                constexpr int F = FMT == AMPQ_FMT_BASE ? AMPQ_FMT_E4M3 : FMT;
                decode8<F>(__ldg(reinterpret_cast<const uint2*>(a.codes + row * a.ld_codes + c0)), h[j]);
                const float p = scale_of(__ldg(a.scales + row * a.ld_scales + c0 / kGroup));
#pragma unroll
                for (int i = 0; i < 8; ++i) h[j][i] *= p;
            } else {
                const T* x = static_cast<const T*>(a.x) + row * a.ld_x + c0;
                if (a.vec_x)
                    load8<true>(r, x, n);
                else
                    load8<false>(r, x, n);
                r.values(h[j]);
            }
            float w[8];
            if (a.w) load_param8(a.w, a.param_bf16, a.vec_p, c0, n, w);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                h[j][i] = i < n ? (h[j][i] - mean) * rstd : 0.0f;
                sum_w[j][i] = fmaf(g[j][i], h[j][i], sum_w[j][i]);
                sum_b[j][i] += g[j][i];
                if (a.w) g[j][i] *= w[i];
                c[0] = fmaf(g[j][i], h[j][i], c[0]);
                c[1] += g[j][i];
            }
        }
        row_sum<WPR, 2>(c, red, warp);
        const float c2 = c[0] * inv_cols, c1 = LAYER ? c[1] * inv_cols : 0.0f;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const int c0 = (j * 32 * WPR + t) * 8;
            const int n = live ? max(0, min(8, a.cols - c0)) : 0;
            if (n <= 0) continue;
            float o[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) o[i] = rstd * (fmaf(-h[j][i], c2, g[j][i]) - c1);
            Raw8<T> r;
            r.set(o);
            T* gx = static_cast<T*>(a.gx) + row * a.ld_gx + c0;
            if (a.vec_gx)
                store8<true>(r, gx, n);
            else
                store8<false>(r, gx, n);
        }
    }
    if (!a.part) return;
    for (int k = 0; k < (a.sum_b ? 2 : 1); ++k) {
        float* out = a.part + ((long long)k * gridDim.x + blockIdx.x) * a.cols;
        if (S::kGroups == 1) {
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const int c0 = (j * 32 * WPR + t) * 8;
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (c0 + i < a.cols) out[c0 + i] = k ? sum_b[j][i] : sum_w[j][i];
            }
        } else {
            constexpr int kSpan = WPR * 256 * V;
            __syncthreads();
#pragma unroll
            for (int j = 0; j < V; ++j)
#pragma unroll
                for (int i = 0; i < 8; ++i) join[group * kSpan + (j * 32 * WPR + t) * 8 + i] = k ? sum_b[j][i] : sum_w[j][i];
            __syncthreads();
            for (int i = threadIdx.x; i < a.cols; i += S::kThreads) {
                float s = 0.0f;
#pragma unroll
                for (int g = 0; g < S::kGroups; ++g) s += join[g * kSpan + i];
                out[i] = s;
            }
        }
    }
}

// CTAs of the backward pass: every row group gets a row before one gets two,
// and no more CTAs than are resident, so that the sums stay in registers.
int backward_ctas(long long rows, int cols, int sms) {
    const int wpr = cols <= 512 ? 1 : cols <= 1024 ? 2 : cols <= 2048 ? 4 : cols <= 4096 ? 8 : cols <= 8192 ? 16 : 32;
    const int groups = wpr < 8 ? 8 / wpr : 1;
    const long long need = (rows + groups - 1) / groups;
    const long long most = (long long)sms * (wpr <= 8 ? 2 : 1);
    return (int)(need < most ? need : most);
}

template <typename T, int FMT>
int launch_forward(const ForwardArgs& a, cudaStream_t st) {
#define AMPQ_FWD(WPR, V)                                                                                      \
    do {                                                                                                      \
        const long long blocks = (a.rows + Shape<WPR>::kGroups - 1) / Shape<WPR>::kGroups;                    \
        norm_forward_kernel<T, FMT, WPR, V><<<(unsigned)blocks, Shape<WPR>::kThreads, 0, st>>>(a);            \
    } while (0)
    if (a.cols <= 256) AMPQ_FWD(1, 1);
    else if (a.cols <= 512) AMPQ_FWD(1, 2);
    else if (a.cols <= 1024) AMPQ_FWD(1, 4);
    else if (a.cols <= 2048) AMPQ_FWD(2, 4);
    else if (a.cols <= 4096) AMPQ_FWD(4, 4);
    else if (a.cols <= 8192) AMPQ_FWD(8, 4);
    else AMPQ_FWD(16, 4);
#undef AMPQ_FWD
    return launched();
}

template <typename T, int FMT, bool LAYER>
int launch_backward(const BackwardArgs& a, int ctas, cudaStream_t st) {
#define AMPQ_BWD(WPR, V) norm_backward_kernel<T, FMT, LAYER, WPR, V><<<(unsigned)ctas, Shape<WPR>::kThreads, 0, st>>>(a)
    if (a.cols <= 256) AMPQ_BWD(1, 1);
    else if (a.cols <= 512) AMPQ_BWD(1, 2);
    else if (a.cols <= 1024) AMPQ_BWD(2, 2);
    else if (a.cols <= 2048) AMPQ_BWD(4, 2);
    else if (a.cols <= 4096) AMPQ_BWD(8, 2);
    else if (a.cols <= 8192) AMPQ_BWD(16, 2);
    else AMPQ_BWD(32, 2);
#undef AMPQ_BWD
    return launched();
}

template <typename T>
int dispatch_forward(int fmt, const ForwardArgs& a, cudaStream_t st) {
    if (fmt == AMPQ_FMT_E4M3) return launch_forward<T, AMPQ_FMT_E4M3>(a, st);
    if (fmt == AMPQ_FMT_E5M2) return launch_forward<T, AMPQ_FMT_E5M2>(a, st);
    return launch_forward<T, AMPQ_FMT_BASE>(a, st);
}

template <typename T, bool LAYER>
int dispatch_backward(int fmt, const BackwardArgs& a, int ctas, cudaStream_t st) {
    if (fmt == AMPQ_FMT_E4M3) return launch_backward<T, AMPQ_FMT_E4M3, LAYER>(a, ctas, st);
    if (fmt == AMPQ_FMT_E5M2) return launch_backward<T, AMPQ_FMT_E5M2, LAYER>(a, ctas, st);
    return launch_backward<T, AMPQ_FMT_BASE, LAYER>(a, ctas, st);
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
    a.vec_x = rows_aligned(x, ld_x, dtype);
    a.vec_y = rows_aligned(y, ld_y, dtype);
    a.vec_p = aligned_to(weight, 16) && aligned_to(bias, 16);
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
        a.vec_gy = rows_aligned(gy, ld_gy, dtype);
        a.vec_x = rows_aligned(x, ld_x, dtype);
        a.vec_gx = rows_aligned(gx, ld_gx, dtype);
        a.vec_p = aligned_to(weight, 16);
        a.sum_b = gbias != nullptr;
        if (dtype == AMPQ_F32)
            rc = layer ? dispatch_backward<float, true>(fmt, a, ctas, st) : dispatch_backward<float, false>(fmt, a, ctas, st);
        else
            rc = layer ? dispatch_backward<__nv_bfloat16, true>(fmt, a, ctas, st) : dispatch_backward<__nv_bfloat16, false>(fmt, a, ctas, st);
        if (rc) return rc;
    }
    if (!sums) return AMPQ_OK;
    return launch_join_columns(static_cast<const float*>(workspace), gbias ? 2 : 1, ctas, cols, gweight, gbias, param_dtype, st);
}

#pragma GCC visibility pop
}  // extern "C"
