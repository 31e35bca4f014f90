// Weight gradient of linear layers from the 8-bit checkpoint of their input
// (include/ampq.h: ampq_ckpt_weight_grad): for every sample r
//   gW[r][k][c] = sum_n gY[r][n][k] * X^[r][n][c],  gb[r][k] = sum_n gY[r][n][k].
#include "ampq_ckpt.h"

namespace ampq {
namespace {

struct WgradArgs {
    const void* gy;
    const unsigned char *codes, *scales;
    void* gw;
    long long ld_gy, ld_codes, ld_scales, samples, rows, cols, outs;
};

constexpr int kT = 64, kStep = 16;

// A 64 x 64 tile of one sample's gradient, sixteen rows at a time through
// shared memory, fp32 products and sums.
template <typename T, int FMT>
__global__ void __launch_bounds__(256) wgrad_simple_kernel(const WgradArgs a) {
    __shared__ float sg[kStep][kT + 4], sx[kStep][kT + 4];
    const long long k0 = (long long)blockIdx.x * kT, c0 = (long long)blockIdx.y * kT;
    const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
    for (long long r = blockIdx.z; r < a.samples; r += gridDim.z) {
        float acc[4][4] = {};
        for (long long n0 = 0; n0 < a.rows; n0 += kStep) {
            __syncthreads();
            for (int i = threadIdx.x; i < kStep * kT; i += 256) {
                const int n = i / kT, q = i % kT;
                const long long row = r * a.rows + n0 + n;
                const bool in = n0 + n < a.rows;
                sg[n][q] = in && k0 + q < a.outs ? load_elem(static_cast<const T*>(a.gy) + row * a.ld_gy + k0 + q) : 0.0f;
            }
            for (int i = threadIdx.x; i < kStep * kT / 8; i += 256) {
                const int n = i / (kT / 8), q = i % (kT / 8) * 8;
                const long long row = r * a.rows + n0 + n;
                float v[8] = {};
                if (n0 + n < a.rows && c0 + q < a.cols) {
                    decode8<FMT>(__ldg(reinterpret_cast<const uint2*>(a.codes + row * a.ld_codes + c0 + q)), v);
                    const float p = scale_of(__ldg(a.scales + row * a.ld_scales + (c0 + q) / kGroup));
#pragma unroll
                    for (int k = 0; k < 8; ++k) v[k] *= p;
                }
#pragma unroll
                for (int k = 0; k < 8; ++k) sx[n][q + k] = v[k];
            }
            __syncthreads();
#pragma unroll
            for (int n = 0; n < kStep; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(sg[n][ty * 4 + i], sx[n][tx * 4 + j], acc[i][j]);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const long long k = k0 + ty * 4 + i, c = c0 + tx * 4 + j;
                if (k < a.outs && c < a.cols) store_elem(static_cast<T*>(a.gw) + (r * a.outs + k) * a.cols + c, acc[i][j]);
            }
    }
}

// Partial column sums: block (x, y, r) sums rows y, y + gridDim.y * 8, ... of
// sample r for 32 columns... one column per thread, eight row lanes per block.
constexpr int kSumCols = 32, kSumWays = 8;

template <typename T>
__global__ void __launch_bounds__(kSumCols * kSumWays) column_sums_kernel(const T* __restrict__ g, long long ld, long long samples, long long rows, long long cols,
                                                                          float* __restrict__ part) {
    __shared__ float sums[kSumWays][kSumCols];
    const long long c = (long long)blockIdx.x * kSumCols + threadIdx.x;
    for (long long r = blockIdx.z; r < samples; r += gridDim.z) {
        float s = 0.0f;
        if (c < cols)
            for (long long n = (long long)blockIdx.y * kSumWays + threadIdx.y; n < rows; n += (long long)gridDim.y * kSumWays)
                s += load_elem(g + (r * rows + n) * ld + c);
        __syncthreads();
        sums[threadIdx.y][threadIdx.x] = s;
        __syncthreads();
        if (threadIdx.y == 0 && c < cols) {
            float t = 0.0f;
#pragma unroll
            for (int k = 0; k < kSumWays; ++k) t += sums[k][threadIdx.x];
            part[(r * gridDim.y + blockIdx.y) * cols + c] = t;
        }
    }
}

// Row lanes of the column sums: about 64 rows to a thread.
int sum_parts(long long rows) {
    const long long p = (rows + 64 * kSumWays - 1) / (64 * kSumWays);
    return (int)(p < 1 ? 1 : p > 256 ? 256 : p);
}

template <typename T, int FMT>
int launch_wgrad(const WgradArgs& a, cudaStream_t st) {
    const long long bx = (a.outs + kT - 1) / kT, by = (a.cols + kT - 1) / kT;
    if (by > 65535) return AMPQ_ERR_TOO_LARGE;
    const unsigned bz = (unsigned)(a.samples < 65535 ? a.samples : 65535);
    wgrad_simple_kernel<T, FMT><<<dim3((unsigned)bx, (unsigned)by, bz), 256, 0, st>>>(a);
    return launched();
}

template <typename T>
int bias_grad(const WgradArgs& a, void* gb, int dtype, float* part, cudaStream_t st) {
    const int parts = sum_parts(a.rows);
    const unsigned bz = (unsigned)(a.samples < 65535 ? a.samples : 65535);
    column_sums_kernel<T><<<dim3((unsigned)((a.outs + kSumCols - 1) / kSumCols), parts, bz), dim3(kSumCols, kSumWays), 0, st>>>(
        static_cast<const T*>(a.gy), a.ld_gy, a.samples, a.rows, a.outs, part);
    const int rc = launched();
    return rc ? rc : launch_join_columns(part, a.samples, parts, a.outs, gb, nullptr, dtype, st);
}

long long workspace_of(long long samples, long long rows, long long outs, int bias) {
    return bias ? samples * sum_parts(rows) * outs * (long long)sizeof(float) : 0;
}

int check_sizes(int dtype, long long samples, long long rows, long long cols, long long outs) {
    if (!known_dtype(dtype) || samples < 0 || rows < 0 || cols < 0 || outs < 0) return AMPQ_ERR_INVALID;
    if (cols > kMaxCols || outs > kMaxCols || samples > kMaxRows || rows > kMaxRows || (samples > 0 && rows > kMaxRows / samples)) return AMPQ_ERR_TOO_LARGE;
    return AMPQ_OK;
}

}  // namespace
}  // namespace ampq

using namespace ampq;

extern "C" {
#pragma GCC visibility push(default)

int ampq_ckpt_weight_grad_workspace(int device, int dtype, const void* gy, long long ld_gy, long long samples, long long rows, long long cols,
                                    long long outs, int bias, long long* bytes) {
    if (!bytes) return AMPQ_ERR_INVALID;
    const int rc = check_sizes(dtype, samples, rows, cols, outs);
    if (rc) return rc;
    CkptDevice cur(device);
    if (cur.status) return cur.status;
    *bytes = workspace_of(samples, rows, outs, bias);
    return AMPQ_OK;
}

int ampq_ckpt_weight_grad(int device, void* cuda_stream, int dtype, int fmt, const void* gy, long long ld_gy, const unsigned char* codes,
                          long long ld_codes, const unsigned char* scales, long long ld_scales, long long samples, long long rows,
                          long long cols, long long outs, void* gw, void* gb, void* workspace, long long workspace_bytes) {
    if (!known_fp8(fmt)) return AMPQ_ERR_INVALID;
    int rc = check_sizes(dtype, samples, rows, cols, outs);
    if (!rc) rc = check_matrix(gy, samples * rows, outs, ld_gy, dtype);
    if (!rc) rc = check_ckpt(codes, ld_codes, scales, ld_scales, samples * rows, cols);
    if (rc) return rc;
    if (samples > 0 && outs > 0 && cols > 0 && !gw) return AMPQ_ERR_INVALID;
    if (!aligned_to(gw, elem_bytes(dtype)) || !aligned_to(gb, elem_bytes(dtype)) || !aligned_to(workspace, 256)) return AMPQ_ERR_ALIGN;
    CkptDevice cur(device);
    if (cur.status) return cur.status;
    if (samples == 0 || outs == 0) return AMPQ_OK;
    const long long need = workspace_of(samples, rows, outs, gb != nullptr);
    if (need > 0 && (!workspace || workspace_bytes < need)) return AMPQ_ERR_INVALID;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
    const WgradArgs a{gy, codes, scales, gw, ld_gy, ld_codes, ld_scales, samples, rows, cols, outs};
    if (cols > 0) {
        const bool e4 = fmt == AMPQ_FMT_E4M3;
        if (dtype == AMPQ_F32)
            rc = e4 ? launch_wgrad<float, AMPQ_FMT_E4M3>(a, st) : launch_wgrad<float, AMPQ_FMT_E5M2>(a, st);
        else
            rc = e4 ? launch_wgrad<__nv_bfloat16, AMPQ_FMT_E4M3>(a, st) : launch_wgrad<__nv_bfloat16, AMPQ_FMT_E5M2>(a, st);
        if (rc) return rc;
    }
    if (!gb) return AMPQ_OK;
    float* part = static_cast<float*>(workspace);
    return dtype == AMPQ_F32 ? bias_grad<float>(a, gb, dtype, part, st) : bias_grad<__nv_bfloat16>(a, gb, dtype, part, st);
}

#pragma GCC visibility pop
}  // extern "C"
