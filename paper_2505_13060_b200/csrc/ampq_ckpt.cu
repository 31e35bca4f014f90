// Writing and reading 8-bit checkpoints (include/ampq.h: ampq_ckpt_pack,
// ampq_ckpt_unpack), and the column sums shared by the gradients' kernels.
#include "ampq_ckpt.h"

#include <atomic>

namespace ampq {
namespace {

constexpr int kThreads = 256;
constexpr int kUnroll = 4;                                     // vectors of eight a thread has in flight
constexpr int kGroupsPerBlock = kThreads / 4 * kUnroll;        // four threads per group

// n / d for n < 2^31 by a multiplication: magic = floor(2^(31+s)/d) + 1 with 2^s >= d.
struct FastDiv {
    unsigned d, magic, shift;
    explicit FastDiv(unsigned div) : d(div), magic(0), shift(0) {
        if (div <= 1) return;
        unsigned s = 0;
        while ((1ull << s) < div) ++s;
        magic = (unsigned)(((1ull << (31 + s)) / div) + 1);
        shift = s - 1;
    }
    __device__ __forceinline__ unsigned operator()(unsigned n) const { return d <= 1 ? n : __umulhi(n, magic) >> shift; }
};

// The group that a thread's vector belongs to: groups are numbered row by row,
// a block takes kGroupsPerBlock of them, four threads share one.  The 64-bit
// division is done once per block.
struct Place {
    long long row;
    unsigned group;
};

struct BlockStart {
    long long row0;
    unsigned group0;
    __device__ __forceinline__ BlockStart(unsigned groups) {
        const long long first = (long long)blockIdx.x * kGroupsPerBlock;
        row0 = first / groups;
        group0 = (unsigned)(first - row0 * groups);
    }
    __device__ __forceinline__ Place at(unsigned local, unsigned groups, const FastDiv& div) const {
        const unsigned n = group0 + local;
        const unsigned q = div(n);
        return Place{row0 + q, n - q * groups};
    }
};

// One read of x, one write of codes and scale bytes: bound by HBM.  A thread
// holds eight consecutive columns (one 16-byte load of bf16, two of fp32), four
// lanes a group, so the group's maximum is two shuffles.
template <typename T, int FMT, bool VEC>
__global__ void __launch_bounds__(kThreads) pack_kernel(const T* __restrict__ x, long long rows, unsigned cols, long long ld,
                                                        unsigned groups, FastDiv div, unsigned char* __restrict__ codes, long long ld_codes,
                                                        unsigned char* __restrict__ scales, long long ld_scales) {
    const BlockStart start(groups);
    Raw8<T> raw[kUnroll];
    Place pl[kUnroll];
    const unsigned lane4 = threadIdx.x & 3;
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
        pl[u] = start.at(u * (kThreads / 4) + threadIdx.x / 4, groups, div);
        const unsigned c0 = pl[u].group * kGroup + lane4 * 8;
        const int n = pl[u].row < rows ? max(0, min(8, (int)cols - (int)c0)) : 0;
        if (n > 0)
            load8<VEC>(raw[u], x + pl[u].row * ld + c0, n);
        else
            raw[u].zero();
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
        float v[8];
        raw[u].values(v);
        unsigned m = amax_bits8(v);
        m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, 1));
        m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, 2));
        const unsigned byte = scale_byte<FMT>(m);
        const uint2 c = encode_group8<FMT>(v, byte);
        if (pl[u].row < rows) {
            *reinterpret_cast<uint2*>(codes + pl[u].row * ld_codes + pl[u].group * kGroup + lane4 * 8) = c;
            if (lane4 == 0) scales[pl[u].row * ld_scales + pl[u].group] = (unsigned char)byte;
        }
    }
}

template <typename T, int FMT, bool VEC>
__global__ void __launch_bounds__(kThreads) unpack_kernel(const unsigned char* __restrict__ codes, long long ld_codes,
                                                          const unsigned char* __restrict__ scales, long long ld_scales, long long rows,
                                                          unsigned cols, unsigned groups, FastDiv div, T* __restrict__ out, long long ld) {
    const BlockStart start(groups);
    uint2 c[kUnroll];
    unsigned byte[kUnroll];
    Place pl[kUnroll];
    const unsigned lane4 = threadIdx.x & 3;
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
        pl[u] = start.at(u * (kThreads / 4) + threadIdx.x / 4, groups, div);
        c[u] = make_uint2(0, 0);
        byte[u] = 127;
        if (pl[u].row < rows) {
            c[u] = __ldg(reinterpret_cast<const uint2*>(codes + pl[u].row * ld_codes + pl[u].group * kGroup + lane4 * 8));
            byte[u] = __ldg(scales + pl[u].row * ld_scales + pl[u].group);
        }
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
        const unsigned c0 = pl[u].group * kGroup + lane4 * 8;
        const int n = pl[u].row < rows ? max(0, min(8, (int)cols - (int)c0)) : 0;
        if (n <= 0) continue;
        float v[8];
        decode8<FMT>(c[u], v);
        const float p = scale_of(byte[u]);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] *= p;
        Raw8<T> r;
        r.set(v);
        store8<VEC>(r, out + pl[u].row * ld + c0, n);
    }
}

// ---------------------------------------------------------------------------
// joining column sums

constexpr int kJoinCols = 32, kJoinWays = 32;

template <typename T>
__global__ void __launch_bounds__(kJoinCols * kJoinWays) join_columns_kernel(const float* __restrict__ part, int parts, long long cols, T* __restrict__ out,
                                                                             T* __restrict__ second) {
    __shared__ float sums[kJoinWays][kJoinCols];
    const long long c = (long long)blockIdx.x * kJoinCols + threadIdx.x;
    const long long batch = blockIdx.y;
    float s = 0.0f;
    if (c < cols)
        for (int p = threadIdx.y; p < parts; p += kJoinWays) s += __ldg(part + (batch * parts + p) * cols + c);
    sums[threadIdx.y][threadIdx.x] = s;
    __syncthreads();
    if (threadIdx.y == 0 && c < cols) {
        float t = 0.0f;
#pragma unroll
        for (int k = 0; k < kJoinWays; ++k) t += sums[k][threadIdx.x];
        store_elem((second && batch > 0 ? second + (batch - 1) * cols : out + batch * cols) + c, t);
    }
}

template <typename T, int FMT>
int launch_pack(const void* x, long long rows, long long cols, long long ld, unsigned char* codes, long long ld_codes,
                unsigned char* scales, long long ld_scales, cudaStream_t st) {
    const unsigned groups = (unsigned)((cols + kGroup - 1) / kGroup);
    const long long blocks = (rows * groups + kGroupsPerBlock - 1) / kGroupsPerBlock;
    if (blocks > 0x7FFFFFFFLL) return AMPQ_ERR_TOO_LARGE;
    const int dtype = sizeof(T) == 4 ? AMPQ_F32 : AMPQ_BF16;
    const T* p = static_cast<const T*>(x);
    if (rows_aligned(x, ld, dtype))
        pack_kernel<T, FMT, true><<<(unsigned)blocks, kThreads, 0, st>>>(p, rows, (unsigned)cols, ld, groups, FastDiv(groups), codes, ld_codes, scales, ld_scales);
    else
        pack_kernel<T, FMT, false><<<(unsigned)blocks, kThreads, 0, st>>>(p, rows, (unsigned)cols, ld, groups, FastDiv(groups), codes, ld_codes, scales, ld_scales);
    return launched();
}

template <typename T, int FMT>
int launch_unpack(const unsigned char* codes, long long ld_codes, const unsigned char* scales, long long ld_scales, long long rows,
                  long long cols, void* out, long long ld, cudaStream_t st) {
    const unsigned groups = (unsigned)((cols + kGroup - 1) / kGroup);
    const long long blocks = (rows * groups + kGroupsPerBlock - 1) / kGroupsPerBlock;
    if (blocks > 0x7FFFFFFFLL) return AMPQ_ERR_TOO_LARGE;
    const int dtype = sizeof(T) == 4 ? AMPQ_F32 : AMPQ_BF16;
    T* p = static_cast<T*>(out);
    if (rows_aligned(out, ld, dtype))
        unpack_kernel<T, FMT, true><<<(unsigned)blocks, kThreads, 0, st>>>(codes, ld_codes, scales, ld_scales, rows, (unsigned)cols, groups, FastDiv(groups), p, ld);
    else
        unpack_kernel<T, FMT, false><<<(unsigned)blocks, kThreads, 0, st>>>(codes, ld_codes, scales, ld_scales, rows, (unsigned)cols, groups, FastDiv(groups), p, ld);
    return launched();
}

}  // namespace

int sm_count(int device) {
    constexpr int kMax = 64;
    static std::atomic<int> known[kMax];  // zero: not asked yet
    if (device >= 0 && device < kMax) {
        const int n = known[device].load(std::memory_order_relaxed);
        if (n > 0) return n;
    }
    int n = 0;
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, device) != cudaSuccess) {
        cudaGetLastError();
        return 0;
    }
    if (device >= 0 && device < kMax) known[device].store(n, std::memory_order_relaxed);
    return n;
}

template <typename T>
static void join_columns(const float* part, long long batches, int parts, long long cols, T* out, T* second, cudaStream_t st) {
    const unsigned bx = (unsigned)((cols + kJoinCols - 1) / kJoinCols);
    for (long long b0 = 0; b0 < batches; b0 += 65535) {  // the largest y extent of a grid
        const unsigned by = (unsigned)(batches - b0 < 65535 ? batches - b0 : 65535);
        join_columns_kernel<T><<<dim3(bx, by), dim3(kJoinCols, kJoinWays), 0, st>>>(part + b0 * parts * cols, parts, cols, out + b0 * cols, second);
    }
}

int launch_join_columns(const float* part, long long batches, int parts, long long cols, void* out, void* second, int dtype, cudaStream_t st) {
    if (batches <= 0 || cols <= 0) return AMPQ_OK;
    if (dtype == AMPQ_F32)
        join_columns(part, batches, parts, cols, static_cast<float*>(out), static_cast<float*>(second), st);
    else
        join_columns(part, batches, parts, cols, static_cast<__nv_bfloat16*>(out), static_cast<__nv_bfloat16*>(second), st);
    return launched();
}

int launch_ckpt_unpack(int dtype, int fmt, const unsigned char* codes, long long ld_codes, const unsigned char* scales, long long ld_scales,
                       long long rows, long long cols, void* out, long long ld, cudaStream_t st) {
    const bool e4 = fmt == AMPQ_FMT_E4M3;
    if (dtype == AMPQ_F32)
        return e4 ? launch_unpack<float, AMPQ_FMT_E4M3>(codes, ld_codes, scales, ld_scales, rows, cols, out, ld, st)
                  : launch_unpack<float, AMPQ_FMT_E5M2>(codes, ld_codes, scales, ld_scales, rows, cols, out, ld, st);
    return e4 ? launch_unpack<__nv_bfloat16, AMPQ_FMT_E4M3>(codes, ld_codes, scales, ld_scales, rows, cols, out, ld, st)
              : launch_unpack<__nv_bfloat16, AMPQ_FMT_E5M2>(codes, ld_codes, scales, ld_scales, rows, cols, out, ld, st);
}

}  // namespace ampq

using namespace ampq;

extern "C" {
#pragma GCC visibility push(default)

int ampq_ckpt_pack(int device, void* cuda_stream, int dtype, int fmt, const void* values, long long rows, long long cols, long long ld,
                   unsigned char* codes, long long ld_codes, unsigned char* scales, long long ld_scales) {
    if (!known_dtype(dtype) || !known_fp8(fmt)) return AMPQ_ERR_INVALID;
    int rc = check_matrix(values, rows, cols, ld, dtype);
    if (rc) return rc;
    rc = check_ckpt(codes, ld_codes, scales, ld_scales, rows, cols);
    if (rc) return rc;
    CkptDevice cur(device);
    if (cur.status) return cur.status;
    if (rows == 0 || cols == 0) return AMPQ_OK;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
    const bool e4 = fmt == AMPQ_FMT_E4M3;
    if (dtype == AMPQ_F32)
        return e4 ? launch_pack<float, AMPQ_FMT_E4M3>(values, rows, cols, ld, codes, ld_codes, scales, ld_scales, st)
                  : launch_pack<float, AMPQ_FMT_E5M2>(values, rows, cols, ld, codes, ld_codes, scales, ld_scales, st);
    return e4 ? launch_pack<__nv_bfloat16, AMPQ_FMT_E4M3>(values, rows, cols, ld, codes, ld_codes, scales, ld_scales, st)
              : launch_pack<__nv_bfloat16, AMPQ_FMT_E5M2>(values, rows, cols, ld, codes, ld_codes, scales, ld_scales, st);
}

int ampq_ckpt_unpack(int device, void* cuda_stream, int dtype, int fmt, const unsigned char* codes, long long ld_codes,
                     const unsigned char* scales, long long ld_scales, long long rows, long long cols, void* dev_out, long long ld) {
    if (!known_dtype(dtype) || !known_fp8(fmt)) return AMPQ_ERR_INVALID;
    int rc = check_matrix(dev_out, rows, cols, ld, dtype);
    if (rc) return rc;
    rc = check_ckpt(codes, ld_codes, scales, ld_scales, rows, cols);
    if (rc) return rc;
    CkptDevice cur(device);
    if (cur.status) return cur.status;
    if (rows == 0 || cols == 0) return AMPQ_OK;
    return launch_ckpt_unpack(dtype, fmt, codes, ld_codes, scales, ld_scales, rows, cols, dev_out, ld, reinterpret_cast<cudaStream_t>(cuda_stream));
}

#pragma GCC visibility pop
}  // extern "C"
