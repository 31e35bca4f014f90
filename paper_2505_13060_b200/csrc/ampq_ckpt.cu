// Writing and reading 8-bit checkpoints (include/ampq.h: ampq_ckpt_pack,
// ampq_ckpt_unpack), and the joining of partial column sums.
#include "ampq_ckpt.h"

#include <atomic>

namespace ampq {
namespace {

constexpr int kThreads = 256;
constexpr int kUnroll = 4;  // chunks a thread has in flight

// Groups of one block: 32 bytes of x to a thread.
template <typename T>
constexpr int kGroupsPerBlock = kThreads / Chunk<T>::kLanes * kUnroll;

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

// The group that a thread's chunk belongs to: groups are numbered row by row and
// a block takes kGroupsPerBlock of them.  The 64-bit division is done once per
// block.
struct Place {
    long long row;
    unsigned group;
};

struct BlockStart {
    long long row0;
    unsigned group0;
    __device__ __forceinline__ BlockStart(unsigned groups, int per_block) {
        const long long first = (long long)blockIdx.x * per_block;
        row0 = first / groups;
        group0 = (unsigned)(first - row0 * groups);
    }
    __device__ __forceinline__ Place at(unsigned local, unsigned groups, const FastDiv& div) const {
        const unsigned n = group0 + local;
        const unsigned q = div(n);
        return Place{row0 + q, n - q * groups};
    }
};

// One read of x, one write of codes and scale bytes: bound by HBM (8192 x 28672
// bf16 105 us, 6.8 TB/s).  A thread holds 32 bytes of a row; two (bf16) or four
// (fp32) lanes make a group, so the group's maximum is one or two shuffles.  With 16
// bytes to a thread the address arithmetic and the conversions of twice the threads
// took as long as the memory (137 us).
template <typename T, int FMT>
__global__ void __launch_bounds__(kThreads) pack_kernel(const T* __restrict__ x, long long rows, unsigned cols, long long ld,
                                                        unsigned groups, FastDiv div, unsigned char* __restrict__ codes, long long ld_codes,
                                                        unsigned char* __restrict__ scales, long long ld_scales) {
    using K = Chunk<T>;
    const BlockStart start(groups, kGroupsPerBlock<T>);
    unsigned w[kUnroll][8];
    Place pl[kUnroll];
    const unsigned part = threadIdx.x % K::kLanes;
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
        pl[u] = start.at((u * kThreads + threadIdx.x) / K::kLanes, groups, div);
        const int c0 = (int)(pl[u].group * kGroup + part * K::kElems);
        const int n = pl[u].row < rows ? min(K::kElems, (int)cols - c0) : 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) w[u][i] = 0;
        if (n > 0) K::load_words(x + pl[u].row * ld + c0, n, w[u]);
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
        K k;
        k.from_words(w[u]);
        const unsigned byte = scale_byte<FMT>(k.group_amax());
        unsigned c[K::kElems / 4];
        k.template encode<FMT>(byte, c);
        if (pl[u].row < rows) {
            store_codes(codes + pl[u].row * ld_codes + pl[u].group * kGroup + part * K::kElems, c);
            if (part == 0) scales[pl[u].row * ld_scales + pl[u].group] = (unsigned char)byte;
        }
    }
}

// The way back, bound by HBM too: 8192 x 8192 to bf16 34 us (6.0 TB/s).
template <typename T, int FMT>
__global__ void __launch_bounds__(kThreads) unpack_kernel(const unsigned char* __restrict__ codes, long long ld_codes,
                                                          const unsigned char* __restrict__ scales, long long ld_scales, long long rows,
                                                          unsigned cols, unsigned groups, FastDiv div, T* __restrict__ out, long long ld) {
    using K = Chunk<T>;
    const BlockStart start(groups, kGroupsPerBlock<T>);
    unsigned c[kUnroll][K::kElems / 4];
    unsigned byte[kUnroll];
    Place pl[kUnroll];
    const unsigned part = threadIdx.x % K::kLanes;
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
        pl[u] = start.at((u * kThreads + threadIdx.x) / K::kLanes, groups, div);
        byte[u] = 127;
        if (pl[u].row < rows) {
            load_codes(codes + pl[u].row * ld_codes + pl[u].group * kGroup + part * K::kElems, c[u]);
            byte[u] = __ldg(scales + pl[u].row * ld_scales + pl[u].group);
        }
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
        const int c0 = (int)(pl[u].group * kGroup + part * K::kElems);
        const int n = pl[u].row < rows ? min(K::kElems, (int)cols - c0) : 0;
        if (n <= 0) continue;
        K k;
        k.template decode<FMT>(c[u]);
        k.scale(scale_of(byte[u]));
        k.store(out + pl[u].row * ld + c0, n);
    }
}

// ---------------------------------------------------------------------------
// joining column sums

// A block joins 32 columns, 32 parts at a time (148 parts of 8192 columns: 4.4 us).
constexpr int kJoinCols = 32, kJoinWays = 32;

template <typename T>
__global__ void __launch_bounds__(kJoinCols * kJoinWays) join_columns_kernel(const float* __restrict__ part, int parts, long long cols, long long pitch, T* __restrict__ out,
                                                                             T* __restrict__ second) {
    __shared__ float sums[kJoinWays][kJoinCols];
    const long long c = (long long)blockIdx.x * kJoinCols + threadIdx.x;
    const long long batch = blockIdx.y;
    float s = 0.0f;
    if (c < cols)
#pragma unroll 5
        for (int p = threadIdx.y; p < parts; p += kJoinWays) s += __ldg(part + (batch * parts + p) * pitch + c);
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
    const long long blocks = (rows * groups + kGroupsPerBlock<T> - 1) / kGroupsPerBlock<T>;
    if (blocks > 0x7FFFFFFFLL) return AMPQ_ERR_TOO_LARGE;
    pack_kernel<T, FMT><<<(unsigned)blocks, kThreads, 0, st>>>(static_cast<const T*>(x), rows, (unsigned)cols, ld, groups, FastDiv(groups), codes, ld_codes,
                                                               scales, ld_scales);
    return launched();
}

template <typename T, int FMT>
int launch_unpack(const unsigned char* codes, long long ld_codes, const unsigned char* scales, long long ld_scales, long long rows,
                  long long cols, void* out, long long ld, cudaStream_t st) {
    const unsigned groups = (unsigned)((cols + kGroup - 1) / kGroup);
    const long long blocks = (rows * groups + kGroupsPerBlock<T> - 1) / kGroupsPerBlock<T>;
    if (blocks > 0x7FFFFFFFLL) return AMPQ_ERR_TOO_LARGE;
    unpack_kernel<T, FMT><<<(unsigned)blocks, kThreads, 0, st>>>(codes, ld_codes, scales, ld_scales, rows, (unsigned)cols, groups, FastDiv(groups),
                                                                 static_cast<T*>(out), ld);
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
static void join_columns(const float* part, long long batches, int parts, long long cols, long long pitch, T* out, T* second, cudaStream_t st) {
    const unsigned bx = (unsigned)((cols + kJoinCols - 1) / kJoinCols);
    for (long long b0 = 0; b0 < batches; b0 += 65535) {  // the largest y extent of a grid
        const unsigned by = (unsigned)(batches - b0 < 65535 ? batches - b0 : 65535);
        join_columns_kernel<T><<<dim3(bx, by), dim3(kJoinCols, kJoinWays), 0, st>>>(part + b0 * parts * pitch, parts, cols, pitch, out + b0 * cols, second);
    }
}

int launch_join_columns(const float* part, long long batches, int parts, long long cols, long long pitch, void* out, void* second, int dtype, cudaStream_t st) {
    if (batches <= 0 || cols <= 0) return AMPQ_OK;
    if (dtype == AMPQ_F32)
        join_columns(part, batches, parts, cols, pitch, static_cast<float*>(out), static_cast<float*>(second), st);
    else
        join_columns(part, batches, parts, cols, pitch, static_cast<__nv_bfloat16*>(out), static_cast<__nv_bfloat16*>(second), st);
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
