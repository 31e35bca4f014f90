// 8-bit checkpoints: the group format, and what the kernels that write or read
// it share (ampq_ckpt.cu, ampq_norm.cu, ampq_wgrad.cu).
//
// A row of `cols` elements is stored in groups of 32 consecutive columns.  A
// group has a power of two p = 2^e and one FP8 code per element:
//   e    = the smallest integer with fmax * 2^e >= max|x|, kept in
//          [kMinScaleExp, kMaxScaleExp]; 0 for a group of zeros,
//   code = RNE_sat(x * 2^-e); scale byte = e + 127.
// A power of two makes x * 2^-e exact (up to values far below the smallest
// code) and code * 2^e exactly representable in bf16: 4 or 3 significant bits,
// and the bounds on e keep the smallest code a normal bf16 (2^-9 * 2^-110 and
// 2^-16 * 2^-110) and the largest one finite.  The products of the weight
// gradient therefore see the stored values without a further rounding.
// A group that holds an Inf or a NaN cannot be stored: its scale byte is 255,
// its codes are 0, and it decodes to NaN as a whole.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "../../include/ampq.h"

namespace ampq {

constexpr int kGroup = 32;
constexpr int kMinScaleExp = -110;
constexpr unsigned kNanScale = 255;

template <int FMT>
struct Fp8;
template <>
struct Fp8<AMPQ_FMT_E4M3> {
    static constexpr int kTopExp = 8;         // fmax = 1.75 * 2^8
    static constexpr int kMaxScaleExp = 119;  // 1.75 * 2^127 is finite
};
template <>
struct Fp8<AMPQ_FMT_E5M2> {
    static constexpr int kTopExp = 15;  // fmax = 1.75 * 2^15
    static constexpr int kMaxScaleExp = 112;
};

// Scale byte of a group from the bits of max|x| (an integer maximum of the
// absolute values' bits, so an Inf or a NaN comes out on top).
template <int FMT>
__device__ __forceinline__ unsigned scale_byte(unsigned amax_bits) {
    if (amax_bits >= 0x7F800000u) return kNanScale;
    if (amax_bits == 0) return 127;
    int e = (int)(amax_bits >> 23) - 127 - Fp8<FMT>::kTopExp + ((amax_bits & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    e = max(kMinScaleExp, min(Fp8<FMT>::kMaxScaleExp, e));
    return (unsigned)(e + 127);
}

// 2^-e of a scale byte.  For the NaN byte any finite value: the caller stores codes 0.
__device__ __forceinline__ float inv_scale_of(unsigned byte) { return __uint_as_float((byte == kNanScale ? 127u : 254u - byte) << 23); }

// 2^e of a scale byte, NaN for the NaN byte.
__device__ __forceinline__ float scale_of(unsigned byte) { return __uint_as_float(byte == kNanScale ? 0x7FC00000u : byte << 23); }

// Eight codes -> their exact values, not yet multiplied by the group's scale.
template <int FMT>
__device__ __forceinline__ void decode8(uint2 c, float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const unsigned short h = (unsigned short)((i < 2 ? c.x : c.y) >> (16 * (i & 1)));
        unsigned r;
        if (FMT == AMPQ_FMT_E4M3)
            asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"(h));
        else
            asm("cvt.rn.f16x2.e5m2x2 %0, %1;" : "=r"(r) : "h"(h));
        const float2 f = __half22float2(*reinterpret_cast<__half2*>(&r));
        v[2 * i] = f.x;
        v[2 * i + 1] = f.y;
    }
}

// ---------------------------------------------------------------------------
// elements

__device__ __forceinline__ unsigned pack_bf16(float lo, float hi) {
    unsigned r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

__device__ __forceinline__ float load_elem(const float* p) { return __ldg(p); }
__device__ __forceinline__ float load_elem(const __nv_bfloat16* p) {
    return __uint_as_float((unsigned)__ldg(reinterpret_cast<const unsigned short*>(p)) << 16);
}
__device__ __forceinline__ void store_elem(float* p, float v) { *p = v; }
__device__ __forceinline__ void store_elem(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }

// The ends of rows, out of line: in line their predicated accesses are issued for
// every chunk.
template <typename T>
__device__ __noinline__ void store_some(T* p, int n, const unsigned* w) {
    for (int i = 0; i < n; ++i) {
        if (sizeof(T) == 4)
            reinterpret_cast<unsigned*>(p)[i] = w[i];
        else
            reinterpret_cast<unsigned short*>(p)[i] = (unsigned short)(w[i / 2] >> (16 * (i & 1)));
    }
}

// ---------------------------------------------------------------------------
// chunks: 32 consecutive bytes of a row, 16 bf16 or 8 fp32, one thread's share

template <typename T>
struct Chunk {
    static constexpr int kElems = 32 / (int)sizeof(T);
    static constexpr int kLanes = kGroup / kElems;  // neighbouring lanes that make a group
    float2 v[kElems / 2];

    __device__ __forceinline__ void zero() {
#pragma unroll
        for (int i = 0; i < kElems / 2; ++i) v[i] = make_float2(0.0f, 0.0f);
    }
    // From the eight words of the chunk.
    __device__ __forceinline__ void from_words(const unsigned (&w)[8]) {
        if (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < kElems / 2; ++i) v[i] = make_float2(__uint_as_float(w[(2 * i) & 7]), __uint_as_float(w[(2 * i + 1) & 7]));
        } else {
#pragma unroll
            for (int i = 0; i < kElems / 2; ++i) v[i] = make_float2(__uint_as_float(w[i & 7] << 16), __uint_as_float(w[i & 7] & 0xFFFF0000u));
        }
    }
    __device__ __forceinline__ void to_words(unsigned (&w)[8]) const {
        if (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = __float_as_uint(i & 1 ? v[(i / 2) % (kElems / 2)].y : v[(i / 2) % (kElems / 2)].x);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = pack_bf16(v[i % (kElems / 2)].x, v[i % (kElems / 2)].y);
        }
    }
    // The words of the first n (<= kElems) elements at p, zeros behind them.  Whole
    // chunks on 16-byte boundaries are two loads, others on 4-byte boundaries eight;
    // bf16 rows that start between two words take their pairs from neighbouring
    // words, of which the outermost two halves are read on their own.
    __device__ static __forceinline__ void load_words(const T* p, int n, unsigned (&w)[8]) {
        const unsigned off = (unsigned)(reinterpret_cast<uintptr_t>(p) & 15);
        if (n < kElems) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (sizeof(T) == 4) {
                    w[i] = i < n ? __ldg(reinterpret_cast<const unsigned*>(p) + i) : 0u;
                } else {
                    const unsigned short* h = reinterpret_cast<const unsigned short*>(p);
                    w[i] = 2 * i < n ? __ldg(h + 2 * i) : 0u;
                    if (2 * i + 1 < n) w[i] |= (unsigned)__ldg(h + 2 * i + 1) << 16;
                }
            }
        } else if (off == 0) {
            if ((reinterpret_cast<uintptr_t>(p) & 16) == 0) {
                asm volatile("ld.global.nc.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                             : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7])
                             : "l"(p));
            } else {
                const uint4 a = __ldg(reinterpret_cast<const uint4*>(p)), b = __ldg(reinterpret_cast<const uint4*>(p) + 1);
                w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w;
                w[4] = b.x; w[5] = b.y; w[6] = b.z; w[7] = b.w;
            }
        } else if ((off & 3) == 0) {
            const unsigned* q = reinterpret_cast<const unsigned*>(p);
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = __ldg(q + i);
        } else {  // bf16 only
            const unsigned short* h = reinterpret_cast<const unsigned short*>(p);
            const unsigned* q = reinterpret_cast<const unsigned*>(h + 1);
            unsigned u = (unsigned)__ldg(h) << 16;
#pragma unroll
            for (int i = 0; i < 7; ++i) {
                const unsigned next = __ldg(q + i);
                w[i] = __funnelshift_r(u, next, 16);
                u = next;
            }
            w[7] = __funnelshift_r(u, (unsigned)__ldg(h + 15), 16);
        }
    }
    __device__ __forceinline__ void load(const T* p, int n) {
        unsigned w[8];
        load_words(p, n, w);
        from_words(w);
    }
    __device__ __forceinline__ void store(T* p, int n) const {
        const unsigned off = (unsigned)(reinterpret_cast<uintptr_t>(p) & 15);
        unsigned w[8];
        to_words(w);
        if (n < kElems) {
            unsigned some[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) some[i] = w[i];
            store_some(p, n, some);
            return;
        }
        if (off == 0) {
            if ((reinterpret_cast<uintptr_t>(p) & 16) == 0) {
                asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]),
                             "r"(w[5]), "r"(w[6]), "r"(w[7])
                             : "memory");
            } else {
                reinterpret_cast<uint4*>(p)[0] = make_uint4(w[0], w[1], w[2], w[3]);
                reinterpret_cast<uint4*>(p)[1] = make_uint4(w[4], w[5], w[6], w[7]);
            }
        } else if ((off & 3) == 0) {
#pragma unroll
            for (int i = 0; i < 8; ++i) reinterpret_cast<unsigned*>(p)[i] = w[i];
        } else {
            unsigned short* h = reinterpret_cast<unsigned short*>(p);
            unsigned* q = reinterpret_cast<unsigned*>(h + 1);
            h[0] = (unsigned short)w[0];
#pragma unroll
            for (int i = 0; i < 7; ++i) q[i] = __funnelshift_r(w[i], w[i + 1], 16);
            h[15] = (unsigned short)(w[7] >> 16);
        }
    }
    // Bits of the largest absolute value of the group this chunk is part of; a NaN
    // comes out on top.  All lanes of the warp call it.
    __device__ __forceinline__ unsigned group_amax() const {
        float m = fabsf(v[0].x);
#pragma unroll
        for (int i = 0; i < kElems / 2; ++i) asm("max.NaN.abs.f32 %0, %0, %1, %2;" : "+f"(m) : "f"(v[i].x), "f"(v[i].y));
#pragma unroll
        for (int o = 1; o < kLanes; o <<= 1) asm("max.NaN.f32 %0, %0, %1;" : "+f"(m) : "f"(__shfl_xor_sync(0xFFFFFFFFu, m, o)));
        return __float_as_uint(m) & 0x7FFFFFFFu;
    }
    // Codes of the chunk under a scale byte, element 0 in the lowest byte.
    template <int FMT>
    __device__ __forceinline__ void encode(unsigned byte, unsigned (&c)[kElems / 4]) const {
        const float inv = inv_scale_of(byte);
#pragma unroll
        for (int i = 0; i < kElems / 4; ++i) {
            const float2 a = __fmul2_rn(v[2 * i], make_float2(inv, inv)), b = __fmul2_rn(v[2 * i + 1], make_float2(inv, inv));
            unsigned short lo, hi;
            if (FMT == AMPQ_FMT_E4M3) {
                asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(a.y), "f"(a.x));
                asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(b.y), "f"(b.x));
            } else {
                asm("cvt.rn.satfinite.e5m2x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(a.y), "f"(a.x));
                asm("cvt.rn.satfinite.e5m2x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(b.y), "f"(b.x));
            }
            c[i] = byte == kNanScale ? 0u : (unsigned)lo | (unsigned)hi << 16;
        }
    }
    // The chunk's codes, not yet multiplied by the scale.
    template <int FMT>
    __device__ __forceinline__ void decode(const unsigned (&c)[kElems / 4]) {
#pragma unroll
        for (int i = 0; i < kElems / 2; ++i) {
            const unsigned short h = (unsigned short)(c[i / 2] >> (16 * (i & 1)));
            unsigned r;
            if (FMT == AMPQ_FMT_E4M3)
                asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"(h));
            else
                asm("cvt.rn.f16x2.e5m2x2 %0, %1;" : "=r"(r) : "h"(h));
            v[i] = __half22float2(*reinterpret_cast<__half2*>(&r));
        }
    }
    __device__ __forceinline__ void scale(float p) {
#pragma unroll
        for (int i = 0; i < kElems / 2; ++i) v[i] = __fmul2_rn(v[i], make_float2(p, p));
    }
};

template <int N>
__device__ __forceinline__ void load_codes(const unsigned char* p, unsigned (&c)[N]) {
    if (N == 4) {
        const uint4 q = __ldg(reinterpret_cast<const uint4*>(p));
        c[0] = q.x; c[1] = q.y; c[2 % N] = q.z; c[3 % N] = q.w;
    } else {
        const uint2 q = __ldg(reinterpret_cast<const uint2*>(p));
        c[0] = q.x; c[1] = q.y;
    }
}
template <int N>
__device__ __forceinline__ void store_codes(unsigned char* p, const unsigned (&c)[N]) {
    if (N == 4)
        *reinterpret_cast<uint4*>(p) = make_uint4(c[0], c[1], c[2 % N], c[3 % N]);
    else
        *reinterpret_cast<uint2*>(p) = make_uint2(c[0], c[1]);
}

// ---------------------------------------------------------------------------
// host side

struct CkptDevice {  // makes `device` current for the life of the object
    int prev = -1;
    int status = AMPQ_OK;
    explicit CkptDevice(int dev) {
        int n = 0;
        if (cudaGetDeviceCount(&n) != cudaSuccess || n <= 0) {
            cudaGetLastError();
            status = AMPQ_ERR_CUDA;
            return;
        }
        if (dev < 0 || dev >= n) {
            status = AMPQ_ERR_INVALID;
            return;
        }
        if (cudaGetDevice(&prev) != cudaSuccess) {
            cudaGetLastError();
            prev = -1;
            status = AMPQ_ERR_CUDA;
            return;
        }
        if (prev == dev)
            prev = -1;
        else if (cudaSetDevice(dev) != cudaSuccess) {
            cudaGetLastError();
            status = AMPQ_ERR_CUDA;
        }
    }
    ~CkptDevice() {
        if (prev >= 0) cudaSetDevice(prev);
    }
};

inline int launched() {
    if (cudaGetLastError() != cudaSuccess) return AMPQ_ERR_CUDA;
    return AMPQ_OK;
}

inline bool aligned_to(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }
inline size_t elem_bytes(int dtype) { return dtype == AMPQ_F32 ? 4 : 2; }
inline bool known_dtype(int dtype) { return dtype == AMPQ_F32 || dtype == AMPQ_BF16; }
inline bool known_fp8(int fmt) { return fmt == AMPQ_FMT_E4M3 || fmt == AMPQ_FMT_E5M2; }
// rows of ld elements can be read 16 bytes at a time
inline bool rows_aligned(const void* p, long long ld, int dtype) { return aligned_to(p, 16) && (ld * (long long)elem_bytes(dtype)) % 16 == 0; }

constexpr long long kMaxRows = 0x7FFFFFFFLL;
constexpr long long kMaxCols = 0x3FFFFFFFLL;

// Arguments of a matrix whose rows lie ld elements apart.
inline int check_matrix(const void* p, long long rows, long long cols, long long ld, int dtype) {
    if (rows < 0 || cols < 0 || ld < cols) return AMPQ_ERR_INVALID;
    if (rows > 0 && cols > 0 && !p) return AMPQ_ERR_INVALID;
    if (rows > kMaxRows || cols > kMaxCols || ld > (1LL << 40)) return AMPQ_ERR_TOO_LARGE;
    if (!aligned_to(p, elem_bytes(dtype))) return AMPQ_ERR_ALIGN;
    return AMPQ_OK;
}

// Arguments of a checkpoint of rows x cols elements.
inline int check_ckpt(const unsigned char* codes, long long ld_codes, const unsigned char* scales, long long ld_scales, long long rows,
                      long long cols) {
    const long long groups = (cols + kGroup - 1) / kGroup;
    if (ld_codes < groups * kGroup || ld_scales < groups) return AMPQ_ERR_INVALID;
    if (rows > 0 && cols > 0 && (!codes || !scales)) return AMPQ_ERR_INVALID;
    if (ld_codes > (1LL << 40) || ld_scales > (1LL << 40)) return AMPQ_ERR_TOO_LARGE;
    if (ld_codes % 16 || !aligned_to(codes, 16)) return AMPQ_ERR_ALIGN;
    return AMPQ_OK;
}

int sm_count(int device);  // multiprocessors of a device, 0 on error

// ampq_ckpt_unpack on a stream of the current device, arguments checked.
int launch_ckpt_unpack(int dtype, int fmt, const unsigned char* codes, long long ld_codes, const unsigned char* scales, long long ld_scales,
                       long long rows, long long cols, void* out, long long ld, cudaStream_t st);

// Sums `parts` fp32 partial rows of `cols` columns, `pitch` apart, in a fixed order
// and stores them in `dtype`: out[b][c] = sum_p part[b][p][c], `batches` of them.  With
// `second` (two batches) batch 1 goes there.
int launch_join_columns(const float* part, long long batches, int parts, long long cols, long long pitch, void* out, void* second, int dtype, cudaStream_t st);

}  // namespace ampq
