// Norms of queries and keys for each head with the position rotation in the same
// pass, forward and backward (include/ampq.h: ampq_head_norm_forward,
// ampq_head_norm_backward).
//
//   r = 1 / sqrt(mean_c x^2 + eps), n = x r w, (y_i, y_j) = (n_i cos - n_j sin, n_j cos + n_i sin)
// backward, with t the gradient turned back, h = x r and u = t w:
//   gx = r (u - h mean_c(u h)), gw = sum over tokens and heads of t h
//
// Layout.  A thread holds two vectors of V columns that need no other's for the
// rotation: columns j V and rot / 2 + j V, which are turned into one another, and
// behind them the two halves of the columns that are not turned; where pairs are
// neighbours, j V and cols / 2 + j V.  Either way neighbouring lanes have neighbouring
// vectors.  A head takes the smallest power of two of lanes that holds it, a warp
// several heads at once; the sum over a head's columns is a few shuffles.
#include "ampq_decoder.h"

#include <cmath>

namespace ampq {
namespace {

constexpr int kHeadCols = AMPQ_HEAD_MAX_COLS;
// Threads of a CTA, CTAs that share an SM, and the steps that a warp works on together.
// The shuffles, the root and the loads of a step are a chain of latencies: two steps
// side by side fill it better than more warps would.  Measured on 2 x 4096 tokens of 64 + 8 heads of 128 columns (one
// step at a time, the same with six CTAs an SM, two together): forward bf16 with a
// checkpoint 74, 80 and 68 us, without 59, 58 and 53 us, fp32 125, 129 and 111 us.
// Backward (one step, two): fp32 124 and 115 us, but bf16, whose sums and factors
// leave no room, from 8 bits 78 and 119 us, from the input 80 and 110 us.  Three CTAs an
// SM instead of four: forward bf16 74 and 59 us, fp32 126 us, backward 85 us and fp32
// 127 us.  At four the bf16 backward kernels of neighbouring pairs that read a checkpoint
// spill 32 to 56 bytes and are no slower for it (84 us, at three 85).  Most backward
// kernels with vectors of two elements spill at three (up to 80 bytes); not tried with two.
constexpr int kForwardThreads = 128, kBackwardThreads = 128, kMostCtas = 4, kForwardTogether = 2;
template <int V>
constexpr int kCtas = V >= 4 ? kMostCtas : 3;  // small vectors come through registers
template <typename T>
constexpr int kBackwardTogether = sizeof(T) == 4 ? 2 : 1;
// Steps of a run.  The same size, runs of 1, 2, 4 and 8: forward bf16 with a checkpoint 121,
// 80, 69 and 70 us, fp32 197, 134, 112 and 132, backward from 8 bits 106, 87, 79 and 78, fp32 180, 127, 116 and 129.
constexpr int kMaxRun = 4;

struct Side {  // queries or keys
    const void *x, *gy, *w;
    void* out;  // y or gx
    float* rstd;
    unsigned char *codes, *scales;
    long long x_batch, x_token, x_head, gy_batch, gy_token, gy_head, out_batch, out_token, out_head, ld_codes, ld_scales;
    int heads;
};

struct HeadArgs {
    Side side[2];
    const float *cos, *sin;
    const void* positions;
    float* part;
    long long position_batch;
    unsigned rows, tokens;  // rows: batch * tokens
    long long angles;
    int cols, half, lanes, vectors, pitch;  // half: rot / 2; vectors: pairs of vectors of a head
    int run[2], runs[2];                    // queries and keys: steps of a run of heads, runs of a token,
    int ctas[2];                            // and CTAs
    float eps, inv_cols;
    bool param_bf16, wide, e4m3, sums;
    bool lane_groups;  // a checkpoint's groups are whole vectors of neighbouring lanes
};

// A kernel's format: none, one of the two, or the one that the arguments say.
constexpr int kEither = 3;

template <int FMT>
__device__ __forceinline__ unsigned group_byte(bool e4m3, unsigned amax) {
    if (FMT == AMPQ_FMT_E4M3 || (FMT == kEither && e4m3)) return scale_byte<AMPQ_FMT_E4M3>(amax);
    return scale_byte<AMPQ_FMT_E5M2>(amax);
}

// V neighbouring elements of T as they lie in memory, aligned to their size, and as
// pairs in fp32 (with V = 1 half a pair).
template <int V>
constexpr int kPairs = (V + 1) / 2;

template <typename T, int V>
struct Raw {
    static constexpr int B = V * (int)sizeof(T), W = (B + 3) / 4;
    unsigned w[W];
    __device__ __forceinline__ void load(const T* p) {
        if constexpr (B == 16) {
            const uint4 q = __ldg(reinterpret_cast<const uint4*>(p));
            w[0] = q.x; w[1] = q.y; w[2] = q.z; w[3] = q.w;
        } else if constexpr (B == 8) {
            const uint2 q = __ldg(reinterpret_cast<const uint2*>(p));
            w[0] = q.x; w[1] = q.y;
        } else if constexpr (B == 4) {
            w[0] = __ldg(reinterpret_cast<const unsigned*>(p));
        } else {
            w[0] = __ldg(reinterpret_cast<const unsigned short*>(p));
        }
    }
    __device__ __forceinline__ void take(const void* smem) {
        if constexpr (B == 16) {
            const uint4 q = *static_cast<const uint4*>(smem);
            w[0] = q.x; w[1] = q.y; w[2] = q.z; w[3] = q.w;
        }
    }
    __device__ __forceinline__ void zero() {
#pragma unroll
        for (int i = 0; i < W; ++i) w[i] = 0;
    }
    __device__ __forceinline__ void unpack(float2 (&v)[kPairs<V>]) const {
#pragma unroll
        for (int i = 0; i < kPairs<V>; ++i) {
            if constexpr (sizeof(T) == 4)
                v[i] = make_float2(__uint_as_float(w[2 * i]), V == 1 ? 0.0f : __uint_as_float(w[(2 * i + 1) % W]));
            else
                v[i] = make_float2(__uint_as_float(w[i] << 16), V == 1 ? 0.0f : __uint_as_float(w[i] & 0xFFFF0000u));
        }
    }
};

// Vectors of 16 bytes come by asynchronous copies into shared memory, each thread's to
// its own places, while the step before is worked on; smaller ones into registers.
template <typename T, int V>
constexpr bool kAsync = V * sizeof(T) == 16;

template <int BYTES>
__device__ __forceinline__ void copy_async(void* smem, const void* p) {
    const unsigned at = (unsigned)__cvta_generic_to_shared(smem);
    if constexpr (BYTES == 16)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(at), "l"(p) : "memory");
    else
        asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(at), "l"(p), "n"(BYTES) : "memory");
}
__device__ __forceinline__ void commit_async() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT>
__device__ __forceinline__ void wait_async() {
    asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory");
}

template <typename T, int V>
__device__ __forceinline__ void store_vec(T* p, const float2 (&v)[kPairs<V>]) {
    constexpr int B = V * (int)sizeof(T);
    if constexpr (V == 1)
        store_elem(p, v[0].x);
    else if constexpr (sizeof(T) == 4 && B == 16)
        *reinterpret_cast<float4*>(p) = make_float4(v[0].x, v[0].y, v[1].x, v[1].y);
    else if constexpr (sizeof(T) == 4)
        *reinterpret_cast<float2*>(p) = v[0];
    else if constexpr (B == 16)
        *reinterpret_cast<uint4*>(p) = make_uint4(pack_bf16(v[0].x, v[0].y), pack_bf16(v[1].x, v[1].y), pack_bf16(v[2].x, v[2].y), pack_bf16(v[3].x, v[3].y));
    else if constexpr (B == 8)
        *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16(v[0].x, v[0].y), pack_bf16(v[1].x, v[1].y));
    else
        *reinterpret_cast<unsigned*>(p) = pack_bf16(v[0].x, v[0].y);
}

// V codes of FP8, element 0 in the lowest byte.
template <int V>
struct RawCodes {
    uint2 c;
    __device__ __forceinline__ void load(const unsigned char* p) {
        c = make_uint2(0, 0);
        if constexpr (V == 8) c = __ldg(reinterpret_cast<const uint2*>(p));
        if constexpr (V == 4) c.x = __ldg(reinterpret_cast<const unsigned*>(p));
        if constexpr (V == 2) c.x = __ldg(reinterpret_cast<const unsigned short*>(p));
        if constexpr (V == 1) c.x = __ldg(p);
    }
    template <int FMT>
    __device__ __forceinline__ void unpack(bool e4m3, float scale, float2 (&v)[kPairs<V>]) const {
        float f[8];
        if (FMT == AMPQ_FMT_E4M3 || (FMT == kEither && e4m3))
            decode8<AMPQ_FMT_E4M3>(c, f);
        else
            decode8<AMPQ_FMT_E5M2>(c, f);
#pragma unroll
        for (int i = 0; i < kPairs<V>; ++i) v[i] = __fmul2_rn(make_float2(f[2 * i], V == 1 ? 0.0f : f[2 * i + 1]), make_float2(scale, scale));
    }
};

template <int V, int FMT>
__device__ __forceinline__ void store_code_vec(unsigned char* p, bool e4m3, unsigned byte, const float2 (&v)[kPairs<V>]) {
    const float inv = inv_scale_of(byte);
    unsigned c[kPairs<V>];
#pragma unroll
    for (int i = 0; i < kPairs<V>; ++i) {
        const float2 f = __fmul2_rn(v[i], make_float2(inv, inv));
        unsigned short h;
        if (FMT == AMPQ_FMT_E4M3 || (FMT == kEither && e4m3))
            asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(h) : "f"(f.y), "f"(f.x));
        else
            asm("cvt.rn.satfinite.e5m2x2.f32 %0, %1, %2;" : "=h"(h) : "f"(f.y), "f"(f.x));
        c[i] = h;
    }
    const unsigned keep = byte == kNanScale ? 0u : 0xFFFFFFFFu;
    if constexpr (V == 8) *reinterpret_cast<uint2*>(p) = make_uint2((c[0] | c[1] << 16) & keep, (c[2] | c[3] << 16) & keep);
    if constexpr (V == 4) *reinterpret_cast<unsigned*>(p) = (c[0] | c[1] << 16) & keep;
    if constexpr (V == 2) *reinterpret_cast<unsigned short*>(p) = (unsigned short)(c[0] & keep);
    if constexpr (V == 1) *p = (unsigned char)(c[0] & keep);
}

// Columns of a thread's j-th two vectors, and the first angle of each (-1: not turned):
// V of them, the same ones for both, or V / 2 for each where pairs are neighbours.
struct Columns {
    int col[2], angle[2];
};
template <int V, bool NEXT>
__device__ __forceinline__ Columns columns_of(int cols, int half, int j) {
    if (NEXT && V > 1) {
        const int a = V * j, b = cols / 2 + V * j;
        return Columns{{a, b}, {a < 2 * half ? a / 2 : -1, b < 2 * half ? b / 2 : -1}};
    }
    const int turned = half / V;  // pairs of vectors that are turned
    const int angle = j < turned ? V * j : -1;
    if (NEXT) return Columns{{2 * j, 2 * j + 1}, {angle, angle}};
    if (j < turned) return Columns{{V * j, half + V * j}, {angle, angle}};
    const int rest = (cols - 2 * half) / 2, at = 2 * half + V * (j - turned);
    return Columns{{at, at + rest}, {-1, -1}};
}

// The elements that those of vector m are turned with, where the pairs are neighbours
// (each float2 is one) and where they are halves of the head.
template <int V, bool NEXT>
__device__ __forceinline__ float2 partner(const float2 (&v)[2][kPairs<V>], int m, int i) {
    if (NEXT && V > 1) return make_float2(v[m][i].y, v[m][i].x);
    return v[1 - m][i];
}

// sum + partner * factor.  Neighbours are multiplied one by one: as a pair they would
// have to change places first.
template <int V, bool NEXT>
__device__ __forceinline__ float2 turn_with(const float2 (&v)[2][kPairs<V>], int m, int i, float2 factor, float2 sum) {
    if (NEXT && V > 1) return make_float2(fmaf(v[m][i].y, factor.x, sum.x), fmaf(v[m][i].x, factor.y, sum.y));
    return __ffma2_rn(v[1 - m][i], factor, sum);
}

// N values of a table, the first one at a multiple of N of a row whose length is one too.
template <int N>
__device__ __forceinline__ void load_row(const float* p, bool known, float (&v)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = NAN;
    if (!known) return;
    if constexpr (N % 4 == 0) {
#pragma unroll
        for (int i = 0; i < N; i += 4) {
            const float4 f = __ldg(reinterpret_cast<const float4*>(p + i));
            v[i] = f.x; v[i + 1] = f.y; v[i + 2] = f.z; v[i + 3] = f.w;
        }
    } else if constexpr (N == 2) {
        const float2 f = __ldg(reinterpret_cast<const float2*>(p));
        v[0] = f.x; v[1] = f.y;
    } else {
        v[0] = __ldg(p);
    }
}

// Cosines and sines of a token for a thread's columns, as factors of its elements:
// turned value = own * c + partner * s, where the columns are turned.  `back` turns the
// other way.  A position outside the table has NaN.
template <int V, bool NEXT>
__device__ __forceinline__ void load_angles(const HeadArgs& p, int half, long long position, const int (&angle)[2], bool back, float2 (&c)[2][kPairs<V>],
                                            float2 (&s)[2][kPairs<V>]) {
    const bool known = position >= 0 && position < p.angles;
    if constexpr (NEXT && V > 1) {
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            if (angle[m] < 0) continue;
            float cv[V / 2], sv[V / 2];
            load_row<V / 2>(p.cos + position * half + angle[m], known, cv);
            load_row<V / 2>(p.sin + position * half + angle[m], known, sv);
#pragma unroll
            for (int i = 0; i < V / 2; ++i) {
                c[m][i] = make_float2(cv[i], cv[i]);
                s[m][i] = back ? make_float2(sv[i], -sv[i]) : make_float2(-sv[i], sv[i]);
            }
        }
    } else if (angle[0] >= 0) {
        float cv[V], sv[V];
        load_row<V>(p.cos + position * half + angle[0], known, cv);
        load_row<V>(p.sin + position * half + angle[0], known, sv);
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int i = 0; i < kPairs<V>; ++i) {
                const float2 y = make_float2(sv[2 * i], sv[(2 * i + 1) % V]);
                c[m][i] = make_float2(cv[2 * i], cv[(2 * i + 1) % V]);
                s[m][i] = (m == 0) != back ? make_float2(-y.x, -y.y) : y;
            }
    }
}

// The weights of both sides in shared memory, in fp32.
__device__ __forceinline__ void stage_weights(const HeadArgs& a, float (*w)[kHeadCols]) {
    for (int k = threadIdx.x; k < 2 * a.cols; k += (int)blockDim.x) {
        const int side = k >= a.cols, c = k - side * a.cols;
        w[side][c] = a.side[side].w ? load_param(a.side[side].w, c, a.param_bf16) : 1.0f;
    }
    __syncthreads();
}
template <int V>
__device__ __forceinline__ void take_weights(const float* w, float2 (&v)[kPairs<V>]) {
    if constexpr (V == 1) {
        v[0] = make_float2(w[0], 0.0f);
    } else if constexpr (V == 2) {
        v[0] = make_float2(w[0], w[1]);
    } else {
#pragma unroll
        for (int i = 0; i < V; i += 4) {
            const float4 f = *reinterpret_cast<const float4*>(w + i);  // columns of a vector begin at a multiple of V
            v[i / 2] = make_float2(f.x, f.y);
            v[i / 2 + 1] = make_float2(f.z, f.w);
        }
    }
}

// Sums over the `lanes` neighbouring lanes of a head, of U heads side by side.
template <int U, int COLS>
__device__ __forceinline__ void head_sums(float (&s)[U], int lanes) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        if (COLS && o >= lanes) continue;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const float t = __shfl_xor_sync(0xFFFFFFFFu, s[u], o);
            s[u] = o < lanes ? s[u] + t : s[u];
        }
    }
}

// 1 / sqrt(v), the hardware's approximation improved by one of Newton's steps, to
// within an ulp; 0 of infinity and infinity of 0.
__device__ __forceinline__ float inverse_root(float v) {
    float r;
    asm("rsqrt.approx.f32 %0, %1;" : "=f"(r) : "f"(v));
    const float e = fmaf(-v * r, r, 1.0f);  // NaN where r is not a number that can be improved
    const float better = fmaf(0.5f * r, e, r);
    return better == better ? better : r;
}

// A warp's share: one run of heads (of the queries or of the keys) of every
// `stride`-th token, so that what goes with the columns is set up once.  The grid's
// first CTAs have queries, the others keys, by how much work there is of each.  It
// walks over its rows, whose batch and token are kept up to date.
struct Share {
    int side, head0, steps;  // head0: the first head of this lane
    unsigned row, stride, batch, token;
    bool some;
    __device__ __forceinline__ Share(const HeadArgs& a, unsigned warp, unsigned warps, int per, int slot) {
        side = (int)blockIdx.x >= a.ctas[0];
        warp += (blockIdx.x - (side ? a.ctas[0] : 0)) * warps;
        const unsigned runs = (unsigned)a.runs[side];
        stride = (unsigned)a.ctas[side] * warps / runs;
        row = warp / runs;
        some = row < stride && row < a.rows;  // the last few warps may have none
        const int step0 = (int)(warp % runs) * a.run[side];
        head0 = step0 * per + slot;
        steps = min(a.run[side], (a.side[side].heads + per - 1) / per - step0);
        batch = row / a.tokens;
        token = row - batch * a.tokens;
    }
    __device__ __forceinline__ bool last(const HeadArgs& a) const { return row + stride >= a.rows; }  // rows < 2^31
    __device__ __forceinline__ void advance(const HeadArgs& a) {
        row += stride;
        token += stride;
        if (token >= a.tokens) {
            const unsigned more = token / a.tokens;
            batch += more;
            token -= more * a.tokens;
        }
    }
    __device__ __forceinline__ long long position(const HeadArgs& a) const {
        return a.positions ? load_index(a.positions, (long long)batch * a.position_batch + token, a.wide) : (long long)token;
    }
    template <typename T>
    __device__ __forceinline__ T* at(T* p, long long by_batch, long long by_token, long long by_head) const {
        return p + ((long long)batch * by_batch + (long long)token * by_token + (long long)head0 * by_head);
    }
};

// ---------------------------------------------------------------------------

// Bound by HBM and, with a checkpoint, by the warps' latencies: 2 x 4096 tokens of
// 64 + 8 heads of 128 columns, bf16, take 53 us (5.8 TB/s) and 68 us with the
// checkpoint (5.7 TB/s), fp32 111 us (6.2 TB/s).
// COLS: heads of so many columns, all of them turned, or 0 for any.  What depends on
// the columns alone is then known to the compiler (a third of the instructions).
template <typename T, int V, int NV, bool NEXT, int FMT, int COLS>
__global__ void __launch_bounds__(kForwardThreads, kCtas<V>) head_norm_forward_kernel(const HeadArgs a) {
    constexpr int kThreads = kForwardThreads, kWarps = kThreads / 32;
    constexpr int P = kPairs<V>;
    constexpr bool ASYNC = kAsync<T, V>;
    constexpr int U = ASYNC ? kForwardTogether : 1;  // steps that a warp works on together
    __shared__ alignas(16) float s_w[2][kHeadCols];
    __shared__ unsigned s_amax[kWarps][64];
    __shared__ uint4 s_in[2][2 * U][ASYNC ? kThreads : 1];  // [turn][step, vector][thread]
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const int cols = COLS ? COLS : a.cols, half = COLS ? COLS / 2 : a.half;
    const float inv_cols = COLS ? 1.0f / (float)COLS : a.inv_cols;
    const int lanes = COLS ? COLS / 2 / V : a.lanes;
    const int per = 32 / lanes, sub = lane % lanes, slot = lane / lanes;  // heads of a warp; this lane's place in its head
    stage_weights(a, s_w);
    Share mine(a, warp, kWarps, per, slot);  // the row that is fetched from
    if (!mine.some) return;
    const Side& q = a.side[mine.side];
    const int heads = q.heads, steps = mine.steps;
    Columns col[NV];
    bool ok[NV], turned[NV][2];
    constexpr int R = ASYNC ? 1 : U;
    Raw<T, V> raw[R][NV][2];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        col[i] = columns_of<V, NEXT>(cols, half, sub + lanes * i);
        ok[i] = COLS > 0 || sub + lanes * i < a.vectors;
        turned[i][0] = COLS > 0 || col[i].angle[0] >= 0;
        turned[i][1] = COLS > 0 || col[i].angle[1] >= 0;
#pragma unroll
        for (int u = 0; u < R; ++u) {  // lanes without a vector keep zeros; those of no head have anything
            raw[u][i][0].zero();
            raw[u][i][1].zero();
        }
    }
    uint4* places = &s_in[0][0][ASYNC ? threadIdx.x : 0];
    constexpr int kTurn = 2 * U * kThreads;
    if constexpr (ASYNC)
#pragma unroll
        for (int k = 0; k < 4 * U; ++k) places[k * kThreads] = make_uint4(0, 0, 0, 0);
    int turn = 0;
    const long long x_step = per * q.x_head, out_step = per * q.out_head;
    const int end = min(heads, mine.head0 + steps * per);  // behind this lane's heads
    const T* in = nullptr;
    auto fetch = [&](int head) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (head + u * per < end) {
#pragma unroll
                for (int i = 0; i < NV; ++i)
                    if (ok[i]) {
#pragma unroll
                        for (int m = 0; m < 2; ++m) {
                            if constexpr (ASYNC)
                                copy_async<16>(places + turn + (2 * u + m) * kThreads, in + col[i].col[m]);
                            else
                                raw[u % R][i][m].load(in + col[i].col[m]);
                        }
                    }
            }
            in += x_step;
        }
    };
    in = mine.at(static_cast<const T*>(q.x), q.x_batch, q.x_token, q.x_head);
    fetch(mine.head0);
    if (ASYNC) commit_async();
    long long position = half > 0 ? mine.position(a) : 0;
    for (bool more = true; more;) {
        const long long here = position;
        T* out = mine.at(static_cast<T*>(q.out), q.out_batch, q.out_token, q.out_head);
        const long long at = (long long)mine.row * heads + mine.head0;  // row of the statistics and of the checkpoint
        float* stat = q.rstd + at;
        unsigned char *codes = nullptr, *scales = nullptr;
        if (FMT) {
            codes = q.codes + at * q.ld_codes;
            scales = q.scales + at * q.ld_scales;
        }
        more = !mine.last(a);
        if (more) mine.advance(a);
        if (half > 0) position = mine.position(a);
        // y = rstd * (own * f + partner * g): the weights times the cosines and sines of this token
        float2 f[NV][2][P], g[NV][2][P];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (!ok[i]) continue;
            float2 w[2][P];
            take_weights<V>(s_w[mine.side] + col[i].col[0], w[0]);
            take_weights<V>(s_w[mine.side] + col[i].col[1], w[1]);
            load_angles<V, NEXT>(a, half, here, col[i].angle, false, f[i], g[i]);
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
                for (int k = 0; k < P; ++k) {
                    f[i][m][k] = turned[i][m] ? __fmul2_rn(f[i][m][k], w[m][k]) : w[m][k];
                    g[i][m][k] = __fmul2_rn(g[i][m][k], partner<V, NEXT>(w, m, k));
                }
        }
        for (int step = 0, head = mine.head0; step < steps; step += U, head += U * per) {
            // the next steps' elements, or the next token's: into the other place, or behind these in the registers
            auto ahead = [&] {
                if (step + U < steps) {
                    fetch(head + U * per);
                } else if (more) {
                    in = mine.at(static_cast<const T*>(q.x), q.x_batch, q.x_token, q.x_head);
                    fetch(mine.head0);
                }
            };
            const uint4* now = places + turn;
            if constexpr (ASYNC) {
                turn ^= kTurn;
                ahead();
                commit_async();
                wait_async<1>();
            }
            float2 x[U][NV][2][P];
            float rstd[U];
            bool live[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                live[u] = head + u * per < end;
                float2 sq = make_float2(0.0f, 0.0f);
#pragma unroll
                for (int i = 0; i < NV; ++i)
#pragma unroll
                    for (int m = 0; m < 2; ++m) {
                        if (ASYNC) raw[0][i][m].take(now + (2 * u + m) * kThreads);
                        raw[u % R][i][m].unpack(x[u][i][m]);
#pragma unroll
                        for (int k = 0; k < P; ++k) sq = __ffma2_rn(x[u][i][m][k], x[u][i][m][k], sq);
                    }
                rstd[u] = sq.x + sq.y;
            }
            if constexpr (!ASYNC) ahead();
            head_sums<U, COLS>(rstd, lanes);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                rstd[u] = inverse_root(rstd[u] * inv_cols + a.eps);
                if (live[u] && sub == 0) stat[u * per] = rstd[u];
            }
            stat += U * per;
            if (FMT) {
                // bits of the largest |x| of each group of 32 columns, a NaN on top
                unsigned top[U][NV][2];
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int i = 0; i < NV; ++i)
#pragma unroll
                        for (int m = 0; m < 2; ++m) {
                            float t = 0.0f;
#pragma unroll
                            for (int k = 0; k < P; ++k) asm("max.NaN.abs.f32 %0, %0, %1, %2;" : "+f"(t) : "f"(x[u][i][m][k].x), "f"(x[u][i][m][k].y));
                            top[u][i][m] = __float_as_uint(t) & 0x7FFFFFFFu;
                        }
                if (COLS || a.lane_groups) {
#pragma unroll
                    for (int u = 0; u < U; ++u)
#pragma unroll
                        for (int i = 0; i < NV; ++i) {
#pragma unroll
                            for (int o = kGroup / V / 2; o > 0; o >>= 1) {
                                top[u][i][0] = max(top[u][i][0], __shfl_xor_sync(0xFFFFFFFFu, top[u][i][0], o));
                                top[u][i][1] = max(top[u][i][1], __shfl_xor_sync(0xFFFFFFFFu, top[u][i][1], o));
                            }
                        }
                } else {
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        unsigned* amax = s_amax[warp] + slot * ((cols + kGroup - 1) / kGroup);
                        __syncwarp();
                        s_amax[warp][lane] = s_amax[warp][lane + 32] = 0;
                        __syncwarp();
#pragma unroll
                        for (int i = 0; i < NV; ++i)
#pragma unroll
                            for (int m = 0; m < 2; ++m)
                                if (live[u] && ok[i]) atomicMax(amax + col[i].col[m] / kGroup, top[u][i][m]);
                        __syncwarp();
#pragma unroll
                        for (int i = 0; i < NV; ++i)
#pragma unroll
                            for (int m = 0; m < 2; ++m)
                                if (live[u] && ok[i]) top[u][i][m] = amax[col[i].col[m] / kGroup];
                    }
                }
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    if (live[u]) {
#pragma unroll
                        for (int i = 0; i < NV; ++i) {
                            if (!ok[i]) continue;
#pragma unroll
                            for (int m = 0; m < 2; ++m) {
                                const int c0 = col[i].col[m];
                                const unsigned byte = group_byte<FMT>(a.e4m3, top[u][i][m]);
                                store_code_vec<V, FMT>(codes + c0, a.e4m3, byte, x[u][i][m]);
                                if (c0 % kGroup == 0) scales[c0 / kGroup] = (unsigned char)byte;  // by whoever holds a group's first column
                            }
                        }
                        if (cols % kGroup)
                            for (int k = cols + sub; k < (cols + kGroup - 1) / kGroup * kGroup; k += lanes) codes[k] = 0;
                    }
                    codes += per * q.ld_codes;
                    scales += per * q.ld_scales;
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (live[u]) {
#pragma unroll
                    for (int i = 0; i < NV; ++i) {
                        if (!ok[i]) continue;
#pragma unroll
                        for (int m = 0; m < 2; ++m) {
                            float2 y[P];
#pragma unroll
                            for (int k = 0; k < P; ++k) {
                                y[k] = __fmul2_rn(x[u][i][m][k], f[i][m][k]);
                                if (turned[i][m]) y[k] = turn_with<V, NEXT>(x[u][i], m, k, g[i][m][k], y[k]);
                                y[k] = __fmul2_rn(y[k], make_float2(rstd[u], rstd[u]));
                            }
                            store_vec<T, V>(out + col[i].col[m], y);
                        }
                    }
                }
                out += out_step;
            }
        }
    }
}

// A warp's sums for the weight's gradient stay in registers over its tokens;
// part[CTA][column] of a side's CTAs are joined afterwards.  The same size: bf16 79 us
// from 8 bits (4.9 TB/s), 80 us from the input (5.7 TB/s), fp32 115 us from 8 bits;
// 16 warps an SM and instructions bound the first.
template <typename T, int V, int NV, bool NEXT, int FMT, int COLS>
__global__ void __launch_bounds__(kBackwardThreads, kCtas<V>) head_norm_backward_kernel(const HeadArgs a) {
    constexpr int kThreads = kBackwardThreads, kWarps = kThreads / 32;
    constexpr int P = kPairs<V>;
    constexpr bool ASYNC = kAsync<T, V>;
    constexpr int U = ASYNC ? kBackwardTogether<T> : 1;  // steps that a warp works on together
    constexpr int R = ASYNC ? 1 : U;
    __shared__ alignas(16) float s_w[2][kHeadCols];
    __shared__ float s_sums[kWarps][kHeadCols];
    __shared__ uint4 s_in[2][4 * U][ASYNC ? kThreads : 1];  // [turn][step, gradient, input or codes][thread]
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const int cols = COLS ? COLS : a.cols, half = COLS ? COLS / 2 : a.half;
    const float inv_cols = COLS ? 1.0f / (float)COLS : a.inv_cols;
    const int lanes = COLS ? COLS / 2 / V : a.lanes;
    const int per = 32 / lanes, sub = lane % lanes, slot = lane / lanes;
    stage_weights(a, s_w);
    Share mine(a, warp, kWarps, per, slot);  // the row that is fetched from
    const Side& q = a.side[mine.side];
    const int heads = q.heads, steps = mine.steps;
    Columns col[NV];
    bool ok[NV], turned[NV][2];
    float2 gw[NV][2][P], w[NV][2][P];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        col[i] = columns_of<V, NEXT>(cols, half, sub + lanes * i);
        ok[i] = COLS > 0 || sub + lanes * i < a.vectors;
        turned[i][0] = COLS > 0 || col[i].angle[0] >= 0;
        turned[i][1] = COLS > 0 || col[i].angle[1] >= 0;
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            if (ok[i]) take_weights<V>(s_w[mine.side] + col[i].col[m], w[i][m]);
#pragma unroll
            for (int k = 0; k < P; ++k) gw[i][m][k] = make_float2(0.0f, 0.0f);
        }
    }
    if (mine.some) {
        Raw<T, V> raw_g[R][NV][2], raw_x[R][NV][2];
        RawCodes<V> raw_c[R][NV][2];
        unsigned raw_s[U][NV][2];
        float raw_r[U];
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int m = 0; m < 2; ++m) {
#pragma unroll
                for (int u = 0; u < R; ++u) {
                    raw_g[u][i][m].zero();
                    raw_x[u][i][m].zero();
                    raw_c[u][i][m].c = make_uint2(0, 0);
                }
#pragma unroll
                for (int u = 0; u < U; ++u) raw_s[u][i][m] = 0;
            }
#pragma unroll
        for (int u = 0; u < U; ++u) raw_r[u] = 0.0f;
        uint4* places = &s_in[0][0][ASYNC ? threadIdx.x : 0];
        constexpr int kTurn = 4 * U * kThreads;
        if constexpr (ASYNC)
#pragma unroll
            for (int k = 0; k < 8 * U; ++k) places[k * kThreads] = make_uint4(0, 0, 0, 0);
        int turn = 0;
        const long long g_step = per * q.gy_head, x_step = per * q.x_head, out_step = per * q.out_head;
        const int end = min(heads, mine.head0 + steps * per);  // behind this lane's heads
        const T *gp = nullptr, *xp = nullptr;
        const unsigned char *cp = nullptr, *sp = nullptr;
        const float* rp = nullptr;
        auto begin = [&] {  // of the row
            const long long at = (long long)mine.row * heads + mine.head0;
            gp = mine.at(static_cast<const T*>(q.gy), q.gy_batch, q.gy_token, q.gy_head);
            rp = q.rstd + at;
            if (FMT) {
                cp = q.codes + at * q.ld_codes;
                sp = q.scales + at * q.ld_scales;
            } else {
                xp = mine.at(static_cast<const T*>(q.x), q.x_batch, q.x_token, q.x_head);
            }
        };
        auto fetch = [&](int head) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (head + u * per < end) {
                    raw_r[u] = __ldg(rp);
#pragma unroll
                    for (int i = 0; i < NV; ++i) {
                        if (!ok[i]) continue;
#pragma unroll
                        for (int m = 0; m < 2; ++m) {
                            const int c0 = col[i].col[m];
                            if constexpr (ASYNC) {
                                copy_async<16>(places + turn + (4 * u + m) * kThreads, gp + c0);
                                if (FMT)
                                    copy_async<V>(places + turn + (4 * u + 2 + m) * kThreads, cp + c0);
                                else
                                    copy_async<16>(places + turn + (4 * u + 2 + m) * kThreads, xp + c0);
                            } else {
                                raw_g[u % R][i][m].load(gp + c0);
                                if (FMT)
                                    raw_c[u % R][i][m].load(cp + c0);
                                else
                                    raw_x[u % R][i][m].load(xp + c0);
                            }
                            if (FMT) raw_s[u][i][m] = __ldg(sp + c0 / kGroup);
                        }
                    }
                }
                gp += g_step;
                rp += per;
                if (FMT) {
                    cp += per * q.ld_codes;
                    sp += per * q.ld_scales;
                } else {
                    xp += x_step;
                }
            }
        };
        begin();
        fetch(mine.head0);
        if (ASYNC) commit_async();
        long long position = half > 0 ? mine.position(a) : 0;
        for (bool more = true; more;) {
            const long long here = position;
            T* out = mine.at(static_cast<T*>(q.out), q.out_batch, q.out_token, q.out_head);
            more = !mine.last(a);
            if (more) mine.advance(a);
            if (half > 0) position = mine.position(a);
            float2 c[NV][2][P], s[NV][2][P];
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (ok[i]) load_angles<V, NEXT>(a, half, here, col[i].angle, true, c[i], s[i]);
            for (int step = 0, head = mine.head0; step < steps; step += U, head += U * per) {
                bool live[U];
                float rstd[U], dot[U];
                float2 g[U][NV][2][P], h[U][NV][2][P];  // in the end u and x * rstd
                float scale[U][NV][2];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    live[u] = head + u * per < end;
                    rstd[u] = raw_r[u];
#pragma unroll
                    for (int i = 0; i < NV; ++i)
#pragma unroll
                        for (int m = 0; m < 2; ++m) scale[u][i][m] = FMT ? scale_of(raw_s[u][i][m]) * rstd[u] : rstd[u];  // a power of two: exact
                }
                auto ahead = [&] {
                    if (step + U < steps) {
                        fetch(head + U * per);
                    } else if (more) {
                        begin();
                        fetch(mine.head0);
                    }
                };
                const uint4* now = places + turn;
                if constexpr (ASYNC) {
                    turn ^= kTurn;
                    ahead();
                    commit_async();
                    wait_async<1>();
                }
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int i = 0; i < NV; ++i)
#pragma unroll
                        for (int m = 0; m < 2; ++m) {
                            if (ASYNC) raw_g[0][i][m].take(now + (4 * u + m) * kThreads);
                            raw_g[u % R][i][m].unpack(g[u][i][m]);
                            if constexpr (FMT != 0) {
                                if (ASYNC) raw_c[0][i][m].c = *reinterpret_cast<const uint2*>(now + (4 * u + 2 + m) * kThreads);  // fp32: the first word
                                raw_c[u % R][i][m].template unpack<FMT>(a.e4m3, scale[u][i][m], h[u][i][m]);
                            } else {
                                if (ASYNC) raw_x[0][i][m].take(now + (4 * u + 2 + m) * kThreads);
                                raw_x[u % R][i][m].unpack(h[u][i][m]);
#pragma unroll
                                for (int k = 0; k < P; ++k) h[u][i][m][k] = __fmul2_rn(h[u][i][m][k], make_float2(rstd[u], rstd[u]));
                            }
                        }
                if constexpr (!ASYNC) ahead();
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    float2 sum = make_float2(0.0f, 0.0f);
                    if (live[u]) {
#pragma unroll
                        for (int i = 0; i < NV; ++i) {
                            if (!ok[i]) continue;
                            float2 t[2][P];
#pragma unroll
                            for (int m = 0; m < 2; ++m)
#pragma unroll
                                for (int k = 0; k < P; ++k) {
                                    t[m][k] = g[u][i][m][k];
                                    if (turned[i][m]) t[m][k] = turn_with<V, NEXT>(g[u][i], m, k, s[i][m][k], __fmul2_rn(t[m][k], c[i][m][k]));
                                    gw[i][m][k] = __ffma2_rn(t[m][k], h[u][i][m][k], gw[i][m][k]);
                                    t[m][k] = __fmul2_rn(t[m][k], w[i][m][k]);
                                    sum = __ffma2_rn(t[m][k], h[u][i][m][k], sum);
                                }
#pragma unroll
                            for (int m = 0; m < 2; ++m)
#pragma unroll
                                for (int k = 0; k < P; ++k) g[u][i][m][k] = t[m][k];
                        }
                    }
                    dot[u] = sum.x + sum.y;
                }
                head_sums<U, COLS>(dot, lanes);
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    if (live[u]) {
                        const float mean = -dot[u] * inv_cols;
#pragma unroll
                        for (int i = 0; i < NV; ++i) {
                            if (!ok[i]) continue;
#pragma unroll
                            for (int m = 0; m < 2; ++m) {
#pragma unroll
                                for (int k = 0; k < P; ++k)
                                    g[u][i][m][k] = __fmul2_rn(__ffma2_rn(h[u][i][m][k], make_float2(mean, mean), g[u][i][m][k]), make_float2(rstd[u], rstd[u]));
                                store_vec<T, V>(out + col[i].col[m], g[u][i][m]);
                            }
                        }
                    }
                    out += out_step;
                }
            }
        }
    }
    if (!a.sums) return;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int k = 0; k < P; ++k) {
                float2 v = gw[i][m][k];
                for (int o = 16; o >= lanes; o >>= 1) {  // the warp's heads
                    v.x += __shfl_xor_sync(0xFFFFFFFFu, v.x, o);
                    v.y += __shfl_xor_sync(0xFFFFFFFFu, v.y, o);
                }
                if (slot == 0 && ok[i]) {
                    s_sums[warp][col[i].col[m] + 2 * k] = v.x;
                    if (V > 1) s_sums[warp][col[i].col[m] + 2 * k + 1] = v.y;
                }
            }
    __syncthreads();
    for (int c = threadIdx.x; c < cols; c += kThreads) {
        float v = 0.0f;
#pragma unroll
        for (int i = 0; i < kWarps; ++i) v += s_sums[i][c];
        a.part[(long long)blockIdx.x * a.pitch + c] = v;
    }
}

// Adds up the CTAs' partial rows of a side, queries (blockIdx.y 0) and keys, in a fixed
// order: eight columns to a block, 128 parts at a time.
struct JoinArgs {
    const float* part[2];
    void* out[2];
    int parts[2], cols, pitch;
    bool bf16;
};
constexpr int kJoinCols = 8, kJoinWays = 128, kJoinSums = 16;
__global__ void __launch_bounds__(kJoinCols* kJoinWays) head_join_kernel(const JoinArgs a) {
    __shared__ float sums[kJoinWays][kJoinCols + 1], few[kJoinSums][kJoinCols + 1];
    const int side = blockIdx.y, x = threadIdx.x, y = threadIdx.y, c = blockIdx.x * kJoinCols + x;
    if (!a.out[side]) return;
    float s = 0.0f;
    if (c < a.cols)
#pragma unroll 5
        for (int p = y; p < a.parts[side]; p += kJoinWays) s += __ldg(a.part[side] + (long long)p * a.pitch + c);
    sums[y][x] = s;
    __syncthreads();
    if (y < kJoinSums) {
        float t = 0.0f;
#pragma unroll
        for (int k = 0; k < kJoinWays / kJoinSums; ++k) t += sums[y * (kJoinWays / kJoinSums) + k][x];
        few[y][x] = t;
    }
    __syncthreads();
    if (y == 0 && c < a.cols) {
        float t = 0.0f;
#pragma unroll
        for (int k = 0; k < kJoinSums; ++k) t += few[k][x];
        if (a.bf16)
            store_elem(static_cast<__nv_bfloat16*>(a.out[side]) + c, t);
        else
            store_elem(static_cast<float*>(a.out[side]) + c, t);
    }
}

// ---------------------------------------------------------------------------
// host side

// CTAs of the backward pass: no more than are resident, four to a token at most.
int backward_ctas(long long rows, int sms) {
    const long long most = (long long)kMostCtas * sms;
    return rows == 0 ? 0 : (int)(4 * rows < most ? 4 * rows : most);
}

int part_pitch(long long cols) { return (int)((cols + 15) / 16 * 16); }

constexpr long long kMaxStride = 1LL << 40;

bool known_strides(long long b, long long t, long long h) {
    return b >= 0 && t >= 0 && h >= 0 && b <= kMaxStride && t <= kMaxStride && h <= kMaxStride;
}

bool element_aligned(const ampq_heads& h, int dtype, int param_dtype) {
    const size_t e = elem_bytes(dtype);
    return aligned_to(h.x, e) && aligned_to(h.gy, e) && aligned_to(h.out, e) && aligned_to(h.weight, elem_bytes(param_dtype)) &&
           aligned_to(h.gweight, elem_bytes(param_dtype)) && aligned_to(h.rstd, 4);
}

int check_side(const ampq_heads& h, int dtype, int param_dtype, int fmt, long long rows, long long cols, bool backward) {
    if (h.heads < 0) return AMPQ_ERR_INVALID;
    if (h.heads > (1 << 20) || rows * h.heads > kMaxRows) return AMPQ_ERR_TOO_LARGE;
    const bool some = rows * h.heads > 0 && cols > 0, kept = fmt != AMPQ_FMT_BASE;
    if (some && (!h.out || !h.rstd)) return AMPQ_ERR_INVALID;
    if (some && (backward ? !h.gy || (!kept && !h.x) : !h.x)) return AMPQ_ERR_INVALID;
    if (!known_strides(h.x_batch, h.x_token, h.x_head) || !known_strides(h.gy_batch, h.gy_token, h.gy_head) ||
        !known_strides(h.out_batch, h.out_token, h.out_head))
        return AMPQ_ERR_INVALID;
    if (!element_aligned(h, dtype, param_dtype)) return AMPQ_ERR_ALIGN;
    if (kept && h.heads > 0) return check_ckpt(h.codes, h.ld_codes, h.scales, h.ld_scales, rows * h.heads, cols);
    return AMPQ_OK;
}

int check_heads(int dtype, int param_dtype, int index_type, int fmt, long long batch, long long tokens, long long cols, long long rot, const float* cos,
                const float* sin, long long angles, const void* positions, long long position_batch, const ampq_heads* q, const ampq_heads* k, bool backward) {
    if (!known_dtype(dtype) || !known_dtype(param_dtype) || !known_index(index_type)) return AMPQ_ERR_INVALID;
    if (fmt != AMPQ_FMT_BASE && !known_fp8(fmt)) return AMPQ_ERR_INVALID;
    if (!q || batch < 0 || tokens < 0 || cols < 0 || cols % 2 || rot < 0 || rot % 2 || rot > cols) return AMPQ_ERR_INVALID;
    if (cols > kHeadCols || batch > kMaxRows || tokens > kMaxRows || batch * tokens > kMaxRows) return AMPQ_ERR_TOO_LARGE;
    if (angles < 0 || position_batch < 0) return AMPQ_ERR_INVALID;
    if (angles > kMaxRows || position_batch > kMaxStride) return AMPQ_ERR_TOO_LARGE;
    if (rot > 0 && angles > 0 && (!cos || !sin)) return AMPQ_ERR_INVALID;
    if (!aligned_to(cos, 16) || !aligned_to(sin, 16) || !aligned_to(positions, index_bytes(index_type))) return AMPQ_ERR_ALIGN;
    int rc = check_side(*q, dtype, param_dtype, fmt, batch * tokens, cols, backward);
    if (!rc && k) rc = check_side(*k, dtype, param_dtype, fmt, batch * tokens, cols, backward);
    return rc;
}

// Elements that one access of V elements may take from this tensor.
bool vectors_fit(const void* p, long long b, long long t, long long h, int dtype, int V) {
    const long long bytes = V * (long long)elem_bytes(dtype), e = (long long)elem_bytes(dtype);
    return !p || (aligned_to(p, (size_t)bytes) && b * e % bytes == 0 && t * e % bytes == 0 && h * e % bytes == 0);
}

bool vectors_fit(const HeadArgs& a, int dtype, int V) {
    if (a.half % V || (a.cols / 2 - a.half) % V) return false;
    for (const Side& s : a.side)
        if (s.heads > 0 && !(vectors_fit(s.x, s.x_batch, s.x_token, s.x_head, dtype, V) && vectors_fit(s.gy, s.gy_batch, s.gy_token, s.gy_head, dtype, V) &&
                             vectors_fit(s.out, s.out_batch, s.out_token, s.out_head, dtype, V)))
            return false;
    return true;
}

Side side_of(const ampq_heads* h, bool backward, bool kept) {
    Side s{};
    if (!h) return s;
    s.heads = (int)h->heads;
    s.x = backward && kept ? nullptr : h->x;
    s.gy = backward ? h->gy : nullptr;
    s.w = h->weight;
    s.out = h->out;
    s.rstd = h->rstd;
    s.codes = h->codes; s.scales = h->scales; s.ld_codes = h->ld_codes; s.ld_scales = h->ld_scales;
    s.x_batch = h->x_batch; s.x_token = h->x_token; s.x_head = h->x_head;
    s.gy_batch = h->gy_batch; s.gy_token = h->gy_token; s.gy_head = h->gy_head;
    s.out_batch = h->out_batch; s.out_token = h->out_token; s.out_head = h->out_head;
    return s;
}

// Sets up the lanes of a head, the runs, and the CTAs of each side; returns the grid's size.
constexpr int kTokenWork = 2;
long long lay_out(HeadArgs& a, int V, int NV, bool next, bool backward, int warps, int together, long long ctas) {
    a.vectors = a.cols / 2 / V;
    a.lanes = 1;
    while (a.lanes * NV < a.vectors) a.lanes *= 2;
    a.lane_groups = V > 1 && kGroup / V <= a.lanes && a.cols / 2 % kGroup == 0 && (next || a.half % kGroup == 0);
    const int per = 32 / a.lanes;
    const int steps[2] = {(a.side[0].heads + per - 1) / per, (a.side[1].heads + per - 1) / per};
    const long long most = ctas * warps;
    // Long runs share a token's angles among more heads; shorter ones while there are
    // warps without one.
    auto set = [&](int longest) {
        long long total = 0;
        for (int s = 0; s < 2; ++s) {
            const int n = (steps[s] + longest - 1) / longest;
            a.run[s] = n ? (steps[s] + n - 1) / n : 1;
            a.runs[s] = (steps[s] + a.run[s] - 1) / a.run[s];
            total += (a.runs[s] + warps - 1) / warps * warps;  // a side has whole CTAs
        }
        return total;
    };
    int longest = kMaxRun;
    long long total = set(longest);
    while (longest > 1 && (long long)a.rows * (a.runs[0] + a.runs[1]) < most) total = set(longest /= 2);
    while (backward && total > most) total = set(longest *= 2);  // every run has its warp
    long long grid = ctas;
    if (!backward) {
        const long long need = ((long long)a.rows * a.runs[0] + warps - 1) / warps + ((long long)a.rows * a.runs[1] + warps - 1) / warps;
        grid = need < most / warps ? need : most / warps;
        if (grid < total / warps) grid = total / warps;
    }
    // The CTAs go to the sides by their work, one warp to a run at least.  What a run does
    // once for a token is about two steps' work, and steps are done `together`.  (64 + 8 heads,
    // forward and backward: counted as none, the keys' CTAs came last, 76 and 84 us; as one, two or four steps 68 and 79.)
    const long long least[2] = {(a.runs[0] + warps - 1) / warps, (a.runs[1] + warps - 1) / warps};
    long long work[2];
    for (int s = 0; s < 2; ++s) work[s] = (long long)a.runs[s] * (kTokenWork + (a.run[s] + together - 1) / together * together);
    long long first = (grid * work[0] + (work[0] + work[1]) / 2) / (work[0] + work[1]);
    first = first < least[0] ? least[0] : first > grid - least[1] ? grid - least[1] : first;
    a.ctas[0] = (int)first;
    a.ctas[1] = (int)(grid - first);
    return grid;
}

template <typename T, int V, int NV, bool NEXT, int FMT, int COLS>
int start(HeadArgs& a, bool backward, int sms, int ctas, cudaStream_t st) {
    long long most = (long long)kCtas<V> * sms;
    if (backward && most > ctas) most = ctas;
    const long long grid = lay_out(a, V, NV, NEXT, backward, (backward ? kBackwardThreads : kForwardThreads) / 32, kAsync<T, V> ? (backward ? kBackwardTogether<T> : kForwardTogether) : 1, most);
    if (grid > 0x7FFFFFFFLL) return AMPQ_ERR_TOO_LARGE;
    if (backward)
        head_norm_backward_kernel<T, V, NV, NEXT, FMT, COLS><<<(unsigned)grid, kBackwardThreads, 0, st>>>(a);
    else
        head_norm_forward_kernel<T, V, NV, NEXT, FMT, COLS><<<(unsigned)grid, kForwardThreads, 0, st>>>(a);
    return launched();
}

// The head sizes of most models.
template <typename T, int V, bool NEXT, int COLS>
int known(HeadArgs& a, int fmt, bool backward, int sms, int ctas, cudaStream_t st) {
    if (fmt == AMPQ_FMT_E4M3) return start<T, V, 1, NEXT, AMPQ_FMT_E4M3, COLS>(a, backward, sms, ctas, st);
    if (fmt == AMPQ_FMT_E5M2) return start<T, V, 1, NEXT, AMPQ_FMT_E5M2, COLS>(a, backward, sms, ctas, st);
    return start<T, V, 1, NEXT, AMPQ_FMT_BASE, COLS>(a, backward, sms, ctas, st);
}

template <typename T, bool NEXT>
int pick(HeadArgs& a, int fmt, bool backward, int dtype, int sms, int ctas, cudaStream_t st) {
    constexpr int kWide = 16 / (int)sizeof(T);
    const bool kept = fmt != AMPQ_FMT_BASE;
    if (vectors_fit(a, dtype, kWide)) {
        if (2 * a.half == a.cols && a.cols == 64) return known<T, kWide, NEXT, 64>(a, fmt, backward, sms, ctas, st);
        if (2 * a.half == a.cols && a.cols == 128) return known<T, kWide, NEXT, 128>(a, fmt, backward, sms, ctas, st);
        if (2 * a.half == a.cols && a.cols == 256) return known<T, kWide, NEXT, 256>(a, fmt, backward, sms, ctas, st);
        return kept ? start<T, kWide, 1, NEXT, kEither, 0>(a, backward, sms, ctas, st) : start<T, kWide, 1, NEXT, AMPQ_FMT_BASE, 0>(a, backward, sms, ctas, st);
    }
    if (vectors_fit(a, dtype, 2))
        return kept ? start<T, 2, kHeadCols / 64, NEXT, kEither, 0>(a, backward, sms, ctas, st)
                    : start<T, 2, kHeadCols / 64, NEXT, AMPQ_FMT_BASE, 0>(a, backward, sms, ctas, st);
    return kept ? start<T, 1, kHeadCols / 64, NEXT, kEither, 0>(a, backward, sms, ctas, st)
                : start<T, 1, kHeadCols / 64, NEXT, AMPQ_FMT_BASE, 0>(a, backward, sms, ctas, st);
}

int dispatch(HeadArgs& a, bool next, int fmt, bool backward, int dtype, int sms, int ctas, cudaStream_t st) {
    if (dtype == AMPQ_F32) return next ? pick<float, true>(a, fmt, backward, dtype, sms, ctas, st) : pick<float, false>(a, fmt, backward, dtype, sms, ctas, st);
    return next ? pick<__nv_bfloat16, true>(a, fmt, backward, dtype, sms, ctas, st) : pick<__nv_bfloat16, false>(a, fmt, backward, dtype, sms, ctas, st);
}

HeadArgs head_args(int param_dtype, int index_type, int fmt, long long batch, long long tokens, long long cols, long long rot, const float* cos, const float* sin,
                   long long angles, const void* positions, long long position_batch, const ampq_heads* q, const ampq_heads* k, bool backward) {
    HeadArgs a{};
    a.side[0] = side_of(q, backward, fmt != AMPQ_FMT_BASE);
    a.side[1] = side_of(k, backward, fmt != AMPQ_FMT_BASE);
    a.cos = cos; a.sin = sin;
    a.positions = positions;
    a.rows = (unsigned)(batch * tokens); a.tokens = (unsigned)tokens; a.angles = angles; a.position_batch = position_batch;
    a.cols = (int)cols; a.half = (int)rot / 2;
    a.inv_cols = cols > 0 ? 1.0f / (float)cols : 0.0f;
    a.pitch = part_pitch(cols);
    a.param_bf16 = param_dtype == AMPQ_BF16;
    a.wide = index_type == AMPQ_I64;
    a.e4m3 = fmt == AMPQ_FMT_E4M3;
    return a;
}

}  // namespace
}  // namespace ampq

using namespace ampq;

extern "C" {
#pragma GCC visibility push(default)

int ampq_head_norm_forward(int device, void* cuda_stream, int dtype, int param_dtype, int index_type, int fmt, int interleaved, long long batch,
                           long long tokens, long long cols, long long rot, const float* cos, const float* sin, long long angles, const void* positions,
                           long long position_batch, float eps, const ampq_heads* q, const ampq_heads* k) {
    const int rc = check_heads(dtype, param_dtype, index_type, fmt, batch, tokens, cols, rot, cos, sin, angles, positions, position_batch, q, k, false);
    if (rc) return rc;
    if (!(eps >= 0.0f) || std::isinf(eps)) return AMPQ_ERR_INVALID;
    CkptDevice cur(device);
    if (cur.status) return cur.status;
    const int sms = sm_count(device);
    if (sms < 1) return AMPQ_ERR_CUDA;
    HeadArgs a = head_args(param_dtype, index_type, fmt, batch, tokens, cols, rot, cos, sin, angles, positions, position_batch, q, k, false);
    if (a.rows == 0 || a.side[0].heads + a.side[1].heads == 0) return AMPQ_OK;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
    if (cols == 0) {  // the mean of nothing: NaN, all bits set
        for (const Side& s : a.side)
            if (s.heads > 0 && s.rstd && cudaMemsetAsync(s.rstd, 0xFF, (size_t)((long long)a.rows * s.heads) * sizeof(float), st) != cudaSuccess) {
                cudaGetLastError();
                return AMPQ_ERR_CUDA;
            }
        return AMPQ_OK;
    }
    a.eps = eps;
    return dispatch(a, interleaved != 0, fmt, false, dtype, sms, 0, st);
}

int ampq_head_norm_backward_workspace(int device, long long batch, long long tokens, long long cols, long long* bytes) {
    if (!bytes || batch < 0 || tokens < 0 || cols < 0 || cols % 2) return AMPQ_ERR_INVALID;
    if (cols > kHeadCols || batch > kMaxRows || tokens > kMaxRows || batch * tokens > kMaxRows) return AMPQ_ERR_TOO_LARGE;
    CkptDevice cur(device);
    if (cur.status) return cur.status;
    const int sms = sm_count(device);
    if (sms < 1) return AMPQ_ERR_CUDA;
    *bytes = (long long)backward_ctas(batch * tokens, sms) * part_pitch(cols) * (long long)sizeof(float);
    return AMPQ_OK;
}

int ampq_head_norm_backward(int device, void* cuda_stream, int dtype, int param_dtype, int index_type, int fmt, int interleaved, long long batch,
                            long long tokens, long long cols, long long rot, const float* cos, const float* sin, long long angles, const void* positions,
                            long long position_batch, const ampq_heads* q, const ampq_heads* k, void* workspace, long long workspace_bytes) {
    int rc = check_heads(dtype, param_dtype, index_type, fmt, batch, tokens, cols, rot, cos, sin, angles, positions, position_batch, q, k, true);
    if (rc) return rc;
    if (!aligned_to(workspace, 256)) return AMPQ_ERR_ALIGN;
    CkptDevice cur(device);
    if (cur.status) return cur.status;
    if (cols == 0) return AMPQ_OK;
    const int sms = sm_count(device);
    if (sms < 1) return AMPQ_ERR_CUDA;
    HeadArgs a = head_args(param_dtype, index_type, fmt, batch, tokens, cols, rot, cos, sin, angles, positions, position_batch, q, k, true);
    const int ctas = backward_ctas(a.rows, sms);
    a.sums = q->gweight || (k && k->gweight);
    if (a.sums && ctas > 0 && (!workspace || workspace_bytes < (long long)ctas * a.pitch * (long long)sizeof(float))) return AMPQ_ERR_INVALID;
    a.part = static_cast<float*>(workspace);
    cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
    const bool some = a.rows > 0 && a.side[0].heads + a.side[1].heads > 0;
    if (some) {
        rc = dispatch(a, interleaved != 0, fmt, true, dtype, sms, ctas, st);
        if (rc) return rc;
    }
    if (!a.sums) return AMPQ_OK;
    JoinArgs j{};
    for (int side = 0; side < 2; ++side) {  // the queries' CTAs come first, then the keys'
        const ampq_heads* h = side ? k : q;
        j.part[side] = a.part + (side ? (long long)a.ctas[0] * a.pitch : 0);
        j.parts[side] = some && a.side[side].heads ? a.ctas[side] : 0;
        j.out[side] = h ? h->gweight : nullptr;
    }
    j.cols = a.cols; j.pitch = a.pitch;
    j.bf16 = a.param_bf16;
    head_join_kernel<<<dim3((unsigned)((a.cols + kJoinCols - 1) / kJoinCols), 2), dim3(kJoinCols, kJoinWays), 0, st>>>(j);
    return launched();
}

#pragma GCC visibility pop
}  // extern "C"
