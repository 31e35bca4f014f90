// Norms of queries and keys for each head with the position rotation in the same
// pass, forward and backward (include/ampq.h: ampq_head_norm_forward,
// ampq_head_norm_backward).
//
//   r = 1 / sqrt(mean_c x^2 + eps), n = x r w, (y_i, y_j) = (n_i cos - n_j sin, n_j cos + n_i sin)
// backward, with t the gradient turned back, h = x r and u = t w:
//   gx = r (u - h mean_c(u h)), gw = sum over tokens and heads of t h
//
// Layout.  A thread holds the two vectors of V columns that are turned into one
// another, so a rotation needs no exchange between threads: columns j V and
// rot / 2 + j V, or 2 V neighbouring columns where the pairs are neighbours.  The
// columns that are not turned are halved in the same way (cos 1, sin 0).  A head
// takes the smallest power of two of lanes that holds it, a warp several heads at
// once; the sum over a head's columns is a few shuffles.
#include "ampq_decoder.h"

#include <cmath>

namespace ampq {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kHeadCols = AMPQ_HEAD_MAX_COLS;

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
    long long rows, tokens, angles, position_batch;  // rows: batch * tokens
    int cols, half, lanes, vectors, runs, pitch;      // half: rot / 2; vectors: pairs of vectors of a head
    float eps, inv_cols;
    bool param_bf16, wide, e4m3, sums;
    bool lane_groups;  // a checkpoint's groups are whole vectors of neighbouring lanes
};

// V neighbouring elements, aligned to their size.
template <typename T, int V>
__device__ __forceinline__ void load_vec(const T* p, float (&v)[V]) {
    constexpr int B = V * (int)sizeof(T);
    if constexpr (B == 16) {
        const uint4 q = __ldg(reinterpret_cast<const uint4*>(p));
        const unsigned w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (sizeof(T) == 4) {
                v[i] = __uint_as_float(w[i]);
            } else {
                v[2 * i] = __uint_as_float(w[i] << 16);
                v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
            }
        }
    } else if constexpr (B == 8) {
        const float2 q = __ldg(reinterpret_cast<const float2*>(p));
        v[0] = q.x;
        v[1] = q.y;
    } else if constexpr (V == 2) {
        const unsigned q = __ldg(reinterpret_cast<const unsigned*>(p));
        v[0] = __uint_as_float(q << 16);
        v[1] = __uint_as_float(q & 0xFFFF0000u);
    } else {
        v[0] = load_elem(p);
    }
}

template <typename T, int V>
__device__ __forceinline__ void store_vec(T* p, const float (&v)[V]) {
    constexpr int B = V * (int)sizeof(T);
    if constexpr (B == 16 && sizeof(T) == 4)
        *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
    else if constexpr (B == 16)
        *reinterpret_cast<uint4*>(p) = make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
    else if constexpr (B == 8)
        *reinterpret_cast<float2*>(p) = make_float2(v[0], v[1]);
    else if constexpr (V == 2)
        *reinterpret_cast<unsigned*>(p) = pack_bf16(v[0], v[1]);
    else
        store_elem(p, v[0]);
}

// V codes of FP8, element 0 in the lowest byte.
template <int V>
__device__ __forceinline__ void load_code_vec(const unsigned char* p, bool e4m3, float scale, float (&v)[V]) {
    uint2 c = make_uint2(0, 0);
    if constexpr (V == 8) c = __ldg(reinterpret_cast<const uint2*>(p));
    if constexpr (V == 4) c.x = __ldg(reinterpret_cast<const unsigned*>(p));
    if constexpr (V == 2) c.x = __ldg(reinterpret_cast<const unsigned short*>(p));
    if constexpr (V == 1) c.x = __ldg(p);
    float f[8];
    if (e4m3)
        decode8<AMPQ_FMT_E4M3>(c, f);
    else
        decode8<AMPQ_FMT_E5M2>(c, f);
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = f[i] * scale;
}

template <int V>
__device__ __forceinline__ void store_code_vec(unsigned char* p, bool e4m3, unsigned byte, const float (&v)[V]) {
    const float inv = inv_scale_of(byte);
    unsigned short c[V / 2 + 1];
#pragma unroll
    for (int i = 0; i < V; i += 2) {
        const float lo = v[i] * inv, hi = i + 1 < V ? v[(i + 1) % V] * inv : 0.0f;
        if (e4m3)
            asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(c[i / 2]) : "f"(hi), "f"(lo));
        else
            asm("cvt.rn.satfinite.e5m2x2.f32 %0, %1, %2;" : "=h"(c[i / 2]) : "f"(hi), "f"(lo));
        if (byte == kNanScale) c[i / 2] = 0;
    }
    if constexpr (V == 8) *reinterpret_cast<uint2*>(p) = make_uint2(c[0] | (unsigned)c[1] << 16, c[2] | (unsigned)c[3] << 16);
    if constexpr (V == 4) *reinterpret_cast<unsigned*>(p) = c[0] | (unsigned)c[1] << 16;
    if constexpr (V == 2) *reinterpret_cast<unsigned short*>(p) = c[0];
    if constexpr (V == 1) *p = (unsigned char)c[0];
}

// Columns of a thread's j-th pair of vectors, and the angle that its first pair has
// (-1: not turned).
struct Columns {
    int a, b, angle;
};
template <int V, bool NEXT>
__device__ __forceinline__ Columns columns_of(const HeadArgs& p, int j) {
    const int turned = p.half / V;  // pairs of vectors that are turned
    if (NEXT) return Columns{2 * V * j, 2 * V * j + V, j < turned ? V * j : -1};
    if (j < turned) return Columns{V * j, p.half + V * j, V * j};
    const int rest = (p.cols - 2 * p.half) / 2, at = 2 * p.half + V * (j - turned);
    return Columns{at, at + rest, -1};
}

// The elements as pairs: x[i] and y[i] are turned into one another.
template <int V, bool NEXT>
__device__ __forceinline__ void to_pairs(float (&x)[V], float (&y)[V]) {
    if (!NEXT || V == 1) return;
    float e[2 * V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        e[i] = x[i];
        e[V + i] = y[i];
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
        x[i] = e[2 * i];
        y[i] = e[2 * i + 1];
    }
}
template <int V, bool NEXT>
__device__ __forceinline__ void from_pairs(float (&x)[V], float (&y)[V]) {
    if (!NEXT || V == 1) return;
    float e[2 * V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        e[2 * i] = x[i];
        e[2 * i + 1] = y[i];
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
        x[i] = e[i];
        y[i] = e[V + i];
    }
}

// Angles of a token for a thread's pairs.  A position outside the table has NaN.
template <int V>
__device__ __forceinline__ void load_angles(const HeadArgs& p, long long position, int angle, float (&c)[V], float (&s)[V]) {
    const bool known = position >= 0 && position < p.angles;
    const long long at = position * p.half + angle;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        c[i] = angle < 0 ? 1.0f : NAN;
        s[i] = angle < 0 ? 0.0f : NAN;
    }
    if (angle < 0 || !known) return;
    if constexpr (V >= 4) {
        if ((p.half & 3) == 0) {  // rows of the table on 16-byte boundaries (its base is)
#pragma unroll
            for (int i = 0; i < V; i += 4) {
                const float4 f = __ldg(reinterpret_cast<const float4*>(p.cos + at + i)), g = __ldg(reinterpret_cast<const float4*>(p.sin + at + i));
                c[i] = f.x; c[i + 1] = f.y; c[(i + 2) % V] = f.z; c[(i + 3) % V] = f.w;
                s[i] = g.x; s[i + 1] = g.y; s[(i + 2) % V] = g.z; s[(i + 3) % V] = g.w;
            }
            return;
        }
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
        c[i] = __ldg(p.cos + at + i);
        s[i] = __ldg(p.sin + at + i);
    }
}

template <int V>
__device__ __forceinline__ void load_weights(const HeadArgs& p, const void* w, int col, float (&v)[V]) {
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = w ? load_param(w, col + i, p.param_bf16) : 1.0f;
}

__device__ __forceinline__ long long position_of(const HeadArgs& p, long long batch, long long token) {
    return p.positions ? load_index(p.positions, batch * p.position_batch + token, p.wide) : token;
}

// Sum over the `lanes` neighbouring lanes of a head.
__device__ __forceinline__ float head_sum(float s, int lanes) {
    for (int o = lanes / 2; o > 0; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
    return s;
}

// ---------------------------------------------------------------------------

// A warp takes a run of heads of one token (a.runs runs cover queries and keys), so
// that its angles are read once.
template <typename T, int V, int NV, bool NEXT, bool KEPT>
__global__ void __launch_bounds__(kThreads) head_norm_forward_kernel(const HeadArgs a) {
    __shared__ unsigned s_amax[kWarps][64];
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const long long task = (long long)blockIdx.x * kWarps + warp;
    if (task >= a.rows * a.runs) return;
    const long long row = task / a.runs;
    const int run = (int)(task - row * a.runs);
    const long long batch = row / a.tokens, token = row - batch * a.tokens;
    const int per = 32 / a.lanes, sub = lane % a.lanes, slot = lane / a.lanes;  // heads of a warp; this lane's place in its head
    const int steps0 = (a.side[0].heads + per - 1) / per, steps1 = (a.side[1].heads + per - 1) / per, steps = steps0 + steps1;
    const int from = (int)((long long)steps * run / a.runs), to = (int)((long long)steps * (run + 1) / a.runs);
    const long long position = a.half > 0 ? position_of(a, batch, token) : 0;

    Columns col[NV];
    float c[NV][V], s[NV][V], wx[NV][V], wy[NV][V];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        col[i] = columns_of<V, NEXT>(a, sub + a.lanes * i);
        if (sub + a.lanes * i < a.vectors) load_angles<V>(a, position, col[i].angle, c[i], s[i]);
    }
    int side = -1;
    for (int step = from; step < to; ++step) {
        if (side < 0 || (side == 0 && step >= steps0)) {
            side = step >= steps0;
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (sub + a.lanes * i < a.vectors) {
                    load_weights<V>(a, a.side[side].w, col[i].a, wx[i]);
                    load_weights<V>(a, a.side[side].w, col[i].b, wy[i]);
                    to_pairs<V, NEXT>(wx[i], wy[i]);
                }
        }
        const Side& q = a.side[side];
        const int head = (step - (side ? steps0 : 0)) * per + slot;
        const bool live = head < q.heads;
        const T* in = static_cast<const T*>(q.x) + batch * q.x_batch + token * q.x_token + head * q.x_head;
        float x[NV][V], y[NV][V];
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
#pragma unroll
            for (int k = 0; k < V; ++k) x[i][k] = y[i][k] = 0.0f;
            if (live && sub + a.lanes * i < a.vectors) {
                load_vec<T, V>(in + col[i].a, x[i]);
                load_vec<T, V>(in + col[i].b, y[i]);
            }
#pragma unroll
            for (int k = 0; k < V; ++k) sum += x[i][k] * x[i][k] + y[i][k] * y[i][k];
        }
        const float rstd = 1.0f / sqrtf(head_sum(sum, a.lanes) * a.inv_cols + a.eps);
        const long long at = row * q.heads + head;  // row of the statistics and of the checkpoint
        if (live && sub == 0) q.rstd[at] = rstd;
        if (KEPT) {
            // largest |x| of each group of 32 columns: an integer maximum of the bits, a NaN on top
            unsigned mx[NV], my[NV];
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                mx[i] = my[i] = 0;
#pragma unroll
                for (int k = 0; k < V; ++k) {
                    mx[i] = max(mx[i], __float_as_uint(x[i][k]) & 0x7FFFFFFFu);
                    my[i] = max(my[i], __float_as_uint(y[i][k]) & 0x7FFFFFFFu);
                }
            }
            if (a.lane_groups) {
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    if (NEXT) mx[i] = my[i] = max(mx[i], my[i]);
                    for (int o = (NEXT ? kGroup / 2 : kGroup) / V / 2; o > 0; o >>= 1) {
                        mx[i] = max(mx[i], __shfl_xor_sync(0xFFFFFFFFu, mx[i], o));
                        my[i] = max(my[i], __shfl_xor_sync(0xFFFFFFFFu, my[i], o));
                    }
                }
            } else {
                const int groups = (a.cols + kGroup - 1) / kGroup;
                unsigned* amax = s_amax[warp] + slot * groups;
                __syncwarp();
                s_amax[warp][lane] = s_amax[warp][lane + 32] = 0;
                __syncwarp();
#pragma unroll
                for (int i = 0; i < NV; ++i)
                    if (live && sub + a.lanes * i < a.vectors) {
                        atomicMax(amax + col[i].a / kGroup, mx[i]);
                        atomicMax(amax + col[i].b / kGroup, my[i]);
                    }
                __syncwarp();
#pragma unroll
                for (int i = 0; i < NV; ++i)
                    if (live && sub + a.lanes * i < a.vectors) {
                        mx[i] = amax[col[i].a / kGroup];
                        my[i] = amax[col[i].b / kGroup];
                    }
            }
            if (live) {
                unsigned char *codes = q.codes + at * q.ld_codes, *scales = q.scales + at * q.ld_scales;
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    if (sub + a.lanes * i >= a.vectors) continue;
                    const unsigned bx = a.e4m3 ? scale_byte<AMPQ_FMT_E4M3>(mx[i]) : scale_byte<AMPQ_FMT_E5M2>(mx[i]);
                    const unsigned by = a.e4m3 ? scale_byte<AMPQ_FMT_E4M3>(my[i]) : scale_byte<AMPQ_FMT_E5M2>(my[i]);
                    store_code_vec<V>(codes + col[i].a, a.e4m3, bx, x[i]);
                    store_code_vec<V>(codes + col[i].b, a.e4m3, by, y[i]);
                    // a group's byte by whoever holds its first column
                    if (col[i].a % kGroup == 0) scales[col[i].a / kGroup] = (unsigned char)bx;
                    if (col[i].b % kGroup == 0) scales[col[i].b / kGroup] = (unsigned char)by;
                }
                for (int k = a.cols + sub; k < (a.cols + kGroup - 1) / kGroup * kGroup; k += a.lanes) codes[k] = 0;
            }
        }
        if (!live) continue;
        T* out = static_cast<T*>(q.out) + batch * q.out_batch + token * q.out_token + head * q.out_head;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (sub + a.lanes * i >= a.vectors) continue;
            to_pairs<V, NEXT>(x[i], y[i]);
#pragma unroll
            for (int k = 0; k < V; ++k) {
                const float nx = x[i][k] * rstd * wx[i][k], ny = y[i][k] * rstd * wy[i][k];
                const bool turn = col[i].angle >= 0;  // 0 * Inf is not 0
                x[i][k] = turn ? nx * c[i][k] - ny * s[i][k] : nx;
                y[i][k] = turn ? ny * c[i][k] + nx * s[i][k] : ny;
            }
            from_pairs<V, NEXT>(x[i], y[i]);
            store_vec<T, V>(out + col[i].a, x[i]);
            store_vec<T, V>(out + col[i].b, y[i]);
        }
    }
}

// A CTA goes through tokens, the queries of all of them and then the keys, so that a
// thread's sums for the weight's gradient stay in registers; its warps share a token's
// heads.  part[side][CTA][column] are joined afterwards.
template <typename T, int V, int NV, bool NEXT, bool KEPT>
__global__ void __launch_bounds__(kThreads) head_norm_backward_kernel(const HeadArgs a) {
    __shared__ float s_sums[kWarps][kHeadCols];
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const int per = 32 / a.lanes, sub = lane % a.lanes, slot = lane / a.lanes;
    Columns col[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) col[i] = columns_of<V, NEXT>(a, sub + a.lanes * i);
    for (int side = 0; side < 2; ++side) {
        const Side& q = a.side[side];
        if (q.heads == 0) continue;
        float wx[NV][V], wy[NV][V], gwx[NV][V], gwy[NV][V];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
#pragma unroll
            for (int k = 0; k < V; ++k) gwx[i][k] = gwy[i][k] = 0.0f;
            if (sub + a.lanes * i < a.vectors) {
                load_weights<V>(a, q.w, col[i].a, wx[i]);
                load_weights<V>(a, q.w, col[i].b, wy[i]);
                to_pairs<V, NEXT>(wx[i], wy[i]);
            }
        }
        // a run of a token's heads to a warp, as in the forward pass
        const int steps = (q.heads + per - 1) / per;
        const int runs = min(a.runs, steps);
        for (long long task = (long long)blockIdx.x * kWarps + warp; task < a.rows * runs; task += (long long)gridDim.x * kWarps) {
            const long long row = task / runs;
            const int run = (int)(task - row * runs);
            const long long batch = row / a.tokens, token = row - batch * a.tokens;
            const int from = (int)((long long)steps * run / runs), to = (int)((long long)steps * (run + 1) / runs);
            const long long position = a.half > 0 ? position_of(a, batch, token) : 0;
            float c[NV][V], s[NV][V];
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (sub + a.lanes * i < a.vectors) load_angles<V>(a, position, col[i].angle, c[i], s[i]);
            for (int step = from; step < to; ++step) {
                const int head = step * per + slot;
                const bool live = head < q.heads;
                const long long at = row * q.heads + head;
                const float rstd = live ? __ldg(q.rstd + at) : 0.0f;
                const T* g = static_cast<const T*>(q.gy) + batch * q.gy_batch + token * q.gy_token + head * q.gy_head;
                float hx[NV][V], hy[NV][V], ux[NV][V], uy[NV][V];
                float sum = 0.0f;
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    if (!live || sub + a.lanes * i >= a.vectors) continue;
                    load_vec<T, V>(g + col[i].a, ux[i]);
                    load_vec<T, V>(g + col[i].b, uy[i]);
                    if (KEPT) {
                        const unsigned char *codes = q.codes + at * q.ld_codes, *scales = q.scales + at * q.ld_scales;
                        load_code_vec<V>(codes + col[i].a, a.e4m3, scale_of(__ldg(scales + col[i].a / kGroup)), hx[i]);
                        load_code_vec<V>(codes + col[i].b, a.e4m3, scale_of(__ldg(scales + col[i].b / kGroup)), hy[i]);
                    } else {
                        const T* x = static_cast<const T*>(q.x) + batch * q.x_batch + token * q.x_token + head * q.x_head;
                        load_vec<T, V>(x + col[i].a, hx[i]);
                        load_vec<T, V>(x + col[i].b, hy[i]);
                    }
                    to_pairs<V, NEXT>(ux[i], uy[i]);
                    to_pairs<V, NEXT>(hx[i], hy[i]);
#pragma unroll
                    for (int k = 0; k < V; ++k) {
                        const bool turn = col[i].angle >= 0;
                        const float tx = turn ? ux[i][k] * c[i][k] + uy[i][k] * s[i][k] : ux[i][k];
                        const float ty = turn ? uy[i][k] * c[i][k] - ux[i][k] * s[i][k] : uy[i][k];
                        hx[i][k] *= rstd;
                        hy[i][k] *= rstd;
                        gwx[i][k] += tx * hx[i][k];
                        gwy[i][k] += ty * hy[i][k];
                        ux[i][k] = tx * wx[i][k];
                        uy[i][k] = ty * wy[i][k];
                        sum += ux[i][k] * hx[i][k] + uy[i][k] * hy[i][k];
                    }
                }
                const float mean = head_sum(sum, a.lanes) * a.inv_cols;
                if (!live) continue;
                T* out = static_cast<T*>(q.out) + batch * q.out_batch + token * q.out_token + head * q.out_head;
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    if (sub + a.lanes * i >= a.vectors) continue;
#pragma unroll
                    for (int k = 0; k < V; ++k) {
                        ux[i][k] = rstd * (ux[i][k] - hx[i][k] * mean);
                        uy[i][k] = rstd * (uy[i][k] - hy[i][k] * mean);
                    }
                    from_pairs<V, NEXT>(ux[i], uy[i]);
                    store_vec<T, V>(out + col[i].a, ux[i]);
                    store_vec<T, V>(out + col[i].b, uy[i]);
                }
            }
        }
        if (!a.sums) continue;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < NV; ++i) {
#pragma unroll
            for (int k = 0; k < V; ++k)  // the warp's heads
                for (int o = 16; o >= a.lanes; o >>= 1) {
                    gwx[i][k] += __shfl_xor_sync(0xFFFFFFFFu, gwx[i][k], o);
                    gwy[i][k] += __shfl_xor_sync(0xFFFFFFFFu, gwy[i][k], o);
                }
            from_pairs<V, NEXT>(gwx[i], gwy[i]);
            if (slot == 0 && sub + a.lanes * i < a.vectors)
#pragma unroll
                for (int k = 0; k < V; ++k) {
                    s_sums[warp][col[i].a + k] = gwx[i][k];
                    s_sums[warp][col[i].b + k] = gwy[i][k];
                }
        }
        __syncthreads();
        if ((int)threadIdx.x < a.cols) {
            float s = 0.0f;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) s += s_sums[w][threadIdx.x];
            a.part[((long long)side * gridDim.x + blockIdx.x) * a.pitch + threadIdx.x] = s;
        }
    }
}

// ---------------------------------------------------------------------------
// host side

// CTAs of the backward pass: enough for every run of heads, no more than are resident.
int backward_ctas(long long rows, int sms) {
    const long long most = 2LL * sms;
    return (int)(rows < most ? rows : most);
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

template <typename T, int V, int NV, bool NEXT, bool KEPT>
int start(HeadArgs a, bool backward, int sms, int ctas, cudaStream_t st) {
    a.vectors = a.cols / 2 / V;
    a.lanes = 1;
    while (a.lanes < 32 && a.lanes < a.vectors) a.lanes *= 2;
    a.lane_groups = NEXT ? a.cols % kGroup == 0 : a.half % kGroup == 0 && (a.cols / 2 - a.half) % kGroup == 0;
    const int per = 32 / a.lanes;
    const int steps = (a.side[0].heads + per - 1) / per + (a.side[1].heads + per - 1) / per;
    // runs of up to eight steps, shorter ones while there are SMs without a CTA
    a.runs = (steps + 7) / 8;
    while (a.runs < steps && a.rows * a.runs < 2LL * sms * kWarps) a.runs = a.runs * 2 < steps ? a.runs * 2 : steps;
    if (backward) {
        head_norm_backward_kernel<T, V, NV, NEXT, KEPT><<<(unsigned)ctas, kThreads, 0, st>>>(a);
        return launched();
    }
    const long long blocks = (a.rows * a.runs + kWarps - 1) / kWarps;
    if (blocks > 0x7FFFFFFFLL) return AMPQ_ERR_TOO_LARGE;
    head_norm_forward_kernel<T, V, NV, NEXT, KEPT><<<(unsigned)blocks, kThreads, 0, st>>>(a);
    return launched();
}

template <typename T, bool NEXT, bool KEPT>
int pick(const HeadArgs& a, bool backward, int dtype, int sms, int ctas, cudaStream_t st) {
    constexpr int kWide = 16 / (int)sizeof(T);
    if (vectors_fit(a, dtype, kWide)) return start<T, kWide, 1, NEXT, KEPT>(a, backward, sms, ctas, st);
    if (vectors_fit(a, dtype, 2)) return start<T, 2, kHeadCols / 128, NEXT, KEPT>(a, backward, sms, ctas, st);
    return start<T, 1, kHeadCols / 64, NEXT, KEPT>(a, backward, sms, ctas, st);
}

template <typename T>
int dispatch(const HeadArgs& a, bool next, bool kept, bool backward, int dtype, int sms, int ctas, cudaStream_t st) {
    if (next) return kept ? pick<T, true, true>(a, backward, dtype, sms, ctas, st) : pick<T, true, false>(a, backward, dtype, sms, ctas, st);
    return kept ? pick<T, false, true>(a, backward, dtype, sms, ctas, st) : pick<T, false, false>(a, backward, dtype, sms, ctas, st);
}

HeadArgs head_args(int param_dtype, int index_type, int fmt, long long batch, long long tokens, long long cols, long long rot, const float* cos, const float* sin,
                   long long angles, const void* positions, long long position_batch, const ampq_heads* q, const ampq_heads* k, bool backward) {
    HeadArgs a{};
    a.side[0] = side_of(q, backward, fmt != AMPQ_FMT_BASE);
    a.side[1] = side_of(k, backward, fmt != AMPQ_FMT_BASE);
    a.cos = cos; a.sin = sin;
    a.positions = positions;
    a.rows = batch * tokens; a.tokens = tokens; a.angles = angles; a.position_batch = position_batch;
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
            if (s.heads > 0 && s.rstd && cudaMemsetAsync(s.rstd, 0xFF, (size_t)(a.rows * s.heads) * sizeof(float), st) != cudaSuccess) {
                cudaGetLastError();
                return AMPQ_ERR_CUDA;
            }
        return AMPQ_OK;
    }
    a.eps = eps;
    const bool kept = fmt != AMPQ_FMT_BASE;
    return dtype == AMPQ_F32 ? dispatch<float>(a, interleaved != 0, kept, false, dtype, sms, 0, st)
                             : dispatch<__nv_bfloat16>(a, interleaved != 0, kept, false, dtype, sms, 0, st);
}

int ampq_head_norm_backward_workspace(int device, long long batch, long long tokens, long long cols, long long* bytes) {
    if (!bytes || batch < 0 || tokens < 0 || cols < 0 || cols % 2) return AMPQ_ERR_INVALID;
    if (cols > kHeadCols || batch > kMaxRows || tokens > kMaxRows || batch * tokens > kMaxRows) return AMPQ_ERR_TOO_LARGE;
    CkptDevice cur(device);
    if (cur.status) return cur.status;
    const int sms = sm_count(device);
    if (sms < 1) return AMPQ_ERR_CUDA;
    *bytes = 2LL * backward_ctas(batch * tokens, sms) * part_pitch(cols) * (long long)sizeof(float);
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
    if (a.sums && ctas > 0 && (!workspace || workspace_bytes < 2LL * ctas * a.pitch * (long long)sizeof(float))) return AMPQ_ERR_INVALID;
    a.part = static_cast<float*>(workspace);
    cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
    const bool kept = fmt != AMPQ_FMT_BASE;
    if (a.rows > 0 && a.side[0].heads + a.side[1].heads > 0) {
        rc = dtype == AMPQ_F32 ? dispatch<float>(a, interleaved != 0, kept, true, dtype, sms, ctas, st)
                               : dispatch<__nv_bfloat16>(a, interleaved != 0, kept, true, dtype, sms, ctas, st);
        if (rc) return rc;
    }
    for (int s = 0; s < 2; ++s) {
        const ampq_heads* h = s ? k : q;
        if (!h || !h->gweight) continue;
        rc = launch_join_columns(a.part + (long long)s * ctas * a.pitch, 1, h->heads > 0 ? ctas : 0, cols, a.pitch, h->gweight, nullptr, param_dtype, st);
        if (rc) return rc;
    }
    return AMPQ_OK;
}

#pragma GCC visibility pop
}  // extern "C"
