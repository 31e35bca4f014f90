// Distillation from a teacher's top logits, forward and backward
// (include/ampq.h: ampq_distill_forward, ampq_distill_backward).
//
// With q = softmax(s / T) over a row of logits and p = softmax(t / T) over the
// row's entries,
//   loss = T^2 sum_k p_k (log p_k - log q_k)
//        = T^2 (sum_k p_k ((t_k - tmax) - (s_k - m)) / T + log(total / sum_k e_k)),
// m = max s, total = sum_j exp((s_j - m) / T), e_k = exp((t_k - tmax) / T), p_k = e_k / sum e.
// The forward pass reads the logits once, every thread with its own running sum; the
// backward pass reads them once more and writes the gradient once.
#include "ampq_decoder.h"

#include <cmath>
#include <type_traits>

namespace ampq {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
// vectors that a thread has in flight, and CTAs that share an SM
constexpr int kForwardAhead = 1, kForwardCtas = 8, kHighCtas = 4;
constexpr int kBackwardAhead = 1, kBackwardCtas = 6;
constexpr int kPartVectors = 8 * kThreads;           // of the gradient's part of a row
constexpr unsigned kPartColumns = 16 * kPartVectors;  // at most
constexpr int kFewEntries = 128;  // 100: 333 us compared, 358 us with bits; 256: 530 and 369 us (4096 rows of 128000)
// Above it the forward pass computes in 64 bits.  Rows of 1000, all listed, loss 0.12: in
// fp32 off by up to 4e-7 at T = 1, 1.4e-5 at 8, in 64 bits by its last rounding at any T;
// but 4096 x 128000 bf16 take 1177 us instead of 170.
constexpr float kHighT = 8.0f;
constexpr int kMaxParts = 8;                            // CTAs that share a row

// log2(e) / T in two parts.  Rounded to fp32 alone it is off by up to 2^-24 of itself,
// which moves every exponent of a row the same way: 4096 x 128000, T = 1, 7e-8 of the
// sums; with the rest what is left is the rounding of each exponent.  `hi` is
// rounded down and `lo` above 0, so that -Inf times both stays -Inf.
struct Factor {
    float hi, lo, slack;  // slack: 16 T log 2
    __device__ __forceinline__ float times(float d) const { return fmaf(d, hi, d * lo); }
    __device__ __forceinline__ float2 times(float2 d) const { return __ffma2_rn(d, make_float2(hi, hi), __fmul2_rn(d, make_float2(lo, lo))); }
};

struct DistillArgs {
    const void *logits, *indices, *teacher;
    const float* gl;
    float *loss, *stats;
    void* gs;
    long long rows, ld, ld_indices, ld_teacher, ld_gs, gl_stride;
    unsigned cols;
    int top, parts;
    float T, inv_T;
    Factor k;
    bool wide, teacher_bf16;
};

// A row as whole 32-byte vectors on 32-byte boundaries and the few elements before
// and behind them, so that rows that start anywhere are read at full width.
template <typename T>
struct Row {
    static constexpr unsigned E = 32 / sizeof(T);
    unsigned head, vectors, tail;
    __device__ __forceinline__ Row(const T* p, unsigned cols) {
        const unsigned over = (unsigned)(reinterpret_cast<uintptr_t>(p) & 31) / (unsigned)sizeof(T);
        head = min(over ? E - over : 0u, cols);
        vectors = (cols - head) / E;
        tail = cols - head - vectors * E;
    }
    __device__ __forceinline__ unsigned edge(unsigned i) const { return i < head ? i : vectors * E + i; }  // column of the i-th other element
    __device__ __forceinline__ unsigned first(unsigned part, unsigned parts) const { return (unsigned)((unsigned long long)vectors * part / parts); }
};

// Sum of exp((s - m) / T) over some of a row, and the largest s of them as m (-Inf for
// none, or NaN alone).  Stored as one word of 8 bytes.
struct alignas(8) Running {
    float m, sum;
    // The sum under a larger maximum.  expf has errors of either sign; exp2_fast is 5e-8 low
    // on average, and in a row's sum the errors of all the times that it is put under a
    // larger maximum add up: with exp2_fast for each of these, sums of 4096 x 128000 were 1.7e-7 low.
    __device__ __forceinline__ float under(float to, const Factor& k) const { return m == to ? sum : sum * expf(k.times(m - to) * 0.6931472f); }
    // Of `n` of them, in a fixed order.
    __device__ __forceinline__ static Running join(const Running* r, int n, const Factor& k) {
        Running all{r[0].m, 0.0f};
        for (int i = 1; i < n; ++i) all.m = fmaxf(all.m, r[i].m);
        for (int i = 0; i < n; ++i) all.sum += r[i].under(all.m, k);
        return all;
    }
    __device__ __forceinline__ void join_warp(const Factor& k) {
        float to = m;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) to = fmaxf(to, __shfl_xor_sync(0xFFFFFFFFu, to, o));
        sum = under(to, k);
        m = to;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
    }
};

// A thread's sum of exp((s - base) / T).  The base is a logit that need not be the
// largest: it is raised to one that is 16 T log 2 above it, so that terms stay below 2^16
// and few sums are ever put under another.
struct Terms {
    float base = 0.0f, limit = -INFINITY, top = -INFINITY, sum = 0.0f;
    __device__ __forceinline__ void raise(float to, const Factor& k) {
        top = fmaxf(top, to);
        if (to > limit) {
            sum = limit == -INFINITY ? sum * 0.0f : Running{base, sum}.under(to, k);  // nothing, or NaN
            base = to;
            limit = to + k.slack;
        }
    }
    __device__ __forceinline__ void add(float s, const Factor& k) {
        raise(s, k);
        sum += exp2_fast(k.times(s - base));
    }
    template <int N>
    __device__ __forceinline__ void add(const float2 (&v)[N], const Factor& k) {
        float most = v[0].x;
#pragma unroll
        for (int i = 0; i < N; ++i) asm("max.f32 %0, %0, %1, %2;" : "+f"(most) : "f"(v[i].x), "f"(v[i].y));
        raise(most, k);
        float2 s = make_float2(0.0f, 0.0f);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float2 d = k.times(__fadd2_rn(v[i], make_float2(-base, -base)));
            s = __fadd2_rn(s, make_float2(exp2_fast(d.x), exp2_fast(d.y)));
        }
        sum += s.x + s.y;
    }
    __device__ __forceinline__ Running under_top(const Factor& k) const {
        return Running{top, limit == -INFINITY ? sum : Running{base, sum}.under(top, k)};
    }
};

// The same at high temperatures, in 64 bits.  There all exponentials are near 1 and the
// loss is what is left of T^2 log(total): the sums are those of exp - 1, of `n` terms.
struct HighFactor {
    double inv_T;
    float slack;
    __device__ __forceinline__ double times(float s, float m) const { return ((double)s - (double)m) * inv_T; }
};
struct alignas(8) HighRunning {
    double sum;
    float m;
    int n;
    __device__ __forceinline__ double under(float to, const HighFactor& k) const {
        if (m == to) return sum;
        const double g = expm1(k.times(m, to));
        return sum + (sum + (double)n) * g;
    }
    __device__ __forceinline__ static HighRunning join(const HighRunning* r, int n, const HighFactor& k) {
        HighRunning all{0.0, r[0].m, 0};
        for (int i = 1; i < n; ++i) all.m = fmaxf(all.m, r[i].m);
        for (int i = 0; i < n; ++i) {
            all.sum += r[i].under(all.m, k);
            all.n += r[i].n;
        }
        return all;
    }
    __device__ __forceinline__ void join_warp(const HighFactor& k) {
        float to = m;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) to = fmaxf(to, __shfl_xor_sync(0xFFFFFFFFu, to, o));
        sum = under(to, k);
        m = to;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
            n += __shfl_xor_sync(0xFFFFFFFFu, n, o);
        }
    }
};
struct HighTerms {
    double sum = 0.0;
    float base = 0.0f, limit = -INFINITY, top = -INFINITY;
    int n = 0;
    __device__ __forceinline__ void raise(float to, const HighFactor& k) {
        top = fmaxf(top, to);
        if (to > limit) {
            if (limit != -INFINITY) sum = HighRunning{sum, base, n}.under(to, k);  // all before were -Inf (or NaN): -1 under any
            base = to;
            limit = to + k.slack;
        }
    }
    __device__ __forceinline__ void add(float s, const HighFactor& k) {
        raise(s, k);
        sum += expm1(k.times(s, base));
        ++n;
    }
    template <int N>
    __device__ __forceinline__ void add(const float2 (&v)[N], const HighFactor& k) {
        float most = v[0].x;
#pragma unroll
        for (int i = 0; i < N; ++i) asm("max.f32 %0, %0, %1, %2;" : "+f"(most) : "f"(v[i].x), "f"(v[i].y));
        raise(most, k);
#pragma unroll
        for (int i = 0; i < N; ++i) sum += expm1(k.times(v[i].x, base)) + expm1(k.times(v[i].y, base));
        n += 2 * N;
    }
    __device__ __forceinline__ HighRunning under_top(const HighFactor& k) const {
        return HighRunning{limit == -INFINITY ? sum : HighRunning{sum, base, n}.under(top, k), top, n};
    }
};

__device__ __forceinline__ float max_nan(float a, float b) {
    asm("max.NaN.f32 %0, %0, %1;" : "+f"(a) : "f"(b));
    return a;
}

// The list of a row in shared memory: column (kNone: no entry, `cols`: no column), the
// teacher's logit and the row's own.  Out of the registers that the streams need.
constexpr unsigned kNone = 0xFFFFFFFFu;
struct List {
    unsigned index[AMPQ_DISTILL_MAX_TOP];
    float t[AMPQ_DISTILL_MAX_TOP], s[AMPQ_DISTILL_MAX_TOP];
    // Thread by thread, each its own entries; whether one of them is there.
    __device__ __forceinline__ bool load(const DistillArgs& a, long long row) {
        bool any = false;
        for (int k = threadIdx.x; k < a.top; k += kThreads) {
            const long long j = load_index(a.indices, row * a.ld_indices + k, a.wide);
            const bool known = j < (long long)a.cols;  // a column that is not there: the row's loss is NaN
            index[k] = j < 0 ? kNone : known ? (unsigned)j : a.cols;
            t[k] = j < 0 ? -INFINITY : known ? load_param(a.teacher, row * a.ld_teacher + k, a.teacher_bf16) : NAN;
            any |= j >= 0;
        }
        return any;
    }
    // The row's logits at the thread's entries (of those that `mine` says).
    template <typename T, typename F>
    __device__ __forceinline__ void gather(const DistillArgs& a, const T* x, F mine) {
        for (int k = threadIdx.x; k < a.top; k += kThreads)
            if (index[k] < a.cols && mine(index[k])) s[k] = load_elem(x + index[k]);
    }
    // Largest t of the row; all threads call it, and each has its own entries.
    __device__ __forceinline__ float largest(const DistillArgs& a, float* red) const {
        float m = -INFINITY;
        for (int k = threadIdx.x; k < a.top; k += kThreads) m = max_nan(m, t[k]);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) m = max_nan(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
        if (threadIdx.x % 32 == 0) red[threadIdx.x / 32] = m;
        __syncthreads();
        m = red[0];
#pragma unroll
        for (int w = 1; w < kWarps; ++w) m = max_nan(m, red[w]);
        return m;
    }
};

// 32 bytes on a 32-byte boundary, read once.
__device__ __forceinline__ void load_vector(const void* p, unsigned (&w)[8]) {
    asm volatile("ld.global.nc.L1::no_allocate.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7])
                 : "l"(p));
}
__device__ __forceinline__ void store_vector(void* p, const unsigned (&w)[8]) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]),
                 "r"(w[6]), "r"(w[7])
                 : "memory");
}

// Sums over the CTA, in a fixed order; all threads call it.
template <typename F, int N>
__device__ __forceinline__ void block_sum(F (&s)[N], F (*red)[N]) {
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) s[n] += __shfl_xor_sync(0xFFFFFFFFu, s[n], o);
    if (threadIdx.x % 32 == 0)
#pragma unroll
        for (int n = 0; n < N; ++n) red[threadIdx.x / 32][n] = s[n];
    __syncthreads();
#pragma unroll
    for (int n = 0; n < N; ++n) {
        s[n] = 0;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) s[n] += red[w][n];
    }
}

__device__ __forceinline__ unsigned cluster_rank() {
    unsigned r;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}

// A row to a CTA, or to a cluster of `parts` CTAs where there are few rows; the parts'
// maxima and sums meet in the first CTA's shared memory.  Bound by HBM, with the
// exponentials' pipe close behind (4096 x 128000 bf16 167 to 184 us by board, 5.4 to 6.0
// TB/s; its exponentials alone 120 us; 2048 x 128000 fp32 153 us, 6.5 TB/s): the more warps
// the better, so one vector in flight a thread and eight CTAs an SM (three vectors and
// four CTAs 184 us, where these took 170; with six CTAs fp32 took 175).  The bf16 kernel
// spills 20 bytes behind its stream.  HIGH computes in 64 bits, bound by these (1177 us).
template <typename T, bool HIGH>
__global__ void __launch_bounds__(kThreads, HIGH ? kHighCtas : kForwardCtas) distill_forward_kernel(const DistillArgs a) {
    using K = Chunk<T>;
    using Sum = std::conditional_t<HIGH, HighRunning, Running>;
    using F = std::conditional_t<HIGH, double, float>;
    __shared__ List list;
    __shared__ Sum s_warps[kWarps];
    __shared__ Sum s_parts[kMaxParts];
    __shared__ float s_top[kWarps];
    __shared__ F s_sums[kWarps][HIGH ? 3 : 2];
    std::conditional_t<HIGH, HighFactor, Factor> factor;
    if constexpr (HIGH)
        factor = HighFactor{1.0 / (double)a.T, a.k.slack};
    else
        factor = a.k;
    const unsigned part = a.parts > 1 ? cluster_rank() : 0u;
    const long long row = a.parts > 1 ? blockIdx.x / (unsigned)a.parts : blockIdx.x;
    if (a.parts > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
    const T* x = static_cast<const T*>(a.logits) + row * a.ld;
    const Row<T> r(x, a.cols);
    const T* body = x + r.head;
    const unsigned end = r.first(part + 1, a.parts);
    unsigned v = r.first(part, a.parts) + threadIdx.x;
    // the first vectors are on their way while the list is looked at
    unsigned w[kForwardAhead][8];
    auto fetch = [&](unsigned from) {
#pragma unroll
        for (int u = 0; u < kForwardAhead; ++u)
            if (from + u * kThreads < end) load_vector(body + (size_t)(from + u * kThreads) * K::kElems, w[u]);
    };
    fetch(v);
    const bool used = __syncthreads_or(list.load(a, row));
    if (!used) {  // the same in every part
        if (part == 0 && threadIdx.x == 0) {
            a.loss[row] = 0.0f;
            a.stats[2 * row] = a.stats[2 * row + 1] = 0.0f;
        }
        if (a.parts > 1) asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
        return;
    }
    if (part == 0) list.gather(a, x, [](unsigned) { return true; });
    std::conditional_t<HIGH, HighTerms, Terms> terms;
    if (part == 0 && threadIdx.x < r.head + r.tail) terms.add(load_elem(x + r.edge(threadIdx.x)), factor);
    for (; v < end; v += kForwardAhead * kThreads) {
#pragma unroll
        for (int u = 0; u < kForwardAhead; ++u)
            if (v + u * kThreads < end) {
                K k;
                k.from_words(w[u]);
                const unsigned next = v + (kForwardAhead + u) * kThreads;
                if (next < end) load_vector(body + (size_t)next * K::kElems, w[u]);
                terms.add(k.v, factor);
            }
    }
    Sum run = terms.under_top(factor);
    run.join_warp(factor);
    if (threadIdx.x % 32 == 0) s_warps[threadIdx.x / 32] = run;
    __syncthreads();
    run = Sum::join(s_warps, kWarps, factor);
    if (a.parts > 1) {
        asm volatile("barrier.cluster.wait.aligned;" ::: "memory");  // the first CTA has begun
        if (threadIdx.x == 0) {
            static_assert(alignof(Sum) == 8 && sizeof(Sum) % 8 == 0, "the stores below");
            unsigned at = (unsigned)__cvta_generic_to_shared(&s_parts[part]), there;
            asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(there) : "r"(at));
            unsigned long long words[sizeof(Sum) / 8];
            memcpy(words, &run, sizeof(Sum));
#pragma unroll
            for (int i = 0; i < (int)sizeof(Sum) / 8; ++i)
                asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(there + 8 * i), "l"(words[i]) : "memory");
        }
        asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
        if (part != 0) return;
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
        run = Sum::join(s_parts, a.parts, factor);
    }
    const float tmax = list.largest(a, s_top);
    if constexpr (HIGH) {
        // with A and B the sums of exponentials of the list and of the row: sum p log(p / q) = sum p (a - b) + log(B / A)
        double sums[3] = {0.0, 0.0, 0.0};  // of exp(a) - 1, of exp(a) (a - b), entries
        for (int k = threadIdx.x; k < a.top; k += kThreads)
            if (list.index[k] != kNone) {
                const double d = factor.times(list.t[k], tmax), e = exp(d);
                sums[0] += expm1(d);
                if (e > 0.0) sums[1] += e * (d - factor.times(list.s[k], run.m));
                sums[2] += 1.0;
            }
        block_sum(sums, s_sums);
        if (threadIdx.x == 0) {
            const double listed = sums[2] + sums[0], more = ((double)a.cols - sums[2]) + (run.sum - sums[0]);
            a.loss[row] = (float)((double)a.T * (double)a.T * (sums[1] / listed + log1p(more / listed)));
            a.stats[2 * row] = run.m;
            a.stats[2 * row + 1] = (float)((double)a.cols + run.sum);
        }
    } else {
        float sums[2] = {0.0f, 0.0f};
        for (int k = threadIdx.x; k < a.top; k += kThreads)
            if (list.index[k] != kNone) {
                const float e = expf((list.t[k] - tmax) * a.inv_T);
                sums[0] += e;
                if (e > 0.0f) sums[1] += e * (((list.t[k] - tmax) - (list.s[k] - run.m)) * a.inv_T);  // p log(p / q) is 0 where p is
            }
        block_sum(sums, s_sums);
        if (threadIdx.x == 0) {
            a.loss[row] = a.T * a.T * (sums[1] / sums[0] + logf(run.sum / sums[0]));  // the logarithms' difference would lose more of it
            a.stats[2 * row] = run.m;
            a.stats[2 * row + 1] = run.sum;
        }
    }
}

// gs_j = gl T (q_j - sum of the p of the entries of column j); bound by HBM (4096 x
// 128000 bf16 322 to 331 us by board, 6.2 to 6.4 TB/s).  A CTA writes its part
// of a row by the formula's first term, and then once more the columns of the list
// that lie in it, by the whole formula: a barrier is between the two.  A column that
// is listed more than once is stored by its first entry, with the sum of all.  Few
// entries are compared with each other.  Of MANY each leaves a bit for its column, and
// who finds it there sets one that says so: compared with each other a thousand took
// 15 times the rest of the kernel, but the bits cost a short list 5 % of it.
// (With the bits the kernels spill up to 48 bytes at six CTAs an SM.  Lists of 64, 256 and
// 1000 at six and five: 323, 370 and 491 us; 340, 353 and 485 us.)
template <typename T, bool MANY>
__global__ void __launch_bounds__(kThreads, kBackwardCtas) distill_backward_kernel(const DistillArgs a) {
    using K = Chunk<T>;
    __shared__ List list;
    __shared__ float s_top[kWarps];
    __shared__ float s_sums[kWarps][1];
    __shared__ unsigned s_listed[MANY ? kPartColumns / 32 + 1 : 1], s_again[MANY ? kPartColumns / 32 + 1 : 1];
    if (MANY)  // seen by all behind the list's barrier
        for (int i = threadIdx.x; i < (int)kPartColumns / 32 + 1; i += kThreads) s_listed[i] = s_again[i] = 0;
    const unsigned part = blockIdx.x % (unsigned)a.parts;
    const long long row = blockIdx.x / (unsigned)a.parts;
    const T* x = static_cast<const T*>(a.logits) + row * a.ld;
    T* out = static_cast<T*>(a.gs) + row * a.ld_gs;
    const Row<T> r(x, a.cols);
    const unsigned begin = r.first(part, a.parts), end = r.first(part + 1, a.parts);
    const T* body = x + r.head;
    T* to = out + r.head;
    const bool alike = (reinterpret_cast<uintptr_t>(to) & 31) == 0;  // the gradient's row lies to the boundaries as the logits' does
    unsigned v = begin + threadIdx.x;
    unsigned w[kBackwardAhead][8];
#pragma unroll
    for (int u = 0; u < kBackwardAhead; ++u)
        if (v + u * kThreads < end) load_vector(body + (size_t)(v + u * kThreads) * K::kElems, w[u]);
    const bool used = __syncthreads_or(list.load(a, row));
    auto write = [&](unsigned at, const K& k) {
        if (alike) {
            unsigned o[8];
            k.to_words(o);
            store_vector(to + (size_t)at * K::kElems, o);
        } else {
            k.store(to + (size_t)at * K::kElems, K::kElems);
        }
    };
    if (!used) {
        K zero;
        zero.zero();
        if (part == 0 && threadIdx.x < r.head + r.tail) store_elem(out + r.edge(threadIdx.x), 0.0f);
        for (; v < end; v += kThreads) write(v, zero);
        return;
    }
    auto mine = [&](unsigned j) {  // a column of this part
        const unsigned at = (j - r.head) / K::kElems;
        return j >= r.head && at < r.vectors ? at >= begin && at < end : part == 0;
    };
    list.gather(a, x, mine);
    const float m = a.stats[2 * row], inv = 1.0f / a.stats[2 * row + 1];
    const float c = a.gl[row * a.gl_stride] * a.T, ci = c * inv;
    if (part == 0 && threadIdx.x < r.head + r.tail) {
        const unsigned j = r.edge(threadIdx.x);
        store_elem(out + j, exp2_fast(a.k.times(load_elem(x + j) - m)) * ci);
    }
    for (; v < end; v += kBackwardAhead * kThreads) {
#pragma unroll
        for (int u = 0; u < kBackwardAhead; ++u)
            if (v + u * kThreads < end) {
                K k;
                k.from_words(w[u]);
                const unsigned next = v + (kBackwardAhead + u) * kThreads;
                if (next < end) load_vector(body + (size_t)next * K::kElems, w[u]);
#pragma unroll
                for (int i = 0; i < K::kElems / 2; ++i) {
                    const float2 d = a.k.times(__fadd2_rn(k.v[i], make_float2(-m, -m)));
                    k.v[i] = __fmul2_rn(make_float2(exp2_fast(d.x), exp2_fast(d.y)), make_float2(ci, ci));
                }
                write(v + u * kThreads, k);
            }
    }
    const float tmax = list.largest(a, s_top);
    float sums[1] = {0.0f};
    for (int k = threadIdx.x; k < a.top; k += kThreads) {
        list.t[k] = list.index[k] != kNone ? expf((list.t[k] - tmax) * a.inv_T) : 0.0f;
        sums[0] += list.t[k];
    }
    block_sum(sums, s_sums);
    const float inv_sum = 1.0f / sums[0];
    auto place = [&](unsigned j) {  // a column's bit: those of the part's vectors, then the row's first and last ones
        const unsigned at = j - r.head, vectors = r.vectors * K::kElems;
        return j >= r.head && at < vectors ? at - begin * K::kElems : kPartColumns + (j < r.head ? j : 16 + at - vectors);
    };
    if (MANY) {
        for (int k = threadIdx.x; k < a.top; k += kThreads) {
            const unsigned j = list.index[k];
            if (j >= a.cols || !mine(j)) continue;
            const unsigned p = place(j);
            if (atomicOr(s_listed + p / 32, 1u << p % 32) >> p % 32 & 1) atomicOr(s_again + p / 32, 1u << p % 32);
        }
        __syncthreads();
    }
    for (int k = threadIdx.x; k < a.top; k += kThreads) {
        const unsigned j = list.index[k];
        if (j >= a.cols || !mine(j)) continue;
        float e = 0.0f;
        bool later = false;
        if (MANY && !(s_again[place(j) / 32] >> place(j) % 32 & 1)) {
            e = list.t[k];
        } else {
            for (int i = 0; i < a.top; ++i)
                if (list.index[i] == j) {
                    e += list.t[i];
                    later |= i < k;
                }
        }
        if (!later) store_elem(out + j, (exp2_fast(a.k.times(list.s[k] - m)) * inv - e * inv_sum) * c);
    }
}

int check_distill(int dtype, int teacher_dtype, int index_type, const void* logits, long long ld, long long rows, long long cols, const void* indices,
                  long long ld_indices, const void* teacher, long long ld_teacher, long long top, float temperature) {
    if (!known_dtype(dtype) || !known_dtype(teacher_dtype) || !known_index(index_type)) return AMPQ_ERR_INVALID;
    int rc = check_matrix(logits, rows, cols, ld, dtype);
    if (rc) return rc;
    if (top < 0 || ld_indices < top || ld_teacher < top) return AMPQ_ERR_INVALID;
    if (!(temperature >= 1.0f / 1048576.0f && temperature <= 1048576.0f)) return AMPQ_ERR_INVALID;
    if (rows > 0 && top > 0 && (!indices || !teacher)) return AMPQ_ERR_INVALID;
    if (top > AMPQ_DISTILL_MAX_TOP || ld_indices > (1LL << 40) || ld_teacher > (1LL << 40)) return AMPQ_ERR_TOO_LARGE;
    if (!aligned_to(indices, index_bytes(index_type)) || !aligned_to(teacher, elem_bytes(teacher_dtype))) return AMPQ_ERR_ALIGN;
    return AMPQ_OK;
}

DistillArgs distill_args(int teacher_dtype, int index_type, const void* logits, long long ld, long long rows, long long cols, const void* indices,
                         long long ld_indices, const void* teacher, long long ld_teacher, long long top, float temperature) {
    DistillArgs a{};
    a.logits = logits; a.indices = indices; a.teacher = teacher;
    a.rows = rows; a.ld = ld; a.ld_indices = ld_indices; a.ld_teacher = ld_teacher;
    a.cols = (unsigned)cols;
    a.top = (int)top;
    a.parts = 1;
    a.T = temperature;
    a.inv_T = 1.0f / temperature;
    const double k = 1.4426950408889634 / (double)temperature;
    a.k.hi = (float)k;
    if ((double)a.k.hi >= k) a.k.hi = std::nextafterf(a.k.hi, 0.0f);
    a.k.lo = (float)(k - (double)a.k.hi);
    a.k.slack = (float)(16.0 * 0.6931471805599453 * (double)temperature);
    a.wide = index_type == AMPQ_I64;
    a.teacher_bf16 = teacher_dtype == AMPQ_BF16;
    return a;
}

template <typename T, bool HIGH>
int launch_forward(DistillArgs a, int sms, cudaStream_t st) {
    // few rows are shared out while that gives every SM up to four CTAs, a part having two vectors a thread at least
    const long long vectors = (long long)a.cols / Row<T>::E;
    while (a.parts < kMaxParts && a.rows * a.parts * 2 <= 4LL * sms && vectors >= 4LL * kThreads * a.parts) a.parts *= 2;
    if (a.rows * a.parts > 0x7FFFFFFFLL) return AMPQ_ERR_TOO_LARGE;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(a.rows * a.parts));
    cfg.blockDim = dim3(kThreads);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)a.parts;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = a.parts > 1 ? 1 : 0;
    if (cudaLaunchKernelEx(&cfg, distill_forward_kernel<T, HIGH>, a) != cudaSuccess) {
        cudaGetLastError();
        return AMPQ_ERR_CUDA;
    }
    return launched();
}

template <typename T>
int launch_backward(DistillArgs a, cudaStream_t st) {
    // a part of a row: eight vectors a thread
    const long long vectors = (long long)a.cols / Row<T>::E;
    const long long parts = (vectors + kPartVectors - 1) / kPartVectors;
    a.parts = parts < 1 ? 1 : (int)parts;
    if (a.rows * a.parts > 0x7FFFFFFFLL) return AMPQ_ERR_TOO_LARGE;
    auto kernel = a.top > kFewEntries ? distill_backward_kernel<T, true> : distill_backward_kernel<T, false>;
    kernel<<<(unsigned)(a.rows * a.parts), kThreads, 0, st>>>(a);
    return launched();
}

}  // namespace
}  // namespace ampq

using namespace ampq;

extern "C" {
#pragma GCC visibility push(default)

int ampq_distill_forward(int device, void* cuda_stream, int dtype, int teacher_dtype, int index_type, const void* logits, long long ld, long long rows,
                         long long cols, const void* indices, long long ld_indices, const void* teacher, long long ld_teacher, long long top,
                         float temperature, float* loss, float* stats) {
    int rc = check_distill(dtype, teacher_dtype, index_type, logits, ld, rows, cols, indices, ld_indices, teacher, ld_teacher, top, temperature);
    if (rc) return rc;
    if (rows > 0 && (!loss || !stats)) return AMPQ_ERR_INVALID;
    if (!aligned_to(loss, 4) || !aligned_to(stats, 4)) return AMPQ_ERR_ALIGN;
    CkptDevice cur(device);
    if (cur.status) return cur.status;
    if (rows == 0) return AMPQ_OK;
    const int sms = sm_count(device);
    if (sms < 1) return AMPQ_ERR_CUDA;
    DistillArgs a = distill_args(teacher_dtype, index_type, logits, ld, rows, cols, indices, ld_indices, teacher, ld_teacher, top, temperature);
    a.loss = loss; a.stats = stats;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
    if (temperature > kHighT) return dtype == AMPQ_F32 ? launch_forward<float, true>(a, sms, st) : launch_forward<__nv_bfloat16, true>(a, sms, st);
    return dtype == AMPQ_F32 ? launch_forward<float, false>(a, sms, st) : launch_forward<__nv_bfloat16, false>(a, sms, st);
}

int ampq_distill_backward(int device, void* cuda_stream, int dtype, int teacher_dtype, int index_type, const float* gl, long long gl_stride,
                          const void* logits, long long ld, long long rows, long long cols, const void* indices, long long ld_indices, const void* teacher,
                          long long ld_teacher, long long top, const float* stats, float temperature, void* gs, long long ld_gs) {
    int rc = check_distill(dtype, teacher_dtype, index_type, logits, ld, rows, cols, indices, ld_indices, teacher, ld_teacher, top, temperature);
    if (!rc) rc = check_matrix(gs, rows, cols, ld_gs, dtype);
    if (rc) return rc;
    if (gl_stride < 0 || (rows > 0 && (!gl || !stats))) return AMPQ_ERR_INVALID;
    if (gl_stride > (1LL << 40)) return AMPQ_ERR_TOO_LARGE;
    if (!aligned_to(gl, 4) || !aligned_to(stats, 4)) return AMPQ_ERR_ALIGN;
    CkptDevice cur(device);
    if (cur.status) return cur.status;
    if (rows == 0 || cols == 0) return AMPQ_OK;
    DistillArgs a = distill_args(teacher_dtype, index_type, logits, ld, rows, cols, indices, ld_indices, teacher, ld_teacher, top, temperature);
    a.gl = gl; a.gl_stride = gl_stride;
    a.stats = const_cast<float*>(stats);
    a.gs = gs; a.ld_gs = ld_gs;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
    return dtype == AMPQ_F32 ? launch_backward<float>(a, st) : launch_backward<__nv_bfloat16>(a, st);
}

#pragma GCC visibility pop
}  // extern "C"
