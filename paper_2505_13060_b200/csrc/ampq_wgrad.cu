// Weight gradient of linear layers from the 8-bit checkpoint of their input
// (include/ampq.h: ampq_ckpt_weight_grad): for every sample r
//   gW[r][k][c] = sum_n gY[r][n][k] * X^[r][n][c],  gb[r][k] = sum_n gY[r][n][k].
//
// The product runs on the tensor cores (tcgen05, kind::f16, fp32 accumulators in
// TMEM).  Its reduction axis is the token n, along which neither operand is
// contiguous, so both are given to the tensor core "MN-major", 128-byte
// swizzled.  gY and the codes of X^ come in by TMA; eight warps widen the codes to
// bf16 (exact, see ampq_ckpt.h) from shared memory into the same swizzled layout:
// 33/32 byte per element of X from HBM and L2 instead of two, and no bf16 copy of
// X in memory.
//
// fp32 gradients are first cut into three bf16 planes, g = g0 + g1 + g2 exactly
// (24 significant bits), and the token axis walks all three: the products stay
// exact.
#include "ampq_ckpt.h"

#include <cuda.h>

#include <atomic>

namespace ampq {
namespace {

constexpr int kStepRows = 64;                 // tokens of one pipeline stage
constexpr int kCtaOuts = 128;                 // gradient columns (k) of one CTA's stage
constexpr int kCtaCols = 128;                 // checkpoint columns (c) of one CTA's stage
constexpr int kBoxBytes = kStepRows * 128;    // 64 tokens x 64 bf16
constexpr int kTileBytes = 2 * kBoxBytes;     // one operand of one stage: 128 x 64 bf16
constexpr int kCodeBytes = kStepRows * kCtaCols;  // the codes of one stage
constexpr int kStages = 6;                    // stages of what is loaded: gY, codes, scale bytes
constexpr int kWideStages = 4;                // stages of the widened codes
constexpr int kProducerWarp = 0, kMmaWarp = 1, kTmemWarp = 2, kScaleWarp = 3, kEpilogueWarp = 4, kDecodeWarp = 8;
constexpr int kEpilogueWarps = 4;
constexpr int kDecodeTeams = 2, kTeamWarps = 4;  // team i widens stages i, i + kDecodeTeams, ...
constexpr int kDecodeWarps = kDecodeTeams * kTeamWarps;
constexpr int kThreads = 32 * (kDecodeWarp + kDecodeWarps);
constexpr int kScaleBytes = 4 * kStepRows;       // their scale bytes, four a row
constexpr int kSmemBytes = kStages * (kTileBytes + kCodeBytes + kScaleBytes) + kWideStages * kTileBytes + 1024;

// Polls of an mbarrier before a wait gives up.  A test build lets the waits
// between the stages give up at once; the waits that drain copies and products
// in flight keep the full limit.
constexpr unsigned kDrainPolls = 1u << 22;
#ifdef AMPQ_TEST_SHORT_WAITS
constexpr unsigned kWaitPolls = 1u;
constexpr unsigned kWaitHintNs = 0u;
#else
constexpr unsigned kWaitPolls = 1u << 22;
constexpr unsigned kWaitHintNs = 2000u;
#endif

__device__ __forceinline__ unsigned smem_u32(const void* p) { return (unsigned)__cvta_generic_to_shared(p); }

__device__ __forceinline__ void mbar_init(unsigned bar, unsigned count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ bool mbar_poll(unsigned bar, unsigned parity, unsigned hint_ns) {
    unsigned ok;
    asm volatile(
        "{\n"
        ".reg .pred p;\n"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n"
        "selp.u32 %0, 1, 0, p;\n"
        "}\n"
        : "=r"(ok)
        : "r"(bar), "r"(parity), "r"(hint_ns)
        : "memory");
    return ok != 0;
}
// Waits for a phase; false when the limit runs out or the CTA has given up.
__device__ __forceinline__ bool mbar_wait(unsigned bar, unsigned parity, volatile int* gave_up) {
    if (mbar_poll(bar, parity, kWaitHintNs)) return true;
    for (unsigned i = 0; i < kWaitPolls; ++i) {
        if (*gave_up) return false;
        if (mbar_poll(bar, parity, kWaitHintNs)) return true;
    }
    *gave_up = 1;
    return false;
}
__device__ __forceinline__ void mbar_drain(unsigned bar, unsigned parity) {
    for (unsigned i = 0; i < kDrainPolls; ++i)
        if (mbar_poll(bar, parity, 2000u)) return;
}
// Address of the same shared-memory variable in CTA `rank` of the cluster.
__device__ __forceinline__ unsigned in_cta(unsigned addr, unsigned rank) {
    unsigned r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
__device__ __forceinline__ void mbar_arrive(unsigned bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void mbar_arrive_cluster(unsigned cluster_bar) {
    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(cluster_bar) : "memory");
}
__device__ __forceinline__ void mbar_expect(unsigned bar, unsigned bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void tma_load(unsigned dst, const CUtensorMap* map, unsigned bar, int k, int n, int r, int plane) {
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];" ::"r"(dst),
        "l"(map), "r"(bar), "r"(k), "r"(n), "r"(r), "r"(plane)
        : "memory");
}
__device__ __forceinline__ void tma_load_codes(unsigned dst, const CUtensorMap* map, unsigned bar, int c, int n, int r) {
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(dst),
                 "l"(map), "r"(bar), "r"(c), "r"(n), "r"(r)
                 : "memory");
}
__device__ __forceinline__ void fence_tcgen05_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_tcgen05_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }

template <int CG>
__device__ __forceinline__ void tcgen05_commit(unsigned bar) {  // arrives when the products issued so far are done; CG = 2: in both CTAs
    if (CG == 1)
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
    else
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar),
                     "h"((unsigned short)3)
                     : "memory");
}

template <int CG>
__device__ __forceinline__ void tcgen05_mma(unsigned tmem, unsigned long long a, unsigned long long b, unsigned idesc, bool accumulate) {
    if (CG == 1)
        asm volatile(
            "{\n"
            ".reg .pred p;\n"
            "setp.ne.b32 p, %4, 0;\n"
            "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n"
            "}\n" ::"r"(tmem),
            "l"(a), "l"(b), "r"(idesc), "r"((unsigned)accumulate)
            : "memory");
    else
        asm volatile(
            "{\n"
            ".reg .pred p;\n"
            "setp.ne.b32 p, %4, 0;\n"
            "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n"
            "}\n" ::"r"(tmem),
            "l"(a), "l"(b), "r"(idesc), "r"((unsigned)accumulate)
            : "memory");
}

__device__ __forceinline__ void tmem_load32(unsigned addr, float (&v)[32]) {
    unsigned r[32];
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
          "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]),
          "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]),
          "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(addr));
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(r[i]);
}

// Shared-memory descriptor of an operand tile: MN-major, 128-byte swizzle.
// Blocks of 64 elements of the non-reduced axis lie kBoxBytes apart (leading
// offset), groups of eight tokens 1024 bytes apart (stride offset).
__device__ __forceinline__ unsigned long long operand_desc(unsigned addr) {
    return (unsigned long long)((addr & 0x3FFFFu) >> 4) | ((unsigned long long)(kBoxBytes >> 4) << 16) |
           ((unsigned long long)(1024 >> 4) << 32) | (1ull << 46) | (2ull << 61);
}

struct WgradArgs {
    const unsigned char* scales;
    void* out;                                // gw, or fp32 partial sums [samples][splits][outs][cols]
    long long ld_scales, cols, outs, rows;
    long long tiles;                          // (sample, split, k tile, c tile)
    int k_tiles, c_tiles, splits, steps_per_plane, steps, steps_per_split;
    bool scale_words;                         // rows of scale bytes start on 4-byte boundaries
    bool vec;                                 // rows of the output start on 16-byte boundaries
};

// A tile of the output: which sample, which part of the token axis, which corner.
struct TilePos {
    int sample, split, kt, ct, first_step, last_step;
    __device__ __forceinline__ TilePos(const WgradArgs& a, long long t) {
        const int per = a.k_tiles * a.c_tiles;
        const long long group = t / per;
        const int in = (int)(t - group * per);
        sample = (int)(group / a.splits);
        split = (int)(group - (long long)sample * a.splits);
        // eight k tiles at a time, so that the tiles in flight share rows and columns in L2
        const int band = in / (8 * a.c_tiles), w = in - band * 8 * a.c_tiles;
        const int height = min(8, a.k_tiles - band * 8);
        kt = band * 8 + w % height;
        ct = w / height;
        first_step = split * a.steps_per_split;
        last_step = min(a.steps, first_step + a.steps_per_split);
    }
};

__device__ __forceinline__ unsigned mul_bf16x2(unsigned a, unsigned b) {
    unsigned r;
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}

// Four codes -> four bf16 values, in the order 0, 2, 1, 3.  A code moved into the
// upper byte of a 16-bit half and shifted right by four (three) has its exponent
// and mantissa fields at the low end of bf16's, subnormal codes among bf16's
// subnormals: the value times 2^-120 (E4M3) or 2^-112 (E5M2).  One exact product
// with `unit` puts that and the group's scale right.
template <int FMT>
__device__ __forceinline__ uint2 widen4(unsigned w, unsigned unit) {
    constexpr unsigned kField = FMT == AMPQ_FMT_E4M3 ? 0x07F007F0u : 0x0FE00FE0u;
    constexpr int kShift = FMT == AMPQ_FMT_E4M3 ? 4 : 3;
    const unsigned even = ((w << (8 - kShift)) & kField) | ((w << 8) & 0x80008000u);
    const unsigned odd = ((w >> kShift) & kField) | (w & 0x80008000u);
    return make_uint2(mul_bf16x2(even, unit), mul_bf16x2(odd, unit));
}

// Sixteen codes of one group -> two 16-byte pieces of a row.  byte: the scale, or
// 0 where there is no row, which decodes to 0.
template <int FMT>
__device__ __forceinline__ void widen16(uint4 q, unsigned byte, uint4& lo, uint4& hi) {
    const unsigned field = byte ? byte + (FMT == AMPQ_FMT_E4M3 ? 120u : 112u) : 0u;  // bf16 exponent field of the factor
    const unsigned unit = (min(field, 254u) << 7) * 0x10001u;
    const uint2 a = widen4<FMT>(q.x, unit), b = widen4<FMT>(q.y, unit), c = widen4<FMT>(q.z, unit), d = widen4<FMT>(q.w, unit);
    lo = make_uint4(a.x, a.y, b.x, b.y);
    hi = make_uint4(c.x, c.y, d.x, d.y);
    if (field > 254u) {  // a scale above 2^7 (2^15): the factor is no bf16 number, its second part follows; NaN for the NaN byte
        const unsigned rest = (byte == kNanScale ? 0x7FC0u : (field - 127u) << 7) * 0x10001u;
        lo = make_uint4(mul_bf16x2(lo.x, rest), mul_bf16x2(lo.y, rest), mul_bf16x2(lo.z, rest), mul_bf16x2(lo.w, rest));
        hi = make_uint4(mul_bf16x2(hi.x, rest), mul_bf16x2(hi.y, rest), mul_bf16x2(hi.z, rest), mul_bf16x2(hi.w, rest));
    }
}

// The scale bytes of a CTA's stages, one after the other through all of its
// tiles: one lane's rows n and n + 32, the four groups of the CTA's 128 columns in
// one word.  0 (decodes to 0) where there is no row or no column.
template <int CG>
struct ScaleWalk {
    long long t;
    const unsigned char* p;
    int step, last_step, plane_step, groups;
    long long n;
    __device__ __forceinline__ void open(const WgradArgs& a, long long tile, unsigned rank, unsigned lane) {
        t = tile;
        if (t >= a.tiles) return;
        const TilePos pos(a, t);
        step = pos.first_step;
        last_step = pos.last_step;
        plane_step = step % a.steps_per_plane;
        n = (long long)plane_step * kStepRows + lane;
        const long long group = (long long)pos.ct * (CG * kCtaCols / kGroup) + rank * (kCtaCols / kGroup);
        groups = (int)max(0LL, min(4LL, (a.cols + kGroup - 1) / kGroup - group));
        p = a.scales + (pos.sample * a.rows + n) * a.ld_scales + group;
    }
    __device__ __forceinline__ unsigned word(const unsigned char* q, bool words) const {
        if (words && groups == 4) return __ldg(reinterpret_cast<const unsigned*>(q));
        unsigned w = 0;
#pragma unroll
        for (int g = 0; g < 4; ++g)
            if (g < groups) w |= (unsigned)__ldg(q + g) << (8 * g);
        return w;
    }
    __device__ __forceinline__ void fetch(const WgradArgs& a, unsigned (&w)[2]) const {
        w[0] = n < a.rows ? word(p, a.scale_words) : 0u;
        w[1] = n + 32 < a.rows ? word(p + 32 * a.ld_scales, a.scale_words) : 0u;
    }
    __device__ __forceinline__ void next(const WgradArgs& a, long long tile_stride, unsigned rank, unsigned lane) {
        if (++step == last_step) {
            open(a, t + tile_stride, rank, lane);
            return;
        }
        n += kStepRows;
        p += kStepRows * a.ld_scales;
        if (++plane_step == a.steps_per_plane) {  // the next plane of the gradient meets the same rows
            plane_step = 0;
            n = lane;
            p -= (long long)a.steps_per_plane * kStepRows * a.ld_scales;
        }
    }
};

template <typename OUT>
__device__ __forceinline__ void store_row(OUT* p, const float (&v)[32], long long n, bool vec) {
    if (vec && n >= 32) {
#pragma unroll
        for (int i = 0; i < 32; i += 8) {
            float w[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) w[j] = v[i + j];
            Raw8<OUT> r;
            r.set(w);
            r.store(p + i);
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 32; ++i)
        if (i < n) store_elem(p + i, v[i]);
}

// A persistent grid of CTAs (CG = 1) or CTA pairs (CG = 2) walks the tiles.  CG =
// 2: one 256 x 256 tile per pair, products issued by the pair's first CTA; each
// CTA holds 128 rows and 128 columns of the operands and 128 rows of the
// accumulators.  CG = 1: one 128 x 128 tile per CTA.  Two accumulators, so that a
// tile is stored while the next one is computed.
//
// Barriers, per stage: `loaded` (gY and the codes have landed), `scaled` (the
// scale bytes), `decoded` (X^ is written), for the own CTA; `peer` (both are in place in the pair's second CTA; held by the
// first); `empty` (the products that read the stage are done).  Per accumulator:
// `filled`, `drained`.  What the second CTA's warps wrote is read by the tensor
// core alone, for which the proxy fence before their arrival makes it visible; the
// arrival itself does not release at cluster scope, which would wait for every
// load in flight (1.5 us a stage).
//
// A wait that runs out raises the CTA's flag; its threads then leave their loops,
// the copies and products in flight are waited for, and what was not stored yet
// becomes NaN.
template <int CG, int FMT, typename OUT>
__global__ void __launch_bounds__(kThreads, 1) wgrad_kernel(const __grid_constant__ CUtensorMap map, const __grid_constant__ CUtensorMap code_map, const WgradArgs a) {
    extern __shared__ unsigned char raw_smem[];
    __shared__ alignas(8) unsigned long long s_bars[5 * kStages + 5];
    __shared__ unsigned s_tmem;
    __shared__ int s_gave_up;
    constexpr int kTileOuts = CG * kCtaOuts, kTileCols = CG * kCtaCols;
    constexpr unsigned kTmemCols = 2 * kTileCols;
    const unsigned warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    unsigned rank = 0;
    if (CG == 2) asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    const unsigned base = (smem_u32(raw_smem) + 1023u) & ~1023u;
    const unsigned tiles_a = base, tiles_b = base + kStages * kTileBytes, tiles_q = tiles_b + kWideStages * kTileBytes,
                   tiles_s = tiles_q + kStages * kCodeBytes;
    const unsigned bars = smem_u32(s_bars);
    auto loaded = [&](unsigned s) { return bars + 8 * s; };
    auto decoded = [&](unsigned s) { return bars + 8 * (kStages + s); };
    auto peer = [&](unsigned s) { return bars + 8 * (2 * kStages + s); };
    auto empty = [&](unsigned s) { return bars + 8 * (3 * kStages + s); };
    auto scaled = [&](unsigned s) { return bars + 8 * (4 * kStages + s); };
    auto filled = [&](unsigned k) { return bars + 8 * (5 * kStages + k); };
    auto drained = [&](unsigned k) { return bars + 8 * (5 * kStages + 2 + k); };
    const unsigned finished = bars + 8 * (5 * kStages + 4);
    volatile int* gave_up = &s_gave_up;

    if (threadIdx.x == 0) {
        for (unsigned s = 0; s < kStages; ++s) {
            mbar_init(loaded(s), 1);
            mbar_init(scaled(s), 1);
            mbar_init(decoded(s), kTeamWarps);
            mbar_init(peer(s), kTeamWarps);
            mbar_init(empty(s), 1);
        }
        for (unsigned k = 0; k < 2; ++k) {
            mbar_init(filled(k), 1);
            mbar_init(drained(k), CG * kEpilogueWarps);
        }
        mbar_init(finished, 1);
        s_gave_up = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == kTmemWarp) {
        if (CG == 1)
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&s_tmem)), "r"(kTmemCols) : "memory");
        else
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&s_tmem)), "r"(kTmemCols) : "memory");
        fence_tcgen05_before();
    }
    __syncthreads();
    if (CG == 2) {
        asm volatile("barrier.cluster.arrive.release;\nbarrier.cluster.wait.acquire;" ::: "memory");
    }
    fence_tcgen05_after();
    const unsigned tmem = s_tmem;

    const long long first_tile = blockIdx.x / CG, tile_stride = gridDim.x / CG;

    if (warp == kProducerWarp) {
        if (lane == 0) {
            unsigned stage = 0, parity = 0;
            unsigned pending = 0;  // loads issued, at most kStages of them not yet known to have landed
            bool ok = true;
            for (long long t = first_tile; t < a.tiles && ok; t += tile_stride) {
                const TilePos p(a, t);
                const int k0 = p.kt * kTileOuts + (int)rank * kCtaOuts, c0 = p.ct * kTileCols + (int)rank * kCtaCols;
                for (int step = p.first_step; step < p.last_step; ++step) {
                    ok = mbar_wait(empty(stage), parity ^ 1, gave_up);
                    if (!ok) break;
                    const int plane = step / a.steps_per_plane, n0 = (step - plane * a.steps_per_plane) * kStepRows;
                    mbar_expect(loaded(stage), kTileBytes + kCodeBytes);
                    tma_load_codes(tiles_q + stage * kCodeBytes, &code_map, loaded(stage), c0, n0, p.sample);
                    tma_load(tiles_a + stage * kTileBytes, &map, loaded(stage), k0, n0, p.sample, plane);
                    tma_load(tiles_a + stage * kTileBytes + kBoxBytes, &map, loaded(stage), k0 + 64, n0, p.sample, plane);
                    ++pending;
                    if (++stage == kStages) {
                        stage = 0;
                        parity ^= 1;
                    }
                }
            }
            // no copy of this CTA is in flight when it ends
            for (unsigned k = 0; k < kStages && k < pending; ++k) {
                if (stage == 0) {
                    stage = kStages;
                    parity ^= 1;
                }
                --stage;
                mbar_drain(loaded(stage), parity);
            }
        }
    } else if (warp == kMmaWarp) {
        if (rank == 0 && lane == 0) {
            // fp32 accumulators, bf16 operands, both MN-major
            constexpr unsigned kIdesc = (1u << 4) | (1u << 7) | (1u << 10) | (1u << 15) | (1u << 16) | ((unsigned)(kTileCols / 8) << 17) |
                                        ((unsigned)(kTileOuts / 16) << 24);
            unsigned stage = 0, parity = 0, wide = 0, acc = 0, acc_parity = 0;
            bool ok = true;
            for (long long t = first_tile; t < a.tiles && ok; t += tile_stride) {
                const TilePos p(a, t);
                ok = mbar_wait(drained(acc), acc_parity ^ 1, gave_up);
                if (!ok) break;
                fence_tcgen05_after();
                for (int step = p.first_step; step < p.last_step; ++step) {
                    ok = mbar_wait(loaded(stage), parity, gave_up) && mbar_wait(decoded(stage), parity, gave_up);
                    if (CG == 2) ok = ok && mbar_wait(peer(stage), parity, gave_up);
                    if (!ok) break;
                    fence_tcgen05_after();
                    const unsigned long long da = operand_desc(tiles_a + stage * kTileBytes), db = operand_desc(tiles_b + wide * kTileBytes);
#pragma unroll
                    for (int i = 0; i < kStepRows / 16; ++i)  // 16 tokens: two groups of eight, 2048 bytes
                        tcgen05_mma<CG>(tmem + acc * kTileCols, da + i * (2048 >> 4), db + i * (2048 >> 4), kIdesc, step > p.first_step || i > 0);
                    tcgen05_commit<CG>(empty(stage));
                    if (++wide == kWideStages) wide = 0;
                    if (++stage == kStages) {
                        stage = 0;
                        parity ^= 1;
                    }
                }
                if (!ok) break;
                tcgen05_commit<CG>(filled(acc));
                acc ^= 1;
                if (acc == 0) acc_parity ^= 1;
            }
            // every product has finished before the memory it reads and writes is given up
            asm volatile("tcgen05.commit.cta_group::%1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(finished), "n"(CG) : "memory");
            mbar_drain(finished, 0);
        }
    } else if (warp == kScaleWarp) {
        // the scale bytes of the stages, some stages ahead of where they go
        constexpr int kAhead = 4;
        unsigned w[kAhead][2];
        bool have[kAhead];
        ScaleWalk<CG> walk;
        walk.open(a, first_tile, rank, lane);
#pragma unroll
        for (int b = 0; b < kAhead; ++b) {
            have[b] = walk.t < a.tiles;
            if (have[b]) {
                walk.fetch(a, w[b]);
                walk.next(a, tile_stride, rank, lane);
            }
        }
        unsigned stage = 0, parity = 0;
        bool ok = true;
        while (have[0] && ok) {
#pragma unroll
            for (int b = 0; b < kAhead; ++b) {
                if (!have[b]) break;
                ok = __all_sync(0xFFFFFFFFu, mbar_wait(empty(stage), parity ^ 1, gave_up));
                if (!ok) break;
                const unsigned to = tiles_s + stage * kScaleBytes + lane * 4;
                asm volatile("st.shared.u32 [%0], %1;" ::"r"(to), "r"(w[b][0]) : "memory");
                asm volatile("st.shared.u32 [%0], %1;" ::"r"(to + 128), "r"(w[b][1]) : "memory");
                __syncwarp();
                if (lane == 0) mbar_arrive(scaled(stage));
                if (++stage == kStages) {
                    stage = 0;
                    parity ^= 1;
                }
                have[b] = walk.t < a.tiles;
                if (have[b]) {
                    walk.fetch(a, w[b]);
                    walk.next(a, tile_stride, rank, lane);
                }
            }
        }
    } else if (warp >= kEpilogueWarp && warp < kEpilogueWarp + kEpilogueWarps) {
        const unsigned quarter = warp - kEpilogueWarp;  // TMEM lanes 32 * quarter .. + 31 are this warp's
        unsigned acc = 0, acc_parity = 0;
        bool ok = true;
        for (long long t = first_tile; t < a.tiles; t += tile_stride) {
            const TilePos p(a, t);
            if (ok) ok = mbar_wait(filled(acc), acc_parity, gave_up);
            ok = __all_sync(0xFFFFFFFFu, ok);
            fence_tcgen05_after();
            const long long k = (long long)p.kt * kTileOuts + rank * kCtaOuts + quarter * 32 + lane;
            const long long c0 = (long long)p.ct * kTileCols;
            OUT* row = static_cast<OUT*>(a.out) + (((long long)p.sample * a.splits + p.split) * a.outs + k) * a.cols + c0;
            for (int c = 0; c < kTileCols && c0 + c < a.cols; c += 32) {
                float v[32];
                __syncwarp();
                if (ok) {
                    tmem_load32(tmem + acc * kTileCols + ((quarter * 32) << 16) + c, v);
                } else {
#pragma unroll
                    for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(0x7FC00000u);
                }
#pragma unroll
                for (int i = 0; i < 32; i += 4) {  // the decoding warps' order of columns
                    const float x = v[i + 1];
                    v[i + 1] = v[i + 2];
                    v[i + 2] = x;
                }
                if (k < a.outs) store_row(row + c, v, a.cols - c0 - c, a.vec);
            }
            fence_tcgen05_before();
            __syncwarp();
            if (ok && lane == 0) mbar_arrive_cluster(CG == 2 ? in_cta(drained(acc), 0) : drained(acc));
            acc ^= 1;
            if (acc == 0) acc_parity ^= 1;
        }
    } else if (warp >= kDecodeWarp) {
        // Eight threads to a row of 128 codes.  Chunk (8 bf16, 16 bytes) j of row n lies
        // at (j ^ (n & 7)) * 16 of the row's 128 bytes; the upper four of eight lanes
        // store their second chunk first, so that the eight meet all 32 banks.
        const unsigned team = (warp - kDecodeWarp) / kTeamWarps, d = threadIdx.x - 32 * (kDecodeWarp + team * kTeamWarps);
        const unsigned c16 = d % 8, row = d / 8;
        const unsigned swap = c16 / 4, j0 = c16 % 4 * 2;
        const unsigned at = tiles_b + swap * kBoxBytes + row * 128;
        const unsigned first = at + ((j0 + swap) ^ (row & 7)) * 16, second = at + ((j0 + 1 - swap) ^ (row & 7)) * 16;
        const unsigned from = tiles_q + row * kCtaCols + c16 * 16, scale_from = tiles_s + row * 4 + c16 / 2;
        constexpr unsigned kTeamRows = 4 * kTeamWarps;
        long long todo = 0;  // stages of this CTA
        for (long long t = first_tile; t < a.tiles; t += tile_stride) {
            const TilePos p(a, t);
            todo += p.last_step - p.first_step;
        }
        unsigned stage = team, parity = 0, wide = team;
        // the stage whose products used the same place for widened codes before: kWideStages back
        unsigned before = (kStages - kWideStages + team) % kStages, before_parity = team < kWideStages ? 1 : 0;
        static_assert(kDecodeTeams <= kWideStages && kWideStages < kStages, "a team's stages wrap once at a time");
        for (long long i = team; i < todo; i += kDecodeTeams) {
            const bool ok = mbar_wait(loaded(stage), parity, gave_up) && mbar_wait(scaled(stage), parity, gave_up) &&
                            (i < kWideStages || mbar_wait(empty(before), before_parity, gave_up));
            if (!__all_sync(0xFFFFFFFFu, ok)) break;
            const unsigned qs = from + stage * kCodeBytes, ss = scale_from + stage * kScaleBytes;
            const unsigned f = first + wide * kTileBytes, g = second + wide * kTileBytes;
#pragma unroll
            for (unsigned h = 0; h < kStepRows; h += kTeamRows) {
                uint4 q, lo, hi;
                unsigned byte;
                asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(q.x), "=r"(q.y), "=r"(q.z), "=r"(q.w) : "r"(qs + h * kCtaCols));
                asm volatile("ld.shared.u8 %0, [%1];" : "=r"(byte) : "r"(ss + h * 4));
                widen16<FMT>(q, byte, lo, hi);
                const uint4 s0 = swap ? hi : lo, s1 = swap ? lo : hi;
                asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(f + h * 128), "r"(s0.x), "r"(s0.y), "r"(s0.z), "r"(s0.w) : "memory");
                asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(g + h * 128), "r"(s1.x), "r"(s1.y), "r"(s1.z), "r"(s1.w) : "memory");
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) {
                if (rank == 0)
                    mbar_arrive(decoded(stage));
                else
                    mbar_arrive_cluster(in_cta(peer(stage), 0));
            }
            stage += kDecodeTeams;
            if (stage >= kStages) {
                stage -= kStages;
                parity ^= 1;
            }
            before += kDecodeTeams;
            if (before >= kStages) {
                before -= kStages;
                before_parity ^= 1;
            }
            wide += kDecodeTeams;
            if (wide >= kWideStages) wide -= kWideStages;
        }
    }

    __syncwarp();
    __syncthreads();
    if (CG == 2) {
        // no CTA of a pair ends, or gives up its TMEM, while the other still works
        asm volatile("barrier.cluster.arrive.release;\nbarrier.cluster.wait.acquire;" ::: "memory");
    }
    if (warp == kTmemWarp) {
        __syncwarp();
        fence_tcgen05_after();
        if (CG == 1) {
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
            asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
        } else {
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
            asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
        }
    }
}

// ---------------------------------------------------------------------------
// gradients that TMA cannot read as they lie

// fp32 -> three bf16 planes that add up to it exactly: the upper 8 significant
// bits, the next 8, the last 8.  A value that is not finite keeps its kind in the
// first plane and leaves the others 0.
__device__ __forceinline__ void cut3(float g, unsigned short (&h)[3]) {
    const unsigned u = __float_as_uint(g);
    if ((u & 0x7F800000u) == 0x7F800000u) {
        h[0] = (u & 0x7FFFFFu) ? 0x7FC0 : (unsigned short)(u >> 16);
        h[1] = h[2] = 0;
        return;
    }
    const float r1 = g - __uint_as_float(u & 0xFFFF0000u);
    const unsigned u1 = __float_as_uint(r1);
    const float r2 = r1 - __uint_as_float(u1 & 0xFFFF0000u);
    h[0] = (unsigned short)(u >> 16);
    h[1] = (unsigned short)(u1 >> 16);
    h[2] = (unsigned short)(__float_as_uint(r2) >> 16);
}

// Copies gY into rows of `pitch` (a multiple of 8) bf16, one plane for bf16, three
// for fp32.  One pair of columns per thread.
template <typename T>
__global__ void __launch_bounds__(256) lay_out_kernel(const T* __restrict__ g, long long ld, long long rows, long long cols, unsigned* __restrict__ out,
                                                      long long pitch) {
    const long long pair = (long long)blockIdx.x * 256 + threadIdx.x;
    if (2 * pair >= cols) return;
    const bool two = 2 * pair + 1 < cols;
    for (long long n = blockIdx.y; n < rows; n += gridDim.y) {
        const T* p = g + n * ld + 2 * pair;
        const long long at = (n * pitch) / 2 + pair;
        if (sizeof(T) == 2) {
            const unsigned short* q = reinterpret_cast<const unsigned short*>(p);
            out[at] = __ldg(q) | (two ? (unsigned)__ldg(q + 1) << 16 : 0u);
        } else {
            unsigned short lo[3], hi[3];
            cut3(load_elem(p), lo);
            cut3(two ? load_elem(p + 1) : 0.0f, hi);
#pragma unroll
            for (int k = 0; k < 3; ++k) out[at + k * (rows * pitch / 2)] = lo[k] | (unsigned)hi[k] << 16;
        }
    }
}

// ---------------------------------------------------------------------------
// partial sums

// out[r][i] = sum over the splits of part[r][s][i], in order.
template <typename T>
__global__ void __launch_bounds__(256) join_splits_kernel(const float* __restrict__ part, long long samples, int splits, long long n, T* __restrict__ out) {
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < samples * n; i += (long long)gridDim.x * 256) {
        const long long r = i / n;
        const float* p = part + r * splits * n + (i - r * n);
        float s = 0.0f;
        for (int k = 0; k < splits; ++k) s += __ldg(p + k * n);
        store_elem(out + i, s);
    }
}

// Partial column sums: block (x, y, r) sums rows y * 8 + lane, + 8 * gridDim.y, ... of
// sample r for 32 columns.
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

// Row parts of the column sums: about 64 rows to a thread.
int sum_parts(long long rows) {
    const long long p = (rows + 64 * kSumWays - 1) / (64 * kSumWays);
    return (int)(p < 1 ? 1 : p > 256 ? 256 : p);
}

// ---------------------------------------------------------------------------
// host side

struct Problem {
    int dtype;
    const void* gy;
    long long ld_gy, samples, rows, cols, outs;
    bool bias;
};

// How a product is run, and what its workspace holds: the copied gradient, the
// partial products, the partial column sums, each at a multiple of 256 bytes.
struct Plan {
    bool copy, pair;
    int planes, splits;
    long long pitch;
    int k_tiles, c_tiles, steps_per_plane, steps, steps_per_split;
    long long tiles;
    long long at_part, at_sums, bytes;
};

long long round_up(long long n, long long to) { return (n + to - 1) / to * to; }

Plan make_plan(const Problem& q, int sms) {
    Plan p;
    p.copy = q.dtype == AMPQ_F32 || !rows_aligned(q.gy, q.ld_gy, q.dtype);
    p.planes = q.dtype == AMPQ_F32 ? 3 : 1;
    p.pitch = p.copy ? round_up(q.outs, 8) : q.ld_gy;
    p.steps_per_plane = (int)((q.rows + kStepRows - 1) / kStepRows);
    p.steps = p.planes * p.steps_per_plane;
    const long long pairs = ((q.outs + 255) / 256) * ((q.cols + 255) / 256) * q.samples;
    p.pair = pairs * 2 >= sms;
    const int side = p.pair ? 256 : 128;
    p.k_tiles = (int)((q.outs + side - 1) / side);
    p.c_tiles = (int)((q.cols + side - 1) / side);
    const long long tiles = (long long)p.k_tiles * p.c_tiles * q.samples;
    const int units = p.pair ? sms / 2 : sms;
    // few tiles and many tokens: several parts of the token axis per tile, at least eight stages each
    long long splits = tiles > 0 && tiles < units ? units / tiles : 1;
    if (splits > p.steps / 8) splits = p.steps / 8;
    if (splits < 1) splits = 1;
    p.steps_per_split = p.steps > 0 ? (int)((p.steps + splits - 1) / splits) : 1;
    p.splits = p.steps > 0 ? (p.steps + p.steps_per_split - 1) / p.steps_per_split : 1;
    p.tiles = tiles * p.splits;
    long long at = 0;
    if (p.copy) at = round_up(2LL * p.planes * q.samples * q.rows * p.pitch, 256);
    p.at_part = at;
    if (p.splits > 1) at += round_up(4LL * q.samples * p.splits * q.outs * q.cols, 256);
    p.at_sums = at;
    if (q.bias) at += round_up(4LL * q.samples * sum_parts(q.rows) * q.outs, 256);
    p.bytes = at;
    return p;
}

using EncodeFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                              const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeFn encode_fn() {
    static std::atomic<EncodeFn> known{nullptr};
    EncodeFn f = known.load(std::memory_order_acquire);
    if (f) return f;
    void* p = nullptr;
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &found) != cudaSuccess ||
        found != cudaDriverEntryPointSuccess || !p) {
        cudaGetLastError();
        return nullptr;
    }
    f = reinterpret_cast<EncodeFn>(p);
    known.store(f, std::memory_order_release);
    return f;
}

// gY as [planes][samples][rows][outs]: 64 tokens x 64 columns per copy, zeros outside each sample.
int gradient_map(CUtensorMap* map, const void* base, const Problem& q, const Plan& p) {
    const EncodeFn encode = encode_fn();
    if (!encode) return AMPQ_ERR_CUDA;
    const unsigned long long row = 2ull * (unsigned long long)p.pitch;
    unsigned long long sample = row * (unsigned long long)q.rows, plane = sample * (unsigned long long)q.samples;
    if (q.samples == 1) sample = row;  // never stepped over
    if (p.planes == 1) plane = row;
    const unsigned long long limit = 1ull << 40;
    if (row >= limit || sample >= limit || plane >= limit) return AMPQ_ERR_TOO_LARGE;
    const cuuint64_t dims[4] = {(cuuint64_t)q.outs, (cuuint64_t)q.rows, (cuuint64_t)q.samples, (cuuint64_t)p.planes};
    const cuuint64_t strides[3] = {row, sample, plane};
    const cuuint32_t box[4] = {64, kStepRows, 1, 1}, one[4] = {1, 1, 1, 1};
    const CUresult rc = encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(base), dims, strides, box, one,
                               CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return rc == CUDA_SUCCESS ? AMPQ_OK : AMPQ_ERR_CUDA;
}

// The codes as [samples][rows][columns with codes]: 64 tokens x 128 columns per copy, zeros outside each sample.
int code_map_of(CUtensorMap* map, const unsigned char* codes, long long ld_codes, const Problem& q) {
    const EncodeFn encode = encode_fn();
    if (!encode) return AMPQ_ERR_CUDA;
    unsigned long long row = (unsigned long long)ld_codes, sample = row * (unsigned long long)q.rows;
    if (q.samples == 1) sample = row;  // never stepped over
    const unsigned long long limit = 1ull << 40;
    if (row >= limit || sample >= limit) return AMPQ_ERR_TOO_LARGE;
    const cuuint64_t dims[3] = {(cuuint64_t)round_up(q.cols, kGroup), (cuuint64_t)q.rows, (cuuint64_t)q.samples};
    const cuuint64_t strides[2] = {row, sample};
    const cuuint32_t box[3] = {kCtaCols, kStepRows, 1}, one[3] = {1, 1, 1};
    const CUresult rc = encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 3, const_cast<unsigned char*>(codes), dims, strides, box, one,
                               CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return rc == CUDA_SUCCESS ? AMPQ_OK : AMPQ_ERR_CUDA;
}

template <int CG, int FMT, typename OUT>
int launch_product(const CUtensorMap& map, const CUtensorMap& code_map, const WgradArgs& a, int device, int sms, cudaStream_t st) {
    constexpr int kMaxDevices = 64;
    static std::atomic<bool> prepared[kMaxDevices];  // the attribute is set once per device and kernel
    if (device >= kMaxDevices || !prepared[device].load(std::memory_order_acquire)) {
        if (cudaFuncSetAttribute(wgrad_kernel<CG, FMT, OUT>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBytes) != cudaSuccess) {
            cudaGetLastError();
            return AMPQ_ERR_CUDA;
        }
        if (device < kMaxDevices) prepared[device].store(true, std::memory_order_release);
    }
    const long long units = sms / CG;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(CG * (a.tiles < units ? a.tiles : units)));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = kSmemBytes;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = CG;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, wgrad_kernel<CG, FMT, OUT>, map, code_map, a) != cudaSuccess) {
        cudaGetLastError();
        return AMPQ_ERR_CUDA;
    }
    return AMPQ_OK;
}

template <int FMT, typename OUT>
int run_product(const CUtensorMap& map, const CUtensorMap& code_map, const WgradArgs& a, bool pair, int device, int sms, cudaStream_t st) {
    return pair ? launch_product<2, FMT, OUT>(map, code_map, a, device, sms, st) : launch_product<1, FMT, OUT>(map, code_map, a, device, sms, st);
}

template <typename T>
int lay_out(const Problem& q, const Plan& p, void* out, cudaStream_t st) {
    const long long rows = q.samples * q.rows, bx = (q.outs + 511) / 512;
    const unsigned by = (unsigned)(rows < 65535 ? rows : 65535);
    lay_out_kernel<T><<<dim3((unsigned)bx, by), 256, 0, st>>>(static_cast<const T*>(q.gy), q.ld_gy, rows, q.outs, static_cast<unsigned*>(out), p.pitch);
    return launched();
}

template <typename T>
int bias_grad(const Problem& q, void* gb, float* part, cudaStream_t st) {
    const int parts = sum_parts(q.rows);
    const unsigned bz = (unsigned)(q.samples < 65535 ? q.samples : 65535);
    column_sums_kernel<T><<<dim3((unsigned)((q.outs + kSumCols - 1) / kSumCols), parts, bz), dim3(kSumCols, kSumWays), 0, st>>>(
        static_cast<const T*>(q.gy), q.ld_gy, q.samples, q.rows, q.outs, part);
    const int rc = launched();
    return rc ? rc : launch_join_columns(part, q.samples, parts, q.outs, gb, nullptr, q.dtype, st);
}

int check_sizes(int dtype, long long samples, long long rows, long long cols, long long outs) {
    if (!known_dtype(dtype) || samples < 0 || rows < 0 || cols < 0 || outs < 0) return AMPQ_ERR_INVALID;
    if (cols > kMaxCols || outs > kMaxCols || samples > kMaxRows || rows > kMaxRows || (samples > 0 && rows > kMaxRows / samples)) return AMPQ_ERR_TOO_LARGE;
    // tiles of one sample are counted in 32 bits
    if (((outs + 127) / 128) * ((cols + 127) / 128) > 0x7FFFFFFFLL) return AMPQ_ERR_TOO_LARGE;
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
    const int sms = sm_count(device);
    if (sms < 2) return AMPQ_ERR_CUDA;
    *bytes = make_plan(Problem{dtype, gy, ld_gy, samples, rows, cols, outs, bias != 0}, sms).bytes;
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
    const int sms = sm_count(device);
    if (sms < 2) return AMPQ_ERR_CUDA;
    const Problem q{dtype, gy, ld_gy, samples, rows, cols, outs, gb != nullptr};
    const Plan p = make_plan(q, sms);
    if (p.bytes > 0 && (!workspace || workspace_bytes < p.bytes)) return AMPQ_ERR_INVALID;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
    unsigned char* ws = static_cast<unsigned char*>(workspace);
    if (rows == 0) {
        if (cols > 0 && cudaMemsetAsync(gw, 0, (size_t)(samples * outs * cols) * elem_bytes(dtype), st) != cudaSuccess) {
            cudaGetLastError();
            return AMPQ_ERR_CUDA;
        }
    } else if (cols > 0) {
        if (p.copy) {
            rc = dtype == AMPQ_F32 ? lay_out<float>(q, p, ws, st) : lay_out<__nv_bfloat16>(q, p, ws, st);
            if (rc) return rc;
        }
        CUtensorMap map, code_map;
        rc = gradient_map(&map, p.copy ? ws : gy, q, p);
        if (!rc) rc = code_map_of(&code_map, codes, ld_codes, q);
        if (rc) return rc;
        const bool partial = p.splits > 1, f32 = partial || dtype == AMPQ_F32;
        WgradArgs a;
        a.scales = scales;
        a.out = partial ? ws + p.at_part : gw;
        a.ld_scales = ld_scales;
        a.cols = cols;
        a.outs = outs;
        a.rows = rows;
        a.tiles = p.tiles;
        a.k_tiles = p.k_tiles;
        a.c_tiles = p.c_tiles;
        a.splits = p.splits;
        a.steps_per_plane = p.steps_per_plane;
        a.steps = p.steps;
        a.steps_per_split = p.steps_per_split;
        a.scale_words = aligned_to(scales, 4) && ld_scales % 4 == 0;
        a.vec = rows_aligned(a.out, cols, f32 ? AMPQ_F32 : AMPQ_BF16);
        if (fmt == AMPQ_FMT_E4M3)
            rc = f32 ? run_product<AMPQ_FMT_E4M3, float>(map, code_map, a, p.pair, device, sms, st) : run_product<AMPQ_FMT_E4M3, __nv_bfloat16>(map, code_map, a, p.pair, device, sms, st);
        else
            rc = f32 ? run_product<AMPQ_FMT_E5M2, float>(map, code_map, a, p.pair, device, sms, st) : run_product<AMPQ_FMT_E5M2, __nv_bfloat16>(map, code_map, a, p.pair, device, sms, st);
        if (rc) return rc;
        if (partial) {
            const long long n = outs * cols, blocks = (samples * n + 255) / 256;
            const unsigned grid = (unsigned)(blocks < 8LL * sms ? blocks : 8LL * sms);
            const float* part = reinterpret_cast<const float*>(ws + p.at_part);
            if (dtype == AMPQ_F32)
                join_splits_kernel<float><<<grid, 256, 0, st>>>(part, samples, p.splits, n, static_cast<float*>(gw));
            else
                join_splits_kernel<__nv_bfloat16><<<grid, 256, 0, st>>>(part, samples, p.splits, n, static_cast<__nv_bfloat16*>(gw));
            rc = launched();
            if (rc) return rc;
        }
    }
    if (!gb) return AMPQ_OK;
    float* part = reinterpret_cast<float*>(ws + p.at_sums);
    return dtype == AMPQ_F32 ? bias_grad<float>(q, gb, part, st) : bias_grad<__nv_bfloat16>(q, gb, part, st);
}

#pragma GCC visibility pop
}  // extern "C"
