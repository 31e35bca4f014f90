// Weight gradient of linear layers from the 8-bit checkpoint of their input
// (include/ampq.h: ampq_ckpt_weight_grad): for every sample r
//   gW[r][k][c] = sum_n gY[r][n][k] * X^[r][n][c],  gb[r][k] = sum_n gY[r][n][k].
//
// Large products run on the tensor cores (tcgen05, kind::f16, fp32 accumulators in
// TMEM).  The reduction axis is the token n, along which neither operand is
// contiguous, so both are given to the tensor core "MN-major", 128-byte swizzled,
// which is how TMA lays 64 tokens x 64 columns down.  X^ is widened to bf16
// (exactly, see ampq_ckpt.h) in one pass before the product: widening it on the
// way into shared memory, for each of the outs / 256 times that the product reads
// it, took the power and the issue slots that the tensor cores need (8192^3: 1200
// TFLOP/s against 1510 with the pass included).
//
// fp32 gradients are cut into three bf16 planes, g = g0 + g1 + g2 (24 significant
// bits, exact from 2^-110 up; below that what is smaller than 2^-133, bf16's last bit,
// is lost), and each 64 tokens are multiplied plane by plane, the smallest first.
//
// The tensor core's additions cut instead of rounding: 2.9e-8 per addition, all
// towards zero, 4e-5 over 8192 tokens of one sign and more than half a step of bf16
// over 2^20.  So the sum of each run of tokens is taken out of TMEM and added to the
// rest in registers, rounded to nearest: of 64 tokens for fp32, of kRunTokens for
// bf16, where up to so many tokens are one run.
//
// Small products (few tokens, few tiles) are one launch of plain fp32 arithmetic.
#include "ampq_ckpt.h"

#include <cuda.h>

#include <atomic>

namespace ampq {
namespace {

constexpr int kStepRows = 64;                 // tokens of one pipeline stage
constexpr int kCtaSide = 128;                 // columns of gY, and of X^, of one CTA's stage
constexpr int kBoxBytes = kStepRows * 128;    // 64 tokens x 64 bf16
constexpr int kTileBytes = 2 * kBoxBytes;     // one operand of one stage: 128 x 64 bf16
constexpr int kStages = 6;
// Tokens whose sum a bf16 gradient leaves to the tensor core: cut by 2e-5 of a sum of
// one sign, a hundredth of half a step of the output or less.  A kernel that adds runs
// up takes longer even where there is one run only (4 x 2048 x 4096 x 4096 268 us
// against 262, 2 x 4096 x 8192 x 28672 3.20 ms against 3.10; runs of 512 tokens 278 us
// and 3.44 ms), so it is used where there are several.
constexpr int kRunTokens = 4096;
constexpr int kProducerWarp = 0, kMmaWarp = 1, kTmemWarp = 2, kStoreWarp = 4;
constexpr int kPatch = 32 * 33;               // floats: a 32 x 32 patch of the output on its way out

// Four storing warps cover the 128 TMEM lanes, eight share the columns too: the
// running sums of fp32 gradients fit their registers, and rows off the 16-byte
// boundaries, which go out two bytes a lane, take half the time.
constexpr int kStoreWarps = 8;
constexpr int kThreads = 32 * (kStoreWarp + kStoreWarps);
constexpr int kSmemBytes = kStages * 2 * kTileBytes + kStoreWarps * kPatch * 4 + 1024;

// Polls of an mbarrier before a wait gives up.  A test build lets the waits
// between the stages give up at once; the wait that drains products in flight
// keeps the full limit.
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
__device__ __forceinline__ bool mbar_drain(unsigned bar, unsigned parity) {
    for (unsigned i = 0; i < kDrainPolls; ++i)
        if (mbar_poll(bar, parity, 2000u)) return true;
    return false;
}
// Address of the same shared-memory variable in CTA `rank` of the cluster.
__device__ __forceinline__ unsigned in_cta(unsigned addr, unsigned rank) {
    unsigned r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
__device__ __forceinline__ void mbar_arrive_cluster(unsigned cluster_bar) {
    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(cluster_bar) : "memory");
}
__device__ __forceinline__ void mbar_expect(unsigned bar, unsigned bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
// CG = 2: the bytes may be counted on a barrier of the pair's other CTA.
template <int CG>
__device__ __forceinline__ void tma_load(unsigned dst, const CUtensorMap* map, unsigned bar, int k, int n, int r, int plane) {
    if (CG == 2)
        asm volatile(
            "cp.async.bulk.tensor.4d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];" ::"r"(dst),
            "l"(map), "r"(bar), "r"(k), "r"(n), "r"(r), "r"(plane)
            : "memory");
    else
        asm volatile(
            "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];" ::"r"(dst),
        "l"(map), "r"(bar), "r"(k), "r"(n), "r"(r), "r"(plane)
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

__device__ __forceinline__ void tmem_load16(unsigned addr, float (&v)[16]) {
    unsigned r[16];
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
          "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(addr));
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = __uint_as_float(r[i]);
}

// Shared-memory descriptor of an operand tile: MN-major, 128-byte swizzle.
// Blocks of 64 elements of the non-reduced axis lie kBoxBytes apart (leading
// offset), groups of eight tokens 1024 bytes apart (stride offset).
__device__ __forceinline__ unsigned long long operand_desc(unsigned addr) {
    return (unsigned long long)((addr & 0x3FFFFu) >> 4) | ((unsigned long long)(kBoxBytes >> 4) << 16) |
           ((unsigned long long)(1024 >> 4) << 32) | (1ull << 46) | (2ull << 61);
}

struct ProductArgs {
    void* out;                                // gw, or fp32 partial sums [samples][splits][outs][cols]
    long long cols, outs;
    long long tiles;                          // (sample, split, k tile, c tile)
    int k_tiles, c_tiles, splits, steps, steps_per_split;  // steps: runs of 64 tokens
    bool vec;                                 // rows of the output start on 16-byte boundaries
};

// A tile of the output: which sample, which part of the token axis, which corner.
struct TilePos {
    int sample, split, kt, ct, first_step, last_step;
    __device__ __forceinline__ TilePos(const ProductArgs& a, long long t) {
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

// Stores 32 columns of 32 rows, lane l holding row l: from `row` for this lane,
// `rows` of them from lane 0 on and `n` columns exist.  Rows on 16-byte boundaries
// go out as they are held, 16 bytes a lane; others through a patch of shared
// memory, a row at a time, so that a warp still writes runs of 32 elements.
template <typename OUT>
__device__ __forceinline__ void store_patch(OUT* row, const float (&v)[32], long long rows, long long n, long long pitch, bool vec, float* patch, unsigned lane) {
    if (vec && n >= 32) {
        if ((long long)lane >= rows) return;
#pragma unroll
        for (int i = 0; i < 32; i += 8) {
            uint4* to = reinterpret_cast<uint4*>(row + i);
            if (sizeof(OUT) == 2) {
                to[0] = make_uint4(pack_bf16(v[i], v[i + 1]), pack_bf16(v[i + 2], v[i + 3]), pack_bf16(v[i + 4], v[i + 5]), pack_bf16(v[i + 6], v[i + 7]));
            } else {
                to[0] = make_uint4(__float_as_uint(v[i]), __float_as_uint(v[i + 1]), __float_as_uint(v[i + 2]), __float_as_uint(v[i + 3]));
                to[1] = make_uint4(__float_as_uint(v[i + 4]), __float_as_uint(v[i + 5]), __float_as_uint(v[i + 6]), __float_as_uint(v[i + 7]));
            }
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 32; ++i) patch[lane * 33 + i] = v[i];
    __syncwarp();
    OUT* first = row - (long long)lane * pitch + lane;
    if ((long long)lane < n) {
        const int m = (int)min(32LL, rows);
#pragma unroll 8
        for (int i = 0; i < m; ++i) store_elem(first + (long long)i * pitch, patch[i * 33 + lane]);
    }
    __syncwarp();
}

template <int CG>
__device__ __forceinline__ unsigned tmem_alloc(unsigned* where, unsigned warp, unsigned cols) {
    if (warp == kTmemWarp) {
        if (CG == 1)
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(where)), "r"(cols) : "memory");
        else
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(where)), "r"(cols) : "memory");
        fence_tcgen05_before();
    }
    __syncthreads();
    if (CG == 2) asm volatile("barrier.cluster.arrive.release;\nbarrier.cluster.wait.acquire;" ::: "memory");
    fence_tcgen05_after();
    return *where;
}

// All threads of the CTA, or of both CTAs of a pair, meet.
template <int CG>
__device__ __forceinline__ void meet() {
    __syncwarp();
    __syncthreads();
    if (CG == 2) asm volatile("barrier.cluster.arrive.release;\nbarrier.cluster.wait.acquire;" ::: "memory");
}

// The end of every thread of a CTA, after all have met: no CTA of a pair ends, or
// gives up its TMEM, while the other still works.
template <int CG>
__device__ __forceinline__ void tmem_free(unsigned tmem, unsigned warp, unsigned cols) {
    if (warp == kTmemWarp) {
        __syncwarp();
        fence_tcgen05_after();
        if (CG == 1) {
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
            asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(cols) : "memory");
        } else {
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
            asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(cols) : "memory");
        }
    }
}

// Where a producer stands when it ends: the position of its next stage in two turns
// of the ring, the stages issued (16 bits), and whether a wait of its CTA ran out.
__device__ __forceinline__ unsigned end_word(unsigned position, unsigned issued, bool gave_up) {
    return position | (issued & 0xFFFFu) << 8 | (gave_up ? 1u << 31 : 0u);
}

// Waits, with a limit, for the copies of stages that were loaded and never
// multiplied.  end[k]: where CTA k's producer stands; one thread of each CTA calls it,
// after all have met.  The bytes of a pair are counted together, so the CTA that is
// behind (by kStages at most: stages that were multiplied had come in both) first
// issues what it lacks, from the operands' first corner; nothing reads it.  The last
// use of every stage is then waited for: uses before that have been multiplied, and
// a stage never used passes at once.
template <int CG>
__device__ __noinline__ void drain_copies(const unsigned (&end)[2], unsigned rank, unsigned tiles_g, unsigned tiles_x, unsigned loaded, const CUtensorMap* g_map,
                                          const CUtensorMap* x_map) {
    const int ahead = CG == 2 ? (short)((end[1] >> 8) - (end[0] >> 8)) : 0;  // of CTA 1
    const int lacks = min(kStages, rank == 0 ? ahead : -ahead);
    for (int i = 0; i < lacks; ++i) {
        const unsigned stage = ((end[rank] & 0xFFu) + i) % kStages, to = stage * kTileBytes, bar = in_cta(loaded + 8 * stage, 0);
        if (rank == 0) mbar_expect(loaded + 8 * stage, CG * 2 * kTileBytes);
        for (unsigned half = 0; half < 2; ++half) {
            tma_load<CG>(tiles_g + to + half * kBoxBytes, g_map, bar, 0, 0, 0, 0);
            tma_load<CG>(tiles_x + to + half * kBoxBytes, x_map, bar, 0, 0, 0, 0);
        }
    }
    if (rank != 0) return;
    const unsigned next = end[ahead > 0 ? 1 : 0] & 0xFFu;
    for (unsigned j = 1; j <= kStages; ++j) {
        const unsigned at = (next + 2 * kStages - j) % (2 * kStages);
        if (!mbar_drain(loaded + 8 * (at % kStages), at / kStages)) return;
    }
}

// A persistent grid of CTAs (CG = 1) or CTA pairs (CG = 2) walks the tiles.  CG =
// 2: one 256 x 256 tile per pair, products issued by the pair's first CTA; each
// CTA holds 128 columns of both operands and 128 rows of the accumulators.  CG =
// 1: one 128 x 128 tile per CTA.  Two accumulators, so that one is read while the
// next is filled: one per tile (RUN = 0) or one per RUN steps of a tile.
//
// Barriers, per stage: `loaded` (both operands have landed, in both CTAs of a
// pair; held by the first), `empty` (the products that read the stage are done).
// Per accumulator: `filled`, `drained`.
//
// Bound by the tensor cores and, over more than a few ms, by the board's power:
// 8192^3 in bf16 (one run) 690 us (1590 TFLOP/s), 2 x 4096 x 8192 x 28672 2.57 ms (1500; a
// library's matrix product reaches 1613 in a burst and 1344 sustained), 4 x 2048 x 4096 x 4096 191 us (1440: 1024 tiles on 74 pairs).  fp32,
// three planes: 2048^3 52 us (330 of fp32 arithmetic).  Six stages or seven, bands
// of 4, 8 or 16 tiles: within 2 % of each other, but for bands of 4 (8 % slower at
// the largest size).
//
// A wait that runs out raises the CTA's flag; its threads then leave their loops,
// what was not stored yet becomes NaN, and the products and copies in flight are
// waited for, with a limit, before the CTA ends: the products by the warp that issues
// them, the copies once all threads have met (the producer may have ended by then,
// with its last stages loaded and never multiplied).
template <int CG, int PLANES, int RUN, typename OUT>
__global__ void __launch_bounds__(kThreads, 1) product_kernel(const __grid_constant__ CUtensorMap g_map, const __grid_constant__ CUtensorMap x_map, const ProductArgs a) {
    extern __shared__ unsigned char raw_smem[];
    __shared__ alignas(8) unsigned long long s_bars[2 * kStages + 5];
    __shared__ unsigned s_tmem, s_end[2];
    __shared__ unsigned s_position, s_issued;
    __shared__ int s_gave_up;
    constexpr int kSide = CG * kCtaSide;  // of the tile
    constexpr unsigned kTmemCols = 2 * kSide;
    const unsigned warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    unsigned rank = 0;
    if (CG == 2) asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    const unsigned base = (smem_u32(raw_smem) + 1023u) & ~1023u;
    const unsigned tiles_g = base, tiles_x = base + kStages * kTileBytes;
    const unsigned bars = smem_u32(s_bars);
    auto loaded = [&](unsigned s) { return bars + 8 * s; };
    auto empty = [&](unsigned s) { return bars + 8 * (kStages + s); };
    auto filled = [&](unsigned k) { return bars + 8 * (2 * kStages + k); };
    auto drained = [&](unsigned k) { return bars + 8 * (2 * kStages + 2 + k); };
    const unsigned finished = bars + 8 * (2 * kStages + 4);
    volatile int* gave_up = &s_gave_up;

    if (threadIdx.x == 0) {
        for (unsigned s = 0; s < kStages; ++s) {
            mbar_init(loaded(s), 1);
            mbar_init(empty(s), 1);
        }
        for (unsigned k = 0; k < 2; ++k) {
            mbar_init(filled(k), 1);
            mbar_init(drained(k), CG * kStoreWarps);
        }
        mbar_init(finished, 1);
        s_gave_up = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    const unsigned tmem = tmem_alloc<CG>(&s_tmem, warp, kTmemCols);
    const long long first_tile = blockIdx.x / CG, tile_stride = gridDim.x / CG;

    if (warp == kProducerWarp) {
        if (lane == 0) {
            unsigned stage = 0, parity = 0, issued = 0;
            bool ok = true;
            for (long long t = first_tile; t < a.tiles && ok; t += tile_stride) {
                const TilePos p(a, t);
                const int k0 = p.kt * kSide + (int)rank * kCtaSide, c0 = p.ct * kSide + (int)rank * kCtaSide;
                for (int step = p.first_step; step < p.last_step && ok; ++step) {
#pragma unroll 1
                    for (int plane = PLANES - 1; plane >= 0; --plane) {
                        ok = mbar_wait(empty(stage), parity ^ 1, gave_up);
                        if (!ok) break;
                        const unsigned to = stage * kTileBytes, bar = CG == 2 ? in_cta(loaded(stage), 0) : loaded(stage);
                        const int n0 = step * kStepRows;
                        if (rank == 0) mbar_expect(loaded(stage), CG * 2 * kTileBytes);
                        tma_load<CG>(tiles_g + to, &g_map, bar, k0, n0, p.sample, plane);
                        tma_load<CG>(tiles_g + to + kBoxBytes, &g_map, bar, k0 + 64, n0, p.sample, plane);
                        tma_load<CG>(tiles_x + to, &x_map, bar, c0, n0, p.sample, 0);
                        tma_load<CG>(tiles_x + to + kBoxBytes, &x_map, bar, c0 + 64, n0, p.sample, 0);
                        ++issued;
                        if (++stage == kStages) {
                            stage = 0;
                            parity ^= 1;
                        }
                    }
                }
            }
            s_position = stage + kStages * parity;
            s_issued = issued;
        }
    } else if (warp == kMmaWarp) {
        if (rank == 0 && lane == 0) {
            // fp32 accumulators, bf16 operands, both MN-major
            constexpr unsigned kIdesc = (1u << 4) | (1u << 7) | (1u << 10) | (1u << 15) | (1u << 16) | ((unsigned)(kSide / 8) << 17) | ((unsigned)(kSide / 16) << 24);
            unsigned stage = 0, parity = 0, acc = 0, acc_parity = 0;
            bool ok = true;
            for (long long t = first_tile; t < a.tiles && ok; t += tile_stride) {
                const TilePos p(a, t);
                for (int step = p.first_step; step < p.last_step && ok; ++step) {
                    const int in_run = RUN > 0 ? (step - p.first_step) % RUN : step - p.first_step;
                    if (in_run == 0) {
                        ok = mbar_wait(drained(acc), acc_parity ^ 1, gave_up);
                        if (!ok) break;
                        fence_tcgen05_after();
                    }
#pragma unroll 1
                    for (int plane = PLANES - 1; plane >= 0; --plane) {
                        ok = mbar_wait(loaded(stage), parity, gave_up);
                        if (!ok) break;
                        fence_tcgen05_after();
                        const unsigned long long dg = operand_desc(tiles_g + stage * kTileBytes), dx = operand_desc(tiles_x + stage * kTileBytes);
                        const bool more = in_run > 0 || plane < PLANES - 1;
#pragma unroll
                        for (int i = 0; i < kStepRows / 16; ++i)  // 16 tokens: two groups of eight, 2048 bytes
                            tcgen05_mma<CG>(tmem + acc * kSide, dg + i * (2048 >> 4), dx + i * (2048 >> 4), kIdesc, more || i > 0);
                        tcgen05_commit<CG>(empty(stage));
                        if (++stage == kStages) {
                            stage = 0;
                            parity ^= 1;
                        }
                    }
                    if (ok && ((RUN > 0 && in_run == RUN - 1) || step + 1 == p.last_step)) {
                        tcgen05_commit<CG>(filled(acc));
                        acc ^= 1;
                        if (acc == 0) acc_parity ^= 1;
                    }
                }
            }
            // every product has finished before the memory it reads and writes is given up
            asm volatile("tcgen05.commit.cta_group::%1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(finished), "n"(CG) : "memory");
            mbar_drain(finished, 0);
        }
    } else if (warp >= kStoreWarp) {
        constexpr int kCols = kSide / (kStoreWarps / 4);  // columns of this warp
        const unsigned quarter = warp % 4;                // TMEM lanes 32 * quarter .. + 31 are this warp's
        const unsigned from = warp < kStoreWarp + 4 ? 0 : kCols;
        float* patch = reinterpret_cast<float*>(raw_smem + (base - smem_u32(raw_smem)) + 2 * kStages * kTileBytes) + (warp - kStoreWarp) * kPatch;
        unsigned acc = 0, acc_parity = 0;
        bool ok = true;
        for (long long t = first_tile; t < a.tiles; t += tile_stride) {
            const TilePos p(a, t);
            const long long k0 = (long long)p.kt * kSide + rank * kCtaSide + quarter * 32, c0 = (long long)p.ct * kSide + from;
            OUT* row = static_cast<OUT*>(a.out) + (((long long)p.sample * a.splits + p.split) * a.outs + k0 + lane) * a.cols + c0;
            const unsigned lanes = tmem + ((quarter * 32) << 16) + from;
            if constexpr (RUN == 0) {
                if (ok) ok = mbar_wait(filled(acc), acc_parity, gave_up);
                ok = __all_sync(0xFFFFFFFFu, ok);
                fence_tcgen05_after();
                for (int c = 0; c < kCols && c0 + c < a.cols; c += 32) {
                    float v[32];
                    __syncwarp();
                    if (ok) {
                        tmem_load32(lanes + acc * kSide + c, v);
                    } else {
#pragma unroll
                        for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(0x7FC00000u);
                    }
                    store_patch(row + c, v, a.outs - k0, a.cols - c0 - c, a.cols, a.vec, patch, lane);
                }
                fence_tcgen05_before();
                __syncwarp();
                if (ok && lane == 0) mbar_arrive_cluster(CG == 2 ? in_cta(drained(acc), 0) : drained(acc));
                acc ^= 1;
                if (acc == 0) acc_parity ^= 1;
            } else {
                float sum[kCols / 32][32];
#pragma unroll
                for (int c = 0; c < kCols / 32; ++c)
#pragma unroll
                    for (int i = 0; i < 32; ++i) sum[c][i] = 0.0f;
                for (int step = p.first_step; step < p.last_step && ok; step += RUN) {
                    ok = __all_sync(0xFFFFFFFFu, mbar_wait(filled(acc), acc_parity, gave_up));
                    if (!ok) break;
                    fence_tcgen05_after();
#pragma unroll
                    for (int c = 0; c < kCols / 16; ++c) {
                        float v[16];
                        __syncwarp();
                        tmem_load16(lanes + acc * kSide + c * 16, v);
#pragma unroll
                        for (int i = 0; i < 16; ++i) sum[c / 2][c % 2 * 16 + i] += v[i];
                    }
                    fence_tcgen05_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive_cluster(CG == 2 ? in_cta(drained(acc), 0) : drained(acc));
                    acc ^= 1;
                    if (acc == 0) acc_parity ^= 1;
                }
#pragma unroll
                for (int c = 0; c < kCols / 32; ++c) {
                    if (!ok) {
#pragma unroll
                        for (int i = 0; i < 32; ++i) sum[c][i] = __uint_as_float(0x7FC00000u);
                    }
                    if (c0 + c * 32 < a.cols) store_patch(row + c * 32, sum[c], a.outs - k0, a.cols - c0 - c * 32, a.cols, a.vec, patch, lane);
                }
            }
        }
    }
    // the CTAs of a pair tell each other how they ended before they meet: the other one's memory is there that long
    __syncwarp();
    __syncthreads();
    if (threadIdx.x == 0) {
        const unsigned end = end_word(s_position, s_issued, s_gave_up);
        s_end[rank] = end;
        if (CG == 2) asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(in_cta(smem_u32(&s_end[rank]), rank ^ 1)), "r"(end) : "memory");
    }
    meet<CG>();
    if ((s_end[0] | (CG == 2 ? s_end[1] : 0u)) >> 31) {
        if (threadIdx.x == 0) drain_copies<CG>(s_end, rank, tiles_g, tiles_x, bars, &g_map, &x_map);
        meet<CG>();
    }
    tmem_free<CG>(tmem, warp, kTmemCols);
}

// ---------------------------------------------------------------------------
// small products

constexpr int kSmallSide = 64, kSmallStep = 32;

// A 64 x 64 tile of one sample's gradient per block, 32 tokens at a time
// through shared memory, fp32 products and sums.  The blocks of the first column
// of tiles also sum the columns of gY.  One launch, bound by its chain of loads: 8
// samples of 128 x 256 x 256 in fp32 10 us (12 us with sixteen tokens at a time).
template <typename T, int FMT>
__global__ void __launch_bounds__(256) small_product_kernel(const T* __restrict__ gy, long long ld_gy, const unsigned char* __restrict__ codes, long long ld_codes,
                                                            const unsigned char* __restrict__ scales, long long ld_scales, long long rows, long long cols,
                                                            long long outs, T* __restrict__ gw, T* __restrict__ gb) {
    __shared__ float sg[kSmallStep][kSmallSide + 4], sx[kSmallStep][kSmallSide + 4];
    const long long k0 = (long long)blockIdx.x * kSmallSide, c0 = (long long)blockIdx.y * kSmallSide, r = blockIdx.z;
    const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
    // this thread's part of a step: a token's gradient elements gk, gk + 8, ..., and eight of its codes
    const int n = threadIdx.x / 8, gk = threadIdx.x % 8, xc = threadIdx.x % 8 * 8;
    float g[8];
    uint2 x;
    unsigned byte;
    auto fetch = [&](long long n0) {
        const long long row = r * rows + n0 + n;
        const bool in = n0 + n < rows;
        const T* p = gy + row * ld_gy + k0;
#pragma unroll
        for (int i = 0; i < 8; ++i) g[i] = in && k0 + gk + 8 * i < outs ? load_elem(p + gk + 8 * i) : 0.0f;
        x = make_uint2(0, 0);
        byte = 127;
        if (in && c0 + xc < cols) {
            x = __ldg(reinterpret_cast<const uint2*>(codes + row * ld_codes + c0 + xc));
            byte = __ldg(scales + row * ld_scales + (c0 + xc) / kGroup);
        }
    };
    float acc[4][4] = {}, sum[4] = {};
    const bool bias = gb && blockIdx.y == 0 && tx == 0;
    fetch(0);
    for (long long n0 = 0; n0 < rows; n0 += kSmallStep) {
        __syncthreads();
        float v[8];
        decode8<FMT>(x, v);
        const float scale = scale_of(byte);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            sg[n][gk + 8 * i] = g[i];
            sx[n][xc + i] = v[i] * scale;
        }
        __syncthreads();
        if (n0 + kSmallStep < rows) fetch(n0 + kSmallStep);
#pragma unroll 16
        for (int m = 0; m < kSmallStep; ++m) {
            const float4 u = *reinterpret_cast<const float4*>(&sg[m][ty * 4]), w = *reinterpret_cast<const float4*>(&sx[m][tx * 4]);
            const float uu[4] = {u.x, u.y, u.z, u.w}, vv[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(uu[i], vv[j], acc[i][j]);
            if (bias)
#pragma unroll
                for (int i = 0; i < 4; ++i) sum[i] += uu[i];
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const long long k = k0 + ty * 4 + i;
        if (k >= outs) break;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (c0 + tx * 4 + j < cols) store_elem(gw + (r * outs + k) * cols + c0 + tx * 4 + j, acc[i][j]);
        if (bias) store_elem(gb + r * outs + k, sum[i]);
    }
}

// ---------------------------------------------------------------------------
// what a large product needs beforehand

// fp32 -> three bf16 planes: the upper 8 significant bits, the next 8, the last 8.
// They add up to it but for bits below 2^-133.  A value that is not finite keeps its kind in the
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

// One read of gY: the sums of its columns per sample (`sums`, may be null), and
// with COPY its bf16 planes in rows of `pitch` elements, for gradients that TMA
// cannot read as they lie (fp32, or rows off the 16-byte boundaries).  A block
// takes eight chunks of columns, 32 rows at a time; the blocks of a cluster (one to
// eight, gridDim.y) share a sample's rows and add their sums up through each
// other's shared memory, in order, so no second launch is needed.  Sums of 2 x 4096 x 28672 bf16 89 us (5.3
// TB/s); of 8192 x 4096 14.5 us; with the copy of 2991 x 4093 bf16, whose rows are
// read four bytes a lane, 24 us.
constexpr int kSweepChunks = 8, kSweepWays = 32;

template <typename T, bool COPY>
__global__ void __launch_bounds__(kSweepChunks * kSweepWays)
    sweep_kernel(const T* __restrict__ g, long long ld, long long samples, long long rows, long long cols, unsigned short* __restrict__ out, long long pitch,
                 T* __restrict__ sums, bool straight) {
    using K = Chunk<T>;
    constexpr int E = K::kElems, kCols = kSweepChunks * E;
    __shared__ float part[kSweepWays][kCols + 1];
    __shared__ float total[kCols];
    const int cx = threadIdx.x % kSweepChunks, way = threadIdx.x / kSweepChunks;
    const long long c = (long long)blockIdx.x * kCols + cx * E;
    const int n_cols = (int)max(0LL, min((long long)E, cols - c));
    for (long long r = blockIdx.z; r < samples; r += gridDim.z) {
        float2 sum[E / 2];
#pragma unroll
        for (int i = 0; i < E / 2; ++i) sum[i] = make_float2(0.0f, 0.0f);
        if (n_cols > 0) {
            auto use = [&](long long row, const unsigned(&w)[8]) {
                K k;
                k.from_words(w);
                if (COPY && sizeof(T) == 2) {
                    uint4* to = reinterpret_cast<uint4*>(out + row * pitch + c);
                    to[0] = make_uint4(w[0], w[1], w[2], w[3]);
                    if (n_cols > 8) to[1] = make_uint4(w[4], w[5], w[6], w[7]);
                }
                if (COPY && sizeof(T) == 4) {
                    unsigned short h[8][3];
#pragma unroll
                    for (int i = 0; i < 8; ++i) cut3(__uint_as_float(w[i]), h[i]);
#pragma unroll
                    for (int p = 0; p < 3; ++p)
                        *reinterpret_cast<uint4*>(out + ((long long)p * samples * rows + row) * pitch + c) =
                            make_uint4(h[0][p] | (unsigned)h[1][p] << 16, h[2][p] | (unsigned)h[3][p] << 16, h[4][p] | (unsigned)h[5][p] << 16,
                                       h[6][p] | (unsigned)h[7][p] << 16);
                }
#pragma unroll
                for (int i = 0; i < E / 2; ++i) sum[i] = __fadd2_rn(sum[i], k.v[i]);
            };
            const long long step = (long long)gridDim.y * kSweepWays;
            long long n = blockIdx.y * kSweepWays + way;
            // four rows at a time without a branch between their loads
            if (n_cols == E && straight) {
                for (; n + 3 * step < rows; n += 4 * step) {
                    unsigned w[4][8];
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
                        const uint4* p = reinterpret_cast<const uint4*>(g + (r * rows + n + u * step) * ld + c);
                        const uint4 lo = __ldg(p), hi = __ldg(p + 1);
                        w[u][0] = lo.x; w[u][1] = lo.y; w[u][2] = lo.z; w[u][3] = lo.w;
                        w[u][4] = hi.x; w[u][5] = hi.y; w[u][6] = hi.z; w[u][7] = hi.w;
                    }
#pragma unroll
                    for (int u = 0; u < 4; ++u) use(r * rows + n + u * step, w[u]);
                }
            } else if (n_cols == E) {
                for (; n + 3 * step < rows; n += 4 * step) {
                    unsigned v[4][9];
                    unsigned shift[4];
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
                        // the words that the chunk's elements lie in; for rows between two words the ninth holds the last one
                        // (both halves of the outermost words are read on their own: they may be all there is)
                        const uintptr_t p = reinterpret_cast<uintptr_t>(g + (r * rows + n + u * step) * ld + c);
                        shift[u] = (unsigned)(p & 2) * 8;
                        const unsigned* q = reinterpret_cast<const unsigned*>(p & ~(uintptr_t)3);
                        v[u][0] = shift[u] ? (unsigned)__ldg(reinterpret_cast<const unsigned short*>(p)) << 16 : __ldg(q);
#pragma unroll
                        for (int i = 1; i < 8; ++i) v[u][i] = __ldg(q + i);
                        v[u][8] = shift[u] ? (unsigned)__ldg(reinterpret_cast<const unsigned short*>(q + 8)) : 0u;
                    }
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
                        unsigned w[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i) w[i] = __funnelshift_r(v[u][i], v[u][i + 1], shift[u]);
                        use(r * rows + n + u * step, w);
                    }
                }
            }
            for (; n < rows; n += step) {
                unsigned w[8];
                K::load_words(g + (r * rows + n) * ld + c, n_cols, w);
                use(r * rows + n, w);
            }
        }
        if (!sums) continue;
#pragma unroll
        for (int i = 0; i < E / 2; ++i) {
            part[way][cx * E + 2 * i] = sum[i].x;
            part[way][cx * E + 2 * i + 1] = sum[i].y;
        }
        __syncthreads();
        if (threadIdx.x < kCols) {
            float t = 0.0f;
#pragma unroll 8
            for (int k = 0; k < kSweepWays; ++k) t += part[k][threadIdx.x];
            total[threadIdx.x] = t;
        }
        asm volatile("barrier.cluster.arrive.release;\nbarrier.cluster.wait.acquire;" ::: "memory");
        const long long col = (long long)blockIdx.x * kCols + threadIdx.x;
        if (blockIdx.y == 0 && threadIdx.x < kCols && col < cols) {
            float t = 0.0f;
            for (unsigned k = 0; k < gridDim.y; ++k) {
                float v;
                asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(in_cta(smem_u32(&total[threadIdx.x]), k)) : "memory");
                t += v;
            }
            store_elem(sums + r * cols + col, t);
        }
        // the sums of every block have been read before they change or the block ends
        asm volatile("barrier.cluster.arrive.release;\nbarrier.cluster.wait.acquire;" ::: "memory");
    }
}

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

// ---------------------------------------------------------------------------
// host side

struct Problem {
    int dtype;
    const void* gy;
    long long ld_gy, samples, rows, cols, outs;
};

// How a product is run, and what its workspace holds: the copied gradient, X^ in
// bf16, the partial products, each at a multiple of 256 bytes.
struct Plan {
    bool small, copy, pair;
    int planes, splits;
    long long pitch, x_pitch;
    int k_tiles, c_tiles, steps, steps_per_split;
    long long tiles;
    long long at_x, at_part, bytes;
};

// Products of at most kSmallRows tokens, and of at most kSmallWork tokens x 64 x 64
// tiles per SM, are small.  The small kernel's time goes with the tokens and the waves
// of tiles; the other form takes three to five launches, and a workspace, whatever the
// size.  Microseconds of a call from Python (in a graph), small against other:
//   fp32, 256 tokens: 128 tiles 16.7 (15.5) against 24.8 (16.6), 256 tiles 24.6 (22.9)
//     against 24.5 (16.6), 576 tiles 43 (42) against 25 (18.5)
//   bf16, 256 tokens: 128 tiles 20.5 (18.4) against 20.6 (11.7), 576 tiles 45 (42)
//     against 21 (12.7)
//   64 tokens: 576 tiles, fp32 15.5 (12.8) against 23.7 (14.8), bf16 14.4 (12.8)
//     against 20.7 (11.4); 1024 tiles 22.6 (21) against 24.7 (18.4), 23.4 (13.2)
constexpr long long kSmallRows = 256, kSmallWork = 320;

long long round_up(long long n, long long to) { return (n + to - 1) / to * to; }

Plan make_plan(const Problem& q, int sms) {
    Plan p = {};
    const long long small_tiles = ((q.outs + kSmallSide - 1) / kSmallSide) * ((q.cols + kSmallSide - 1) / kSmallSide);
    p.small = q.rows <= kSmallRows && small_tiles <= 65535 && q.samples <= 65535 && small_tiles * q.samples * q.rows <= kSmallWork * sms;
    if (p.small) return p;
    p.copy = q.dtype == AMPQ_F32 || !rows_aligned(q.gy, q.ld_gy, q.dtype);
    p.planes = q.dtype == AMPQ_F32 ? 3 : 1;
    p.pitch = p.copy ? round_up(q.outs, 8) : q.ld_gy;
    p.x_pitch = round_up(q.cols, 8);
    p.steps = (int)((q.rows + kStepRows - 1) / kStepRows);
    const long long pairs = ((q.outs + 255) / 256) * ((q.cols + 255) / 256) * q.samples;
    // A pair's tile runs at twice the rate per SM (its operands are read from shared
    // memory half as often): 1 x 2048 x 2048 x 2048, 64 pairs, 26.6 us against 34.5.
    // With few tiles single CTAs spread better: 1 x 4096 x 1024 x 1024, 16 pairs,
    // 35.6 us against 32.4.
    p.pair = pairs * 4 >= sms;
    const int side = p.pair ? 256 : 128;
    p.k_tiles = (int)((q.outs + side - 1) / side);
    p.c_tiles = (int)((q.cols + side - 1) / side);
    const long long tiles = (long long)p.k_tiles * p.c_tiles * q.samples;
    const int units = p.pair ? sms / 2 : sms;
    // few tiles and many tokens: several parts of the token axis per tile, at least 512 tokens each
    long long splits = tiles > 0 && tiles < units ? units / tiles : 1;
    if (splits > p.steps / 8) splits = p.steps / 8;
    if (splits < 1) splits = 1;
    p.steps_per_split = p.steps > 0 ? (int)((p.steps + splits - 1) / splits) : 1;
    p.splits = p.steps > 0 ? (p.steps + p.steps_per_split - 1) / p.steps_per_split : 1;
    p.tiles = tiles * p.splits;
    long long at = 0;
    if (p.copy) at = round_up(2LL * p.planes * q.samples * q.rows * p.pitch, 256);
    p.at_x = at;
    at += round_up(2LL * q.samples * q.rows * p.x_pitch, 256);
    p.at_part = at;
    if (p.splits > 1) at += round_up(4LL * q.samples * p.splits * q.outs * q.cols, 256);
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

// A bf16 matrix as [planes][samples][rows][cols], rows `pitch` elements apart: 64
// tokens x 64 columns per copy, zeros outside each sample.
int operand_map(CUtensorMap* map, const void* base, long long pitch, long long cols, const Problem& q, int planes) {
    const EncodeFn encode = encode_fn();
    if (!encode) return AMPQ_ERR_CUDA;
    const unsigned long long row = 2ull * (unsigned long long)pitch;
    unsigned long long sample = row * (unsigned long long)q.rows, plane = sample * (unsigned long long)q.samples;
    if (q.samples == 1) sample = row;  // never stepped over
    if (planes == 1) plane = row;
    const unsigned long long limit = 1ull << 40;
    if (row >= limit || sample >= limit || plane >= limit) return AMPQ_ERR_TOO_LARGE;
    const cuuint64_t dims[4] = {(cuuint64_t)cols, (cuuint64_t)q.rows, (cuuint64_t)q.samples, (cuuint64_t)planes};
    const cuuint64_t strides[3] = {row, sample, plane};
    const cuuint32_t box[4] = {64, kStepRows, 1, 1}, one[4] = {1, 1, 1, 1};
    const CUresult rc = encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(base), dims, strides, box, one,
                               CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return rc == CUDA_SUCCESS ? AMPQ_OK : AMPQ_ERR_CUDA;
}

constexpr int kMaxDevices = 64;

using ProductKernel = void (*)(const CUtensorMap, const CUtensorMap, const ProductArgs);

// One CTA (pair) per SM (two), no more than there are tiles.  `prepared`: on which
// devices the kernel may use its shared memory already.
int launch_persistent(ProductKernel kernel, std::atomic<bool>* prepared, int cg, int threads, int smem, const CUtensorMap& map, const CUtensorMap& second,
                      const ProductArgs& a, int device, int sms, cudaStream_t st) {
    if (device >= kMaxDevices || !prepared[device].load(std::memory_order_acquire)) {
        if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess) {
            cudaGetLastError();
            return AMPQ_ERR_CUDA;
        }
        if (device < kMaxDevices) prepared[device].store(true, std::memory_order_release);
    }
    const long long units = sms / cg;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(cg * (a.tiles < units ? a.tiles : units)));
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = cg;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, kernel, map, second, a) != cudaSuccess) {
        cudaGetLastError();
        return AMPQ_ERR_CUDA;
    }
    return AMPQ_OK;
}

template <int CG, int PLANES, int RUN, typename OUT>
int launch_product(const CUtensorMap& g_map, const CUtensorMap& x_map, const ProductArgs& a, int device, int sms, cudaStream_t st) {
    static std::atomic<bool> prepared[kMaxDevices];
    return launch_persistent(product_kernel<CG, PLANES, RUN, OUT>, prepared, CG, kThreads, kSmemBytes, g_map, x_map, a, device, sms, st);
}

template <int PLANES, int RUN, typename OUT>
int run_product(const CUtensorMap& g_map, const CUtensorMap& x_map, const ProductArgs& a, bool pair, int device, int sms, cudaStream_t st) {
    return pair ? launch_product<2, PLANES, RUN, OUT>(g_map, x_map, a, device, sms, st) : launch_product<1, PLANES, RUN, OUT>(g_map, x_map, a, device, sms, st);
}

// OUT: the type of gw, or fp32 for partial products.
template <typename T, typename OUT>
int choose_product(const CUtensorMap& g_map, const CUtensorMap& x_map, const ProductArgs& a, bool pair, int device, int sms, cudaStream_t st) {
    constexpr int kRun = kRunTokens / kStepRows;
    if constexpr (sizeof(T) == 4) return run_product<3, 1, OUT>(g_map, x_map, a, pair, device, sms, st);
    else if (a.steps_per_split <= kRun) return run_product<1, 0, OUT>(g_map, x_map, a, pair, device, sms, st);
    else return run_product<1, kRun, OUT>(g_map, x_map, a, pair, device, sms, st);
}

struct Operands {
    const unsigned char *codes, *scales;
    long long ld_codes, ld_scales;
    int fmt;
    void *gw, *gb;
    unsigned char* ws;
};

template <typename T, int FMT>
int run_small(const Problem& q, const Operands& o, cudaStream_t st) {
    const dim3 grid((unsigned)((q.outs + kSmallSide - 1) / kSmallSide), (unsigned)((q.cols + kSmallSide - 1) / kSmallSide), (unsigned)q.samples);
    small_product_kernel<T, FMT><<<grid, 256, 0, st>>>(static_cast<const T*>(q.gy), q.ld_gy, o.codes, o.ld_codes, o.scales, o.ld_scales, q.rows, q.cols, q.outs,
                                                       static_cast<T*>(o.gw), static_cast<T*>(o.gb));
    return launched();
}

template <typename T>
int sweep(const Problem& q, const Operands& o, bool copy, long long pitch, int sms, cudaStream_t st) {
    if (!copy && !o.gb) return AMPQ_OK;
    constexpr int kCols = kSweepChunks * Chunk<T>::kElems;
    const T* gy = static_cast<const T*>(q.gy);
    const bool straight = rows_aligned(q.gy, q.ld_gy, q.dtype);  // rows on 16-byte boundaries
    // Parts of the rows: the fewest microseconds by a rough count, three blocks on an
    // SM at a time, 6 us for a block's joining and 1.5 us for each 128 rows of a part.
    const long long blocks = (q.outs + kCols - 1) / kCols * q.samples;
    int parts = 1;
    double least = 0.0;
    for (int p = 1; p <= 8; p *= 2) {
        const double us = (double)((blocks * p + 3LL * sms - 1) / (3LL * sms)) * (6.0 + 1.5 * (double)((q.rows + 128LL * p - 1) / (128LL * p)));
        if (p == 1 || us < least) {
            least = us;
            parts = p;
        }
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((q.outs + kCols - 1) / kCols), parts, (unsigned)(q.samples < 65535 ? q.samples : 65535));
    cfg.blockDim = dim3(kSweepChunks * kSweepWays);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = attr[0].val.clusterDim.z = 1;
    attr[0].val.clusterDim.y = parts;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    unsigned short* out = copy ? reinterpret_cast<unsigned short*>(o.ws) : nullptr;
    if (cudaLaunchKernelEx(&cfg, copy ? sweep_kernel<T, true> : sweep_kernel<T, false>, gy, q.ld_gy, q.samples, q.rows, q.outs, out, pitch, static_cast<T*>(o.gb),
                           straight) != cudaSuccess) {
        cudaGetLastError();
        return AMPQ_ERR_CUDA;
    }
    return AMPQ_OK;
}

template <typename T>
int run_large(const Problem& q, const Plan& p, const Operands& o, int device, int sms, cudaStream_t st) {
    const long long rows = q.samples * q.rows;
    int rc;
    if ((rc = sweep<T>(q, o, p.copy, p.pitch, sms, st))) return rc;
    if ((rc = launch_ckpt_unpack(AMPQ_BF16, o.fmt, o.codes, o.ld_codes, o.scales, o.ld_scales, rows, q.cols, o.ws + p.at_x, p.x_pitch, st))) return rc;
    CUtensorMap g_map, x_map;
    if ((rc = operand_map(&g_map, p.copy ? o.ws : q.gy, p.pitch, q.outs, q, p.planes))) return rc;
    if ((rc = operand_map(&x_map, o.ws + p.at_x, p.x_pitch, q.cols, q, 1))) return rc;
    const bool partial = p.splits > 1;
    ProductArgs a;
    a.out = partial ? o.ws + p.at_part : o.gw;
    a.cols = q.cols;
    a.outs = q.outs;
    a.tiles = p.tiles;
    a.k_tiles = p.k_tiles;
    a.c_tiles = p.c_tiles;
    a.splits = p.splits;
    a.steps = p.steps;
    a.steps_per_split = p.steps_per_split;
    a.vec = rows_aligned(a.out, q.cols, partial ? AMPQ_F32 : q.dtype);
    rc = partial ? choose_product<T, float>(g_map, x_map, a, p.pair, device, sms, st) : choose_product<T, T>(g_map, x_map, a, p.pair, device, sms, st);
    if (rc || !partial) return rc;
    const long long n = q.outs * q.cols, blocks = (q.samples * n + 255) / 256;
    join_splits_kernel<T><<<(unsigned)(blocks < 8LL * sms ? blocks : 8LL * sms), 256, 0, st>>>(reinterpret_cast<const float*>(o.ws + p.at_part), q.samples, p.splits, n,
                                                                                               static_cast<T*>(o.gw));
    return launched();
}

template <typename T>
int run(const Problem& q, const Plan& p, const Operands& o, int device, int sms, cudaStream_t st) {
    if (q.rows > 0 && q.cols > 0) {
        if (p.small) return o.fmt == AMPQ_FMT_E4M3 ? run_small<T, AMPQ_FMT_E4M3>(q, o, st) : run_small<T, AMPQ_FMT_E5M2>(q, o, st);
        return run_large<T>(q, p, o, device, sms, st);
    }
    // no product: zeros, or no columns at all
    bool ok = true;
    if (q.rows == 0) {
        if (q.cols > 0) ok = cudaMemsetAsync(o.gw, 0, (size_t)(q.samples * q.outs * q.cols) * sizeof(T), st) == cudaSuccess;
        if (o.gb) ok = ok && cudaMemsetAsync(o.gb, 0, (size_t)(q.samples * q.outs) * sizeof(T), st) == cudaSuccess;
    }
    if (!ok) {
        cudaGetLastError();
        return AMPQ_ERR_CUDA;
    }
    return q.rows == 0 ? AMPQ_OK : sweep<T>(q, o, false, 0, sms, st);
}

int check_sizes(int dtype, long long samples, long long rows, long long cols, long long outs) {
    if (!known_dtype(dtype) || samples < 0 || rows < 0 || cols < 0 || outs < 0) return AMPQ_ERR_INVALID;
    if (cols > kMaxCols || outs > kMaxCols || samples > kMaxRows || rows > kMaxRows || (samples > 0 && rows > kMaxRows / samples)) return AMPQ_ERR_TOO_LARGE;
    // tiles of one sample are counted in 32 bits
    if (((outs + 127) / 128) * ((cols + 127) / 128) > 0x7FFFFFFFLL) return AMPQ_ERR_TOO_LARGE;
    // gradients and workspaces are counted in 64 bits (the partial products of few tiles are at most one per SM)
    const double tokens = (double)samples * (double)rows, most = 4503599627370496.0;  // 2^52 bytes
    if (12.0 * tokens * (double)outs > most || 2.0 * tokens * (double)cols > most || 4.0 * (double)samples * (double)outs * (double)cols > most)
        return AMPQ_ERR_TOO_LARGE;
    return AMPQ_OK;
}

}  // namespace
}  // namespace ampq

using namespace ampq;

extern "C" {
#pragma GCC visibility push(default)

int ampq_ckpt_weight_grad_workspace(int device, int dtype, const void* gy, long long ld_gy, long long samples, long long rows, long long cols,
                                    long long outs, long long* bytes) {
    if (!bytes) return AMPQ_ERR_INVALID;
    const int rc = check_sizes(dtype, samples, rows, cols, outs);
    if (rc) return rc;
    CkptDevice cur(device);
    if (cur.status) return cur.status;
    const int sms = sm_count(device);
    if (sms < 2) return AMPQ_ERR_CUDA;
    *bytes = rows > 0 && cols > 0 ? make_plan(Problem{dtype, gy, ld_gy, samples, rows, cols, outs}, sms).bytes : 0;
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
    const Problem q{dtype, gy, ld_gy, samples, rows, cols, outs};
    const Plan p = make_plan(q, sms);
    if (rows > 0 && cols > 0 && p.bytes > 0 && (!workspace || workspace_bytes < p.bytes)) return AMPQ_ERR_INVALID;
    const Operands o{codes, scales, ld_codes, ld_scales, fmt, gw, gb, static_cast<unsigned char*>(workspace)};
    cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
    return dtype == AMPQ_F32 ? run<float>(q, p, o, device, sms, st) : run<__nv_bfloat16>(q, p, o, device, sms, st);
}

#pragma GCC visibility pop
}  // extern "C"
