// Matrix products on the 5th-generation tensor cores, shared by the classifier loss and the orthogonalised update.
//
// D[b] = A[b] * B[b]^T with A [M x K], B [N x K], 16-bit operands (both fp16 or both bf16), fp32 accumulators in
// tensor memory. Either operand may lie K-contiguous ("K-major": rows of A as stored) or M/N-contiguous ("MN-major":
// the transposed matrix as stored), so no product of this library transposes anything in memory. What becomes of the
// accumulators is the epilogue's business: a functor reads them from tensor memory, 8 consecutive columns of one row
// at a time, or a whole row of a tile.
//
// One CTA per SM, 12 warps: warp 0 loads K-tiles of 64 by TMA into a ring of shared-memory stages (128-byte swizzle),
// warp 1 issues the MMAs, warp 2 owns the tensor memory, warps 4-11 run the epilogue of one accumulator while the
// other one is being filled (two accumulators of BN columns). Two shapes:
//   CG = 2, BN = 256: a pair of SMs computes a 256 x 256 tile (cta_group::2); each holds 128 rows of A and 128 rows
//           of B, so a K-tile costs 32 KB of shared memory per SM for twice the MMA work of a lone 128 x 128 tile.
//   CG = 1, BN = 128: 128 x 128 tiles for problems with fewer than a GPU's worth of large tiles. With SPLIT, a cluster
//           of up to 8 CTAs shares one tile, each a slice of K; the partial sums meet in distributed shared memory
//           and are added in the order of the slices, so results do not depend on timing.
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "ac_common.h"
#include "tc_ptx.cuh"

namespace ac {
namespace mm {

using namespace tc;

constexpr int kThreads = 384;
constexpr int kEpiWarps = 8;
constexpr int kBK = 64;                      // K-tile: one 128-byte swizzle row of 16-bit elements
constexpr int kStages = 6;
constexpr int kMaxSplit = 8;

struct Params {
    int m, n;             // extents of the result
    int ktiles;           // ceil(K / 64)
    int tiles_m, tiles_n;
    int per_batch;        // tiles of one matrix of the batch
    int tiles;            // per_batch * batch
    int group;            // tiles of the fast direction that are cycled before the slow direction advances
    int fast_m;           // 1: tiles of M are the fast direction
    int sym;              // 1: the result is symmetric; only tiles with tile_n >= tile_m are computed
    int split;            // CTAs that share a tile's K (SPLIT kernels)
    uint32_t idesc;
    uint32_t* status;     // status block of the workspace
    int reset_status;     // 1: first launch of the call
};

struct Tile {
    int batch, tm, tn;
};

__device__ __forceinline__ Tile decode_tile(const Params& p, int t) {
    Tile r;
    r.batch = t / p.per_batch;
    int i = t - r.batch * p.per_batch;
    if (p.sym) {
        int row = 0;
        while (i >= p.tiles_n - row) { i -= p.tiles_n - row; ++row; }
        r.tm = row;
        r.tn = row + i;
        return r;
    }
    const int tf = p.fast_m ? p.tiles_m : p.tiles_n, ts = p.fast_m ? p.tiles_n : p.tiles_m;
    const int g = i / (p.group * ts), first = g * p.group;
    i -= first * ts;
    const int size = min(p.group, tf - first), s = i / size, f = first + i - s * size;
    r.tm = p.fast_m ? f : s;
    r.tn = p.fast_m ? s : f;
    return r;
}

// ---- PTX that only these kernels use ----------------------------------------

__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t map_rank(uint32_t addr, uint32_t rank) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
__device__ __forceinline__ float ld_cluster(uint32_t addr) {
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ void mbar_arrive_cluster(uint32_t cluster_addr) {
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}
__device__ __forceinline__ void fence_barrier_init() {
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
}
template <int CG>
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const void* tmap, uint32_t bar, int c0, int c1, int c2) {
    if constexpr (CG == 2)
        asm volatile(
            "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes "
            "[%0], [%1, {%3, %4, %5}], [%2];" ::"r"(dst),
            "l"(reinterpret_cast<uint64_t>(tmap)), "r"(bar), "r"(c0), "r"(c1), "r"(c2)
            : "memory");
    else
        asm volatile(
            "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes "
            "[%0], [%1, {%3, %4, %5}], [%2];" ::"r"(dst),
            "l"(reinterpret_cast<uint64_t>(tmap)), "r"(bar), "r"(c0), "r"(c1), "r"(c2)
            : "memory");
}
template <int CG>
__device__ __forceinline__ void tmem_alloc_cg(uint32_t* dst, uint32_t cols) {
    if constexpr (CG == 2) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(dst)), "r"(cols)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else {
        tmem_alloc(dst, cols);
    }
}
template <int CG>
__device__ __forceinline__ void tmem_dealloc_cg(uint32_t addr, uint32_t cols) {
    if constexpr (CG == 2)
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(addr), "r"(cols) : "memory");
    else
        tmem_dealloc(addr, cols);
}
template <int CG>
__device__ __forceinline__ void mma_words(uint32_t d, uint32_t a_lo, uint32_t a_hi, uint32_t b_lo, uint32_t b_hi,
                                          uint32_t idesc, uint32_t accumulate) {
    if constexpr (CG == 2)
        asm volatile(
            "{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\t"
            "mov.b64 da, {%1, %2};\n\t"
            "mov.b64 db, {%3, %4};\n\t"
            "setp.ne.b32 p, %6, 0;\n\t"
            "tcgen05.mma.cta_group::2.kind::f16 [%0], da, db, %5, p;\n\t}" ::"r"(d),
            "r"(a_lo), "r"(a_hi), "r"(b_lo), "r"(b_hi), "r"(idesc), "r"(accumulate)
            : "memory");
    else
        mma_bf16_words(d, a_lo, a_hi, b_lo, b_hi, idesc, accumulate);
}
// Arrives on `bar` when the MMAs issued so far are complete; of a pair, on both CTAs' barrier at that offset.
template <int CG>
__device__ __forceinline__ void commit_cg(uint64_t* bar) {
    if constexpr (CG == 2) {
        const uint16_t both = 3;
        asm volatile(
            "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(
                smem_u32(bar)),
            "h"(both)
            : "memory");
    } else {
        mma_commit(bar);
    }
}
__device__ __forceinline__ float ex2(float x) {   // 2^x, about 2 ulp; 0 for very negative x
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// ---- 8 consecutive 16-bit values of one row ----------------------------------

template <class T> __device__ __forceinline__ uint32_t pack2(float a, float b);
template <> __device__ __forceinline__ uint32_t pack2<__half>(float a, float b) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}
template <> __device__ __forceinline__ uint32_t pack2<__nv_bfloat16>(float a, float b) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}
template <class T>
__device__ __forceinline__ void store8(T* dst, const float* v) {      // dst 16-byte aligned
    uint4 u;
    u.x = pack2<T>(v[0], v[1]);
    u.y = pack2<T>(v[2], v[3]);
    u.z = pack2<T>(v[4], v[5]);
    u.w = pack2<T>(v[6], v[7]);
    *reinterpret_cast<uint4*>(dst) = u;
}
__device__ __forceinline__ void load8(const __half* src, float* v) {
    const uint4 u = *reinterpret_cast<const uint4*>(src);
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
        v[2 * i] = f.x;
        v[2 * i + 1] = f.y;
    }
}

// ---- the kernel ---------------------------------------------------------------

struct Shared {
    uint64_t full[kStages], empty[kStages], tfull[2], tempty[2];
    uint32_t tmem;
    int abort;
};

__device__ __forceinline__ void flag_timeout(int* abort_s, uint32_t* status, uint32_t code) {
    if (atomicExch(abort_s, 1) == 0) {
        status[1] = code;
        atomicExch(&status[0], 1u);
    }
}

template <int CG, int BN> __host__ __device__ constexpr int stage_bytes() { return 128 * 128 + BN / CG * 128; }
template <int CG, int BN> __host__ __device__ constexpr int smem_bytes() { return kStages * stage_bytes<CG, BN>() + 1024; }

// Hands 8 columns of one row at a time to the functor, from tensor memory.
template <int COLS, class Epi>
__device__ __forceinline__ void epilogue_by_8(const Epi& epi, uint32_t taddr, int batch, int row, int col, bool mirror) {
#pragma unroll 1
    for (int c = 0; c < COLS; c += 32) {
        uint32_t r[32];
        tmem_ld32(taddr + c, r);
#pragma unroll
        for (int j = 0; j < 32; j += 8) {
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(r[j + i]);
            epi.apply8(batch, row, col + c + j, v, mirror);
        }
    }
}

template <int CG, int BN, bool AMN, bool BMN, bool SPLIT, class Epi>
__global__ void __launch_bounds__(kThreads, 1)
mm_kernel(const __grid_constant__ CUtensorMap ta, const __grid_constant__ CUtensorMap tb,
          const __grid_constant__ Params p, const __grid_constant__ Epi epi) {
    static_assert(!SPLIT || CG == 1, "a split tile is a cluster of single CTAs");
    constexpr int NB = BN / CG;               // rows of B that one CTA holds
    constexpr uint32_t kStage = stage_bytes<CG, BN>();
    constexpr bool kCluster = CG == 2 || SPLIT;
    extern __shared__ uint8_t smem_raw[];
    __shared__ Shared sh;
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t rank = kCluster ? cluster_rank() : 0;
    const int per_tile = SPLIT ? p.split : CG;                       // CTAs of one tile
    const int unit = blockIdx.x / per_tile, units = gridDim.x / per_tile;
    const int k_begin = SPLIT ? (int)((long long)p.ktiles * rank / p.split) : 0;
    const int k_end = SPLIT ? (int)((long long)p.ktiles * (rank + 1) / p.split) : p.ktiles;
    volatile int* abort_flag = &sh.abort;

    if (tid == 0) {
        sh.abort = 0;
        for (int s = 0; s < kStages; ++s) { mbar_init(&sh.full[s], 1); mbar_init(&sh.empty[s], 1); }
        for (int a = 0; a < 2; ++a) { mbar_init(&sh.tfull[a], 1); mbar_init(&sh.tempty[a], kEpiWarps * CG); }
        fence_barrier_init();
        prefetch_tmap(&ta);
        prefetch_tmap(&tb);
    }
    if (warp == 2) tmem_alloc_cg<CG>(&sh.tmem, 2 * BN);
    tc_fence_before();
    __syncthreads();
    if constexpr (kCluster) cluster_sync();
    tc_fence_after();
    const uint32_t tmem = sh.tmem;
    pdl_launch_dependents();
    if (p.reset_status && blockIdx.x == 0 && tid == 96) {
        pdl_wait();
        p.status[0] = 0u;
        p.status[1] = 0u;
    }

    if (warp == 0) {
        // ---------------------------------------------------------------- loads
        if (elect_one()) {
            pdl_wait();
            int it = 0;
            bool ok = true;
            for (int t = unit; t < p.tiles && ok; t += units) {
                const Tile tile = decode_tile(p, t);
                const int row0 = tile.tm * (128 * CG) + (CG == 2 ? (int)rank * 128 : 0);
                const int col0 = tile.tn * BN + (CG == 2 ? (int)rank * NB : 0);
                for (int kt = k_begin; kt < k_end; ++kt, ++it) {
                    const int s = it % kStages;
                    if (!mbar_wait(&sh.empty[s], ((it / kStages) & 1) ^ 1, abort_flag)) {
                        flag_timeout(&sh.abort, p.status, 0x1100u + s);
                        ok = false;
                        break;
                    }
                    // a pair's loads all complete on the leader's barrier; it alone announces the bytes of both
                    if (CG == 1 || rank == 0) mbar_arrive_expect_tx(&sh.full[s], kStage * CG);
                    uint32_t bar = smem_u32(&sh.full[s]);
                    if constexpr (CG == 2) bar = map_rank(bar, 0);
                    const uint32_t a = base + s * kStage, b = a + 128 * 128;
                    if constexpr (AMN) {
#pragma unroll
                        for (int j = 0; j < 2; ++j)
                            tma_load_3d<CG>(a + j * 8192, &ta, bar, row0 + 64 * j, kt * kBK, tile.batch);
                    } else {
                        tma_load_3d<CG>(a, &ta, bar, kt * kBK, row0, tile.batch);
                    }
                    if constexpr (BMN) {
#pragma unroll
                        for (int j = 0; j < NB / 64; ++j)
                            tma_load_3d<CG>(b + j * 8192, &tb, bar, col0 + 64 * j, kt * kBK, tile.batch);
                    } else {
                        tma_load_3d<CG>(b, &tb, bar, kt * kBK, col0, tile.batch);
                    }
                }
            }
        }
    } else if (warp == 1 && (CG == 1 || rank == 0)) {
        // ----------------------------------------------------------------- MMAs
        // The whole warp runs the loop, so that the descriptor arithmetic stays in uniform registers.
        const bool leader = elect_one();
        const uint32_t hi = desc_hi(1024, 2);
        int it = 0, n = 0;
        bool ok = true;
        for (int t = unit; t < p.tiles && ok; t += units, ++n) {
            const int acc = n & 1;
            bool got = mbar_wait(&sh.tempty[acc], ((n >> 1) & 1) ^ 1, abort_flag);
            if (!__all_sync(0xffffffffu, got)) {
                if (leader) flag_timeout(&sh.abort, p.status, 0x1200u + acc);
                ok = false;
                break;
            }
            tc_fence_after();
            const uint32_t d = tmem + acc * BN;
            for (int kt = k_begin; kt < k_end; ++kt, ++it) {
                const int s = it % kStages;
                got = mbar_wait(&sh.full[s], (it / kStages) & 1, abort_flag);
                if (!__all_sync(0xffffffffu, got)) {
                    if (leader) flag_timeout(&sh.abort, p.status, 0x1300u + s);
                    ok = false;
                    break;
                }
                tc_fence_after();
                const uint32_t a_lo = desc_lo(base + s * kStage, AMN ? 8192 : 16);
                const uint32_t b_lo = desc_lo(base + s * kStage + 128 * 128, BMN ? 8192 : 16);
#pragma unroll
                for (int kk = 0; kk < 4; ++kk)     // K = 16 each: 32 bytes along a K-major row, 16 rows of an MN-major slab
                    if (leader)
                        mma_words<CG>(d, a_lo + kk * (AMN ? 128 : 2), hi, b_lo + kk * (BMN ? 128 : 2), hi, p.idesc,
                                      (uint32_t)(kt > k_begin || kk > 0));
                if (leader) commit_cg<CG>(&sh.empty[s]);
                __syncwarp();
            }
            if (ok && leader) commit_cg<CG>(&sh.tfull[acc]);
            __syncwarp();
        }
    } else if (warp >= 4) {
        // ------------------------------------------------------------- epilogue
        const int quarter = warp & 3, half = (warp - 4) >> 2;       // the TMEM lanes this warp may read; its columns
        const uint32_t lanes = tmem + ((uint32_t)(quarter * 32) << 16) + half * (BN / 2);
        pdl_wait();
        int n = 0;
        for (int t = unit; t < p.tiles; t += units, ++n) {
            const int acc = n & 1;
            const bool got = mbar_wait(&sh.tfull[acc], (n >> 1) & 1, abort_flag);
            if (!__all_sync(0xffffffffu, got)) {
                if (lane == 0) flag_timeout(&sh.abort, p.status, 0x1400u + acc);
                break;
            }
            tc_fence_after();
            const Tile tile = decode_tile(p, t);
            if constexpr (SPLIT) {
                // partial sums to shared memory, [column][row]; the stages are free once the MMAs are complete
                float* part = reinterpret_cast<float*>(smem_raw + (base - smem_u32(smem_raw)));
#pragma unroll 1
                for (int c = 0; c < BN / 2; c += 32) {
                    uint32_t r[32];
                    tmem_ld32(lanes + acc * BN + c, r);
#pragma unroll
                    for (int j = 0; j < 32; ++j)
                        part[(half * (BN / 2) + c + j) * 128 + quarter * 32 + lane] = __uint_as_float(r[j]);
                }
            } else {
                const int row = tile.tm * (128 * CG) + (CG == 2 ? (int)rank * 128 : 0) + quarter * 32 + lane;
                const int col = tile.tn * BN + half * (BN / 2);
                if constexpr (Epi::kWholeRow)
                    epi.template row<BN / 2>(lanes + acc * BN, row, col);
                else
                    epilogue_by_8<BN / 2>(epi, lanes + acc * BN, tile.batch, row, col, p.sym && tile.tm != tile.tn);
                tc_fence_before();
                __syncwarp();
                if (lane == 0) {
                    uint32_t bar = smem_u32(&sh.tempty[acc]);
                    if constexpr (CG == 2)
                        mbar_arrive_cluster(map_rank(bar, 0));
                    else
                        mbar_arrive(&sh.tempty[acc]);
                }
            }
        }
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (*abort_flag) {      // copies of an abandoned tile may still be in flight: let them land before this CTA ends
        const long long t0 = clock64();
        while (clock64() - t0 < (1ll << 22)) __nanosleep(1000);
        __syncthreads();
    }
    if constexpr (kCluster) cluster_sync();
    if constexpr (SPLIT) {
        // every CTA of the cluster adds up its share of the columns, slice 0 first
        if (warp >= 4 && !*abort_flag) {
            const Tile tile = decode_tile(p, unit);
            const int width = BN / p.split, e = tid - 128;
            for (int i = e; i < width / 8 * 128; i += kEpiWarps * 32) {
                const int r = i & 127, c = (int)rank * width + (i >> 7) * 8;
                float v[8] = {};
                for (int s = 0; s < p.split; ++s) {
                    const uint32_t from = map_rank(base + (uint32_t)(c * 128 + r) * 4, s);
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[j] += ld_cluster(from + j * 512);
                }
                epi.apply8(tile.batch, tile.tm * 128 + r, tile.tn * BN + c, v, p.sym && tile.tm != tile.tn);
            }
        }
        __syncwarp();
        cluster_sync();
    }
    tc_fence_after();
    if (warp == 2) tmem_dealloc_cg<CG>(tmem, 2 * BN);
}

// ---- host side ------------------------------------------------------------------

// One operand: `rows` rows of `inner` 16-bit elements, `pitch` elements apart, `batch` matrices `stride` elements
// apart. mn: the inner direction is the result's (M or N) and the rows are K.
struct Operand {
    const void* p;
    long long inner, rows, pitch;
    int batch;
    long long stride;
    bool mn;
};

ac_status make_map(CUtensorMap* map, const Operand& o, bool bf16, int tile_rows);     // mm_host.cu
// Tile grid, raster and instruction descriptor of a product [m x n x k].
Params make_params(int m, int n, long long k, int batch, int cg, int bn, bool a_mn, bool b_mn, bool bf16, bool sym);
// Whether 256 x 256 tiles of CTA pairs fill the GPU; else 128 x 128 tiles and, in *split, the CTAs that share one.
bool use_pairs(int m, int n, long long k, int batch, bool sym, int* split);

template <int CG, int BN, bool AMN, bool BMN, bool SPLIT, class Epi>
ac_status launch_one(const Operand& a, const Operand& b, bool bf16, const Params& p, const Epi& epi, cudaStream_t st) {
    static bool attr_done[64] = {};
    CUtensorMap ta, tb;
    ac_status rc = make_map(&ta, a, bf16, 128);
    if (rc == AC_OK) rc = make_map(&tb, b, bf16, BN / CG);
    auto kernel = mm_kernel<CG, BN, AMN, BMN, SPLIT, Epi>;
    if (rc == AC_OK) rc = ensure_smem_limit(kernel, smem_bytes<CG, BN>(), attr_done);
    if (rc != AC_OK) return rc;
    const int per_tile = SPLIT ? p.split : CG;
    const int units = SPLIT ? p.tiles : (p.tiles < kNumSMs / CG ? p.tiles : kNumSMs / CG);
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(units * per_tile);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = smem_bytes<CG, BN>();
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = per_tile;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = per_tile > 1 ? 2 : 1;
    AC_CUDA_TRY(cudaLaunchKernelEx(&cfg, kernel, ta, tb, p, epi));
    return AC_OK;
}

// D = A B^T for operands of one layout pair, on tiles of CTA pairs or on 128 x 128 tiles whose K `split` CTAs share.
template <bool AMN, bool BMN, class Epi>
ac_status launch_shaped(bool pairs, int split, const Operand& a, const Operand& b, int m, int n, long long k, int batch,
                        bool bf16, bool sym, uint32_t* status, bool reset, const Epi& epi, cudaStream_t st) {
    Params p = make_params(m, n, k, batch, pairs ? 2 : 1, pairs ? 256 : 128, AMN, BMN, bf16, sym);
    p.status = status;
    p.reset_status = reset;
    if (pairs) return launch_one<2, 256, AMN, BMN, false>(a, b, bf16, p, epi, st);
    if constexpr (!Epi::kWholeRow) {
        if (split > 1) {
            p.split = split;
            return launch_one<1, 128, AMN, BMN, true>(a, b, bf16, p, epi, st);
        }
    }
    return launch_one<1, 128, AMN, BMN, false>(a, b, bf16, p, epi, st);
}

// The same with the shape chosen by use_pairs.
template <bool AMN, bool BMN, class Epi>
ac_status launch(const Operand& a, const Operand& b, int m, int n, long long k, int batch, bool bf16, bool sym,
                 uint32_t* status, bool reset, const Epi& epi, cudaStream_t st) {
    int split = 1;
    const bool pairs = use_pairs(m, n, k, batch, sym, &split);
    return launch_shaped<AMN, BMN>(pairs, split, a, b, m, n, k, batch, bf16, sym, status, reset, epi, st);
}

}  // namespace mm
}  // namespace ac
