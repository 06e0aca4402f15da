// The whole update of a small matrix in one kernel: at most 128 on the shorter side (k), 1536 on the longer (l).
//
// A cluster of up to 8 CTAs per matrix; each keeps a slice of at most 192 columns of X (k x l; a matrix with more rows
// than columns is taken transposed) in shared memory from the gradient to the update, as two fp16 terms. Per step:
//   Gram sum of the slice (tensor cores) -> partial sums to the workspace -> cluster barrier -> every CTA adds all of
//   them, in the order of the slices -> A as two fp16 terms -> A^2 -> P = b A + c A^2 as two terms -> X <- a X + P X.
// The slice of X is stored once, 64-column slabs of 128-byte rows: read along the rows it is the K-major operand of the
// Gram product, read across them the MN-major operand of P X. Every product is formed from both terms of both operands
// (hi hi + hi lo + lo hi), about 22 bits: at this size the products are a fourth of the time, and the small matrices'
// errors do not average out. What bounds it is the chain of 15 products, each with its way through tensor memory and
// shared memory: 64 x 576 takes 73 us in place of 80 for 17 launches of the kernels for large matrices.
#pragma once

#include "mm_core.cuh"

namespace ac {

using namespace mm;

namespace {

constexpr int kOnchipK = 128, kOnchipSlabs = 3, kOnchipCluster = 8;
constexpr int kOnchipL = kOnchipSlabs * 64 * kOnchipCluster;
constexpr uint32_t kSlab = 128 * 128;                     // 128 rows of 64 16-bit elements
constexpr uint32_t kOnchipSmem = (2 * kOnchipSlabs + 4) * kSlab + 1024;

struct Onchip {
    const void* grad;
    const float* v_in;
    float* v_out;
    __nv_bfloat16* update;
    float* partial;         // [2][batch][cluster][k16][128]: Gram sums, columns of 128 rows; two so that one barrier suffices
    float* norms;           // [batch][cluster]
    uint32_t* status;
    float beta, a, b, c, eps, scale;
    int nesterov, bf16, steps;
    int rows, cols, k, l;
    int slabs;              // per CTA
};

__device__ __forceinline__ uint32_t slab_at(int row, int col) {       // byte offset of an element, 128-byte swizzle
    return (uint32_t)(col >> 6) * kSlab + (uint32_t)row * 128 + ((uint32_t)((col & 63) * 2) ^ ((uint32_t)(row & 7) << 4));
}
// 8 values as two fp16 terms, at the 16-byte group that holds columns col .. col + 7 of a row
__device__ __forceinline__ void store_terms(uint8_t* hi, uint8_t* lo, int row, int col, float (&v)[8]) {
    const uint32_t at = slab_at(row, col);
    store8(reinterpret_cast<__half*>(hi + at), v);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] -= __half2float(__float2half(v[j]));
    store8(reinterpret_cast<__half*>(lo + at), v);
}

__global__ void __launch_bounds__(256, 1) onchip_kernel(const __grid_constant__ Onchip p) {
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint64_t done;
    __shared__ uint32_t tmem_s;
    __shared__ int abort_s;
    __shared__ float part[8];
    uint8_t* smem = smem_raw + (((smem_u32(smem_raw) + 1023u) & ~1023u) - smem_u32(smem_raw));
    uint8_t *xh = smem, *xl = xh + kOnchipSlabs * kSlab, *sh = xl + kOnchipSlabs * kSlab, *sl = sh + 2 * kSlab;
    const uint32_t xh_a = smem_u32(xh), xl_a = smem_u32(xl), sh_a = smem_u32(sh), sl_a = smem_u32(sl);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int ctas = gridDim.x, rank = blockIdx.x, matrix = blockIdx.y;         // the cluster spans x
    const bool tall = p.rows > p.cols;
    const int k16 = (p.k + 15) & ~15;
    const int c0 = rank * p.slabs * 64, width = min(p.slabs * 64, p.l - c0);   // this CTA's columns of X
    const int slabs = (width + 63) / 64;
    const uint32_t idesc0 = (1u << 4) | ((uint32_t)(128 >> 4) << 24);           // fp16 operands, fp32 sums, M = 128
    volatile int* abort_flag = &abort_s;

    if (tid == 0) {
        abort_s = 0;
        mbar_init(&done, 1);
        fence_barrier_init();
    }
    if (warp == 0) tmem_alloc(&tmem_s, 512);
    for (uint32_t i = tid * 16; i < 2 * kOnchipSlabs * kSlab; i += 256 * 16)
        *reinterpret_cast<uint4*>(xh + i) = make_uint4(0, 0, 0, 0);             // rows past k and columns past l stay zero
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_s, d_sym = tmem, d_x = tmem + 128;
    pdl_launch_dependents();
    pdl_wait();
    if (rank == 0 && matrix == 0 && tid == 0) {
        p.status[0] = 0u;
        p.status[1] = 0u;
    }

    // ---- v' and |u|^2, then X. Threads run along the rows of the matrix as it lies.
    const long long base = (long long)matrix * p.rows * p.cols;
    const int fast = tall ? p.k : width, n = p.k * width;
    auto locate = [&](int i, int& r, int& c) -> long long {       // element i of the slice: its row and column of X, its place
        const int s = i / fast, f = i - s * fast;
        r = tall ? f : s;
        c = tall ? s : f;
        return base + (tall ? (long long)(c0 + c) * p.cols + r : (long long)r * p.cols + c0 + c);
    };
    auto load_g = [&](long long at) {
        return p.bf16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(p.grad)[at]) : static_cast<const float*>(p.grad)[at];
    };
    float sum = 0.f;
#pragma unroll 4
    for (int i = tid; i < n; i += 256) {
        int r, c;
        const long long at = locate(i, r, c);
        float u = load_g(at);
        if (p.v_in) {
            const float v = p.beta * p.v_in[at] + u;
            p.v_out[at] = v;
            u = p.nesterov ? fmaf(p.beta, v, u) : v;
        }
        sum = fmaf(u, u, sum);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (lane == 0) part[warp] = sum;
    __syncthreads();
    if (tid == 0) {
        for (int w = 1; w < 8; ++w) sum += part[w];
        p.norms[matrix * ctas + rank] = sum;
    }
    __syncthreads();
    cluster_sync();
    sum = 0.f;
    for (int i = 0; i < ctas; ++i) sum += __ldcg(p.norms + matrix * ctas + i);
    const float inv = 1.f / (sqrtf(sum) + p.eps);
#pragma unroll 4
    for (int i = tid; i < n; i += 256) {
        int r, c;
        const long long at = locate(i, r, c);
        float u;
        if (p.v_in) {
            u = p.v_out[at];         // this thread wrote it
            if (p.nesterov) u = fmaf(p.beta, u, load_g(at));
        } else {
            u = load_g(at);
        }
        u *= inv;
        const uint32_t to = slab_at(r, c);
        const __half h = __float2half(u);
        *reinterpret_cast<__half*>(xh + to) = h;
        *reinterpret_cast<__half*>(xl + to) = __float2half(u - __half2float(h));
    }
    fence_proxy_async_smem();
    __syncthreads();

    const uint32_t hi = desc_hi(1024, 2);
    const int quarter = warp & 3, half = warp >> 2;       // the TMEM lanes this warp may read; which 32-column groups
    const int row = quarter * 32 + lane;
    const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
    uint32_t phase = 0;
    bool ok = true;
    // three products of one K step: hi hi, hi lo, lo hi
    auto three = [&](uint32_t d, uint32_t ah, uint32_t al, uint32_t bh, uint32_t bl, uint32_t idesc, bool first) {
        mma_words<1>(d, ah, hi, bh, hi, idesc, first ? 0u : 1u);
        mma_words<1>(d, ah, hi, bl, hi, idesc, 1u);
        mma_words<1>(d, al, hi, bh, hi, idesc, 1u);
    };
    auto finish = [&]() {            // waits for the products that thread 0 has issued and committed
        const bool got = mbar_wait(&done, phase, abort_flag);
        phase ^= 1;
        if (!got) flag_timeout(&abort_s, p.status, 0x1500u);
        ok = ok && got;
        __syncwarp();
        tc_fence_after();
    };
    for (int step = 0; step < p.steps; ++step) {
        // ---- A = X X^T
        float a[2][32];
        if (tid == 0) {
            const uint32_t idesc = idesc0 | ((uint32_t)(k16 >> 3) << 17);
            for (int s = 0; s < slabs * 4; ++s) {
                const uint32_t off = (uint32_t)(s >> 2) * kSlab + (s & 3) * 32;
                const uint32_t h = desc_lo(xh_a + off, 16), l = desc_lo(xl_a + off, 16);
                three(d_sym, h, l, h, l, idesc, s == 0);
            }
            mma_commit(&done);
        }
        __syncwarp();
        finish();
        float* mine = p.partial + (((long long)(step & 1) * gridDim.y + matrix) * ctas + rank) * k16 * 128;
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            const int c = (g * 2 + half) * 32;
            if (c >= k16) continue;
            uint32_t r[32];
            tmem_ld32(d_sym + lanes + c, r);
#pragma unroll
            for (int j = 0; j < 32; ++j) a[g][j] = __uint_as_float(r[j]);
            if (ctas > 1 && quarter * 32 < p.k) {
#pragma unroll
                for (int j = 0; j < 32; ++j)
                    if (c + j < k16) mine[(c + j) * 128 + row] = a[g][j];
            }
        }
        if (ctas > 1) {
            __syncwarp();
            cluster_sync();
            const float* all = p.partial + ((long long)(step & 1) * gridDim.y + matrix) * ctas * k16 * 128;
#pragma unroll
            for (int g = 0; g < 2; ++g) {
                const int c = (g * 2 + half) * 32;
                if (c >= k16 || quarter * 32 >= p.k) continue;
#pragma unroll
                for (int j = 0; j < 32; ++j) a[g][j] = 0.f;
                for (int s = 0; s < ctas; ++s) {
                    const float* from = all + (long long)s * k16 * 128 + row;
#pragma unroll
                    for (int j = 0; j < 32; ++j)
                        if (c + j < k16) a[g][j] += __ldcg(from + (c + j) * 128);
                }
            }
        }
        // both terms of A, then A^2, then both terms of P in their place
        auto put = [&](auto&& value) {
#pragma unroll
            for (int g = 0; g < 2; ++g) {
                const int c = (g * 2 + half) * 32;
                if (c >= k16) continue;
#pragma unroll
                for (int j = 0; j < 32; j += 8) {
                    if (c + j >= k16 || row >= p.k) continue;
                    float v[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[i] = c + j + i < p.k ? value(g, j + i) : 0.f;
                    store_terms(sh, sl, row, c + j, v);
                }
            }
            fence_proxy_async_smem();
            tc_fence_before();
            __syncthreads();
            tc_fence_after();
        };
        put([&](int g, int j) { return a[g][j]; });
        if (tid == 0) {
            const uint32_t idesc = idesc0 | ((uint32_t)(k16 >> 3) << 17);
            for (int s = 0; s < k16 / 16; ++s) {
                const uint32_t off = (uint32_t)(s >> 2) * kSlab + (s & 3) * 32;
                const uint32_t h = desc_lo(sh_a + off, 16), l = desc_lo(sl_a + off, 16);
                three(d_sym, h, l, h, l, idesc, s == 0);
            }
            mma_commit(&done);
        }
        __syncwarp();
        finish();
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            const int c = (g * 2 + half) * 32;
            if (c >= k16) continue;
            uint32_t r[32];
            tmem_ld32(d_sym + lanes + c, r);
#pragma unroll
            for (int j = 0; j < 32; ++j) a[g][j] = fmaf(p.b, a[g][j], p.c * __uint_as_float(r[j]));
        }
        put([&](int g, int j) { return a[g][j]; });
        // ---- X <- a X + P X
        if (tid == 0) {
            const uint32_t idesc = idesc0 | (1u << 16) | ((uint32_t)(slabs * 64 >> 3) << 17);
            for (int s = 0; s < k16 / 16; ++s) {
                const uint32_t pa = (uint32_t)(s >> 2) * kSlab + (s & 3) * 32, xb = (uint32_t)s * 2048;
                three(d_x, desc_lo(sh_a + pa, 16), desc_lo(sl_a + pa, 16), desc_lo(xh_a + xb, kSlab), desc_lo(xl_a + xb, kSlab),
                      idesc, s == 0);
            }
            mma_commit(&done);
        }
        __syncwarp();
        finish();
        const bool last = step + 1 == p.steps;
#pragma unroll 1
        for (int c = half * 32; c < slabs * 64; c += 64) {
            uint32_t r[32];
            tmem_ld32(d_x + lanes + c, r);
            if (row < p.k) {
#pragma unroll
                for (int j = 0; j < 32; j += 8) {
                    const uint32_t at = slab_at(row, c + j);
                    float v[8], w[8];
                    load8(reinterpret_cast<const __half*>(xh + at), v);
                    load8(reinterpret_cast<const __half*>(xl + at), w);
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[i] = fmaf(p.a, v[i] + w[i], __uint_as_float(r[j + i]));
                    if (!last) {
                        store_terms(xh, xl, row, c + j, v);
                        continue;
                    }
                    const int col = c0 + c + j;
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[i] *= p.scale;
                    if (!tall && p.cols % 8 == 0) {
                        if (col < p.l) store8(p.update + base + (long long)row * p.cols + col, v);
                        continue;
                    }
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if (col + i < p.l)
                            p.update[base + (tall ? (long long)(col + i) * p.cols + row : (long long)row * p.cols + col + i)] =
                                __float2bfloat16(v[i]);
                }
            }
            __syncwarp();
        }
        fence_proxy_async_smem();
        tc_fence_before();
        __syncthreads();
        tc_fence_after();
    }
    if (p.steps == 0) {
        for (int i = tid; i < n; i += 256) {
            int r, c;
            const long long at = locate(i, r, c);
            const uint32_t from = slab_at(r, c);
            p.update[at] = __float2bfloat16(p.scale * (__half2float(*reinterpret_cast<__half*>(xh + from)) +
                                                       __half2float(*reinterpret_cast<__half*>(xl + from))));
        }
    }
    __syncwarp();
    __syncthreads();
    if (warp == 0) tmem_dealloc(tmem, 512);
}

}  // namespace
}  // namespace ac
