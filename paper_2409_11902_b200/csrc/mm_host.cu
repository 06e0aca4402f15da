// Host side of the shared matrix product: tensor maps, tile grids and the choice of the tile shape.
#include "mm_core.cuh"

namespace ac {
namespace mm {

namespace {

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                  const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiledFn encode_fn() {
    static const EncodeTiledFn fn = [] {
        void* f = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &f, cudaEnableDefault, &q) == cudaSuccess &&
            q == cudaDriverEntryPointSuccess)
            return reinterpret_cast<EncodeTiledFn>(f);
        return static_cast<EncodeTiledFn>(nullptr);
    }();
    return fn;
}

int ceil_div(long long a, long long b) { return (int)((a + b - 1) / b); }

}  // namespace

// K-major: a box of 64 elements of K by `tile_rows` rows. MN-major: 64 elements of M/N by 64 rows of K, one such slab
// per 64 rows of the tile. Elements beyond the extents read as zero, so ragged sizes need no masks in the products.
ac_status make_map(CUtensorMap* map, const Operand& o, bool bf16, int tile_rows) {
    const EncodeTiledFn enc = encode_fn();
    if (!enc) return AC_ERR_CUDA;
    const cuuint64_t dims[3] = {(cuuint64_t)o.inner, (cuuint64_t)o.rows, (cuuint64_t)o.batch};
    const cuuint64_t strides[2] = {(cuuint64_t)o.pitch * 2, (cuuint64_t)(o.batch > 1 ? o.stride : o.pitch * o.rows) * 2};
    const cuuint32_t box[3] = {64, (cuuint32_t)(o.mn ? 64 : tile_rows), 1}, es[3] = {1, 1, 1};
    if (enc(map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, const_cast<void*>(o.p),
            dims, strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
            CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
        return AC_ERR_CUDA;
    return AC_OK;
}

Params make_params(int m, int n, long long k, int batch, int cg, int bn, bool a_mn, bool b_mn, bool bf16, bool sym) {
    Params p{};
    p.m = m;
    p.n = n;
    p.ktiles = ceil_div(k, kBK);
    p.tiles_m = ceil_div(m, 128 * cg);
    p.tiles_n = ceil_div(n, bn);
    p.sym = sym;
    p.per_batch = sym ? p.tiles_n * (p.tiles_n + 1) / 2 : p.tiles_m * p.tiles_n;
    p.tiles = p.per_batch * batch;
    // The smaller operand is cycled through while the larger one streams past once, as far as the panels of the
    // smaller one fit a third of the L2 (126 MB); at least 8 tiles, so that the tiles in flight stay squarish.
    p.fast_m = m <= n;
    const long long panel = (p.fast_m ? 128ll * cg : bn) * k * 2;
    long long g = (40ll << 20) / panel;
    const int tf = p.fast_m ? p.tiles_m : p.tiles_n;
    p.group = (int)(g < 8 ? 8 : g);
    if (p.group > tf) p.group = tf;
    p.split = 1;
    const uint32_t type = bf16 ? 1u : 0u;
    p.idesc = (1u << 4) | (type << 7) | (type << 10) | ((a_mn ? 1u : 0u) << 15) | ((b_mn ? 1u : 0u) << 16) |
              ((uint32_t)(bn >> 3) << 17) | ((uint32_t)(128 * cg >> 4) << 24);
    return p;
}

bool use_pairs(int m, int n, long long k, int batch, bool sym, int* split) {
    const int tm = ceil_div(m, 256), tn = ceil_div(n, 256);
    const long long large = (long long)(sym ? tn * (tn + 1) / 2 : tm * tn) * batch;
    *split = 1;
    if (large >= kNumSMs / 2) return true;
    const int sm = ceil_div(m, 128), sn = ceil_div(n, 128);
    const long long small = (long long)(sym ? sn * (sn + 1) / 2 : sm * sn) * batch;
    const int ktiles = ceil_div(k, kBK);
    // as many slices as leave every SM at most one CTA, each at least two K-tiles long
    while (*split < kMaxSplit && small * *split * 2 <= kNumSMs && ktiles >= *split * 4) *split *= 2;
    return false;
}

}  // namespace mm
}  // namespace ac
