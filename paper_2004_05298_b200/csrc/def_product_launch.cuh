// Host side of the products on tensor cores: operands, their tensor maps, the launch.
#pragma once

#include "def_planes_kernels.cuh"
#include "def_product_kernels.cuh"
#include "def_train_checks.cuh"

namespace {

// An operand [rows, cols] as the kernels take it: where it lies, or the 16-bit pieces that a copy of it is cut into.
struct Operand {
    const void *p;
    int64_t rows, cols, ld;
    bool copy;
    int planes;
    int64_t bytes;                          // of the copy
};
Operand operand(int32_t dtype, const void *p, int64_t rows, int64_t cols, int64_t ld) {
    const int es = element_size(dtype);
    Operand o = {p, rows, cols, rows > 1 ? ld : ceil_div(cols, 8) * 8, false, es == 4 ? 3 : 1, 0};
    o.copy = es == 4 || !wide(p, o.ld, es) || o.ld >= ((int64_t)1 << 40) / es;
    if (o.copy) {
        o.ld = ceil_div(cols, 8) * 8;
        o.bytes = o.planes * rows * o.ld * 2;
    }
    return o;
}
// Where the copy goes in the workspace; `at` moves on behind it.
void place(Operand &o, char *&at) {
    if (!o.copy) return;
    o.p = at;
    at += o.bytes;
}
// The copies of those of N operands that need one, in one launch.
template <int N> int fill(const Operand (&o)[N], int32_t dtype, const void *const (&from)[N], const int64_t (&ld)[N], cudaStream_t stream, const char *what) {
    deft::Planes p = {};
    int n = 0;
    int64_t lanes = 0, rows = 0;
    for (int i = 0; i < N; ++i) {
        if (!o[i].copy) continue;
        p.of[n++] = {from[i], (uint4 *)const_cast<void *>(o[i].p), ld[i], o[i].rows, o[i].ld, (int)o[i].cols};
        lanes = std::max(lanes, ceil_div(o[i].cols, 8));
        rows = std::max(rows, o[i].rows);
    }
    if (n == 0) return DEF_OK;
    on_plane(false, rows, lanes * 8, [&](auto, dim3 grid, dim3 block) {
        grid.z = (unsigned)n;
        if (dtype == DEF_DTYPE_F32) deft::planes_kernel<float><<<grid, block, 0, stream>>>(p);
        else deft::planes_kernel<__half><<<grid, block, 0, stream>>>(p);
    });
    return launched(what);
}

// Map of [z][rows][cols] 16-bit elements in boxes of 64 columns and `box_rows` rows.
int operand_map(CUtensorMap &map, bool half, const void *p, int64_t cols, int64_t rows, int64_t z, int64_t ld, int box_rows) {
    const EncodeTiled encode = encode_tiled();
    if (!encode) return fail(DEF_ERR_CUDA, "the driver does not offer tensor maps");
    const cuuint64_t dim[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)z}, stride[2] = {(cuuint64_t)ld * 2, (cuuint64_t)ld * 2 * (cuuint64_t)(z > 1 ? rows : 1)};
    const cuuint32_t box[3] = {64, (cuuint32_t)box_rows, 1}, one[3] = {1, 1, 1};
    if (encode(&map, half ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void *>(p), dim, stride, box, one,
               CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
        return fail(DEF_ERR_CUDA, "the driver refused a tensor map");
    return DEF_OK;
}
int operand_map(CUtensorMap &map, int32_t dtype, const Operand &o, bool k_rows) {
    return operand_map(map, dtype == DEF_DTYPE_F16, o.p, o.cols, o.rows, o.planes, o.ld, k_rows ? deft::kTileK : deft::kTileRows);
}

// fp32 values in three bf16 pieces of 8 bits each: the six products above 2^-24, small ones first.
deft::Product product_of(int32_t dtype, int64_t m, int64_t tiles_n, int64_t k, int step_n, int second) {
    deft::Product p = {};
    p.tiles_m = (int)ceil_div(m, 2 * deft::kTileRows);
    p.tiles_n = (int)tiles_n;
    p.batch = 1;
    p.blocks = (int)ceil_div(k, deft::kTileK);
    const bool pieces = dtype == DEF_DTYPE_F32;
    p.pairs = pieces ? 6 : 1;
    p.planes_a = p.planes_b = pieces ? 3 : 1;
    p.order_a = pieces ? 0x001102u : 0u;
    p.order_b = pieces ? 0x010120u : 0u;
    p.step_n = step_n;
    p.second = second;
    p.bf16 = dtype != DEF_DTYPE_F16;
    return p;
}

// How tiles that do not fill a round of the pairs are cut along k.  Each part has `least` stages (pieces with short chains, whose
// results take long to store: 2, 100 x 8000 orthogonalised 282 against 261 us; else 4, 512 x 512 x 1408 bf16 forward 28 against 29),
// and the cut has to save kJoinStages, which are worth the join, a launch and a pass over the parts.
constexpr int kJoinStages = 4;
constexpr int64_t kMostPartBytes = (int64_t)kUsualSms * deft::kPartFloats * 4;
int64_t plan_cuts(deft::Product &p, int64_t most_bytes = kMostPartBytes, int least = 4) {
    const int64_t tiles = deft::product_tiles(p), workers = kUsualSms / 2, rest = tiles % workers, each = 2 * deft::kPartFloats * 4;
    const int per_tile = p.blocks * p.pairs;
    p.whole = tiles;
    p.cuts = 1;
    if (rest == 0) return 0;
    int64_t cuts = workers / rest;
    if (cuts > per_tile / least) cuts = per_tile / least;
    if (cuts > most_bytes / (rest * each)) cuts = most_bytes / (rest * each);
    if (cuts < 2 || per_tile - per_tile / cuts < kJoinStages) return 0;
    p.whole = tiles - rest;
    p.cuts = (int)cuts;
    return rest * cuts * each;
}

template <bool BN, int CHAIN, typename EPILOGUE>
int launch_product(const deft::Product &p, const EPILOGUE &epilogue, const CUtensorMap &map_a, const CUtensorMap &map_b, cudaStream_t stream, const char *what) {
    using S = deft::ProductShape<EPILOGUE, CHAIN>;
    constexpr auto kernel = deft::product_kernel<EPILOGUE, BN, CHAIN>;
    if (deft::product_pieces(p) >= (int64_t)1 << 30) return fail(DEF_ERR_ARG, "%s: the result is too large", what);
    cudaError_t err = allow_smem<kernel>(S::smem);
    if (err == cudaSuccess) {
        const int64_t pieces = deft::product_pieces(p);
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3((unsigned)((pieces < kUsualSms / 2 ? pieces : kUsualSms / 2) * 2));
        deft::Product q = p;
        q.early = pieces <= kUsualSms / 4;
        cfg.blockDim = dim3(S::threads);
        cfg.dynamicSmemBytes = S::smem;
        cfg.stream = stream;
        cudaLaunchAttribute attr[2];
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = 2;
        attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
        attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[1].val.programmaticStreamSerializationAllowed = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 2;
        err = cudaLaunchKernelEx(&cfg, kernel, q, epilogue, map_a, map_b);
        if (const int64_t cut = deft::product_tiles(p) - p.whole; cut > 0 && err == cudaSuccess) {
            cfg.gridDim = dim3((unsigned)(cut * (EPILOGUE::kBoth ? 8 : 16)));
            cfg.blockDim = dim3(deft::kJoinThreads);
            cfg.dynamicSmemBytes = 0;
            cfg.attrs = attr + 1;
            cfg.numAttrs = 1;
            err = cudaLaunchKernelEx(&cfg, deft::product_join_kernel<EPILOGUE>, q, epilogue);
        }
    }
    if (err == cudaSuccess) return DEF_OK;
    cudaGetLastError();
    return cuda_fail(err, what);
}

}  // namespace
