// C boundary of the operators between a model's input and its gradient rows (see include/def_train.h): recurrence over tokens.
#include <algorithm>

#include "def_recurrence_kernels.cuh"
#include "def_train_checks.cuh"

// ---------------------------------------------------------------------------
// Recurrence
// ---------------------------------------------------------------------------
namespace {

constexpr int64_t kMostSteps = (int64_t)1 << 30;
// Up to this many steps rows are read element by element, without tensor maps, which cost the host some 0.5 us a call.  Elements against
// copies, us, 2048 channels bf16: 64 steps 9.1 against 9.6, 128 9.1 against 9.6, 192 9.6 against 9.7, 1024 11.6 against 9.9; 8192 channels:
// 128 steps 9.4 against 9.9, 192 11.1 against 10.0, 512 15.4 against 11.6; backward 128 12.3 against 12.4, 192 17.5 against 12.9.  (fp32 backward
// of 2048 channels stays ahead by elements up to 1024 steps, 17.6 against 24.9, and of 8192 up to 256, 17.5 against 19.6.)
constexpr int64_t kFewSteps = 64;

// Where even clusters leave SMs idle, long calls are cut into parts, whose maps a first kernel finds, reading the gate and x (or
// dy) once more.  Clusters against parts, forward and back, us: 16384 x 1024 bf16 70 against 44, 100 against 60; 65536 x 1024 210
// against 162, 339 against 250; 16384 x 2048 74 against 86, 109 against 123; few rounds: 2048 x 1024 15 against 18, 21 each.
constexpr int kFewRounds = 4;
// How a call is cut: channels per CTA, CTAs of a cluster along time, parts of time.
struct RecurrencePlan {
    int tiles, ranks, parts, part_steps;
};
RecurrencePlan recurrence_plan(int64_t T, int64_t C, int lanes, int steps, int ctas) {
    RecurrencePlan p;
    p.tiles = (int)ceil_div(C, 32 * lanes);
    const int64_t blocks = ceil_div(T, steps);
    p.ranks = 1;
    p.parts = 1;
    while (p.ranks < deft::kMostCluster && p.ranks * 2 <= blocks && (int64_t)p.tiles * p.ranks * 2 <= ctas * kUsualSms) p.ranks *= 2;
    int64_t each = blocks;
    if ((int64_t)p.tiles * p.ranks < kUsualSms && blocks > kFewRounds * p.ranks) {
        p.ranks = 1;
        const int64_t space = 1 + 4096 * C / (ceil_div(C, 64) * 64 * 8);      // parts that the documented workspace has room for
        const int64_t want = std::min(ceil_div(ctas * kUsualSms, p.tiles), space), most = std::min<int64_t>(want, deft::kMostParts);
        each = ceil_div(blocks, blocks < most ? blocks : most);
        p.parts = (int)ceil_div(blocks, each);
    }
    p.part_steps = (int)((each > 0 ? each : 1) * steps);
    return p;
}
constexpr int kMostCtas = 4, kShortBlock = 64, kLongBlock = 128;
// The workspace is sized for every form a call of this size may take.
int64_t recurrence_need(int32_t dtype, int64_t T, int64_t C) {
    int64_t parts = 1;
    for (int lanes = 1; lanes <= 2; ++lanes)
        for (int steps : {kShortBlock, kLongBlock})
            for (int ctas = 2; ctas <= kMostCtas; ++ctas) {
                const int64_t n = recurrence_plan(T, C, lanes, steps, ctas).parts;
                if (n > parts) parts = n;
            }
    return parts > 1 ? (parts - 1) * ceil_div(C, 64) * 64 * 8 : 0;
}

// Rows that a tensor map takes, in boxes of 64 columns by the steps of a block.
bool mapped(const void *p, int64_t ld, int64_t T, int64_t es) { return ((uintptr_t)p & 15u) == 0 && (T == 1 || (ld * es % 16 == 0 && ld * es < (int64_t)1 << 40)); }
int rows_map(CUtensorMap &map, int32_t dtype, const void *p, int64_t T, int64_t C, int64_t ld, int steps) {
    const EncodeTiled encode = encode_tiled();
    if (!encode) return fail(DEF_ERR_CUDA, "the driver does not offer tensor maps");
    const cuuint64_t es = element_size(dtype), dim[2] = {(cuuint64_t)C, (cuuint64_t)T}, stride[1] = {T > 1 ? (cuuint64_t)ld * es : (cuuint64_t)ceil_div(C * es, 16) * 16};
    const cuuint32_t box[2] = {64, (cuuint32_t)steps}, one[2] = {1, 1};
    const CUtensorMapDataType type = dtype == DEF_DTYPE_F32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : dtype == DEF_DTYPE_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
    if (encode(&map, type, 2, const_cast<void *>(p), dim, stride, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE,
               CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
        return fail(DEF_ERR_CUDA, "the driver refused a tensor map");
    return DEF_OK;
}

// `pairs`: 16-bit rows can be read two elements at a time; `streamed`: rows can be copied by tensor maps, too.
template <bool BACK> int recurrence(int32_t dtype, deft::Recurrence a, bool pairs, bool streamed, cudaStream_t stream, const char *what) {
    int ctas = kMostCtas, steps = deft::kRecSteps;
    if (streamed)
        by_dtype(dtype, [&](auto type) {
            using B = deft::StreamBlock<decltype(type), BACK>;
            static_assert(B::steps == kLongBlock || B::steps == kShortBlock);
            static_assert(B::ctas >= 2 && B::ctas <= kMostCtas && (deft::kRecSteps == kLongBlock || deft::kRecSteps == kShortBlock));
            ctas = B::ctas;
            steps = B::steps;
        });
    const RecurrencePlan p = recurrence_plan(a.T, a.C, streamed || pairs ? 2 : 1, steps, ctas);
    a.tiles = p.tiles;
    a.parts = p.parts;
    a.part_steps = p.part_steps;
    deft::RecurrenceMaps maps = {};
    if (streamed) {
        DEF_TRY(rows_map(maps.gate, dtype, a.gate, a.T, a.C, a.ldg, steps));
        DEF_TRY(rows_map(maps.first, dtype, BACK ? a.dy : a.x, a.T, a.C, BACK ? a.lddy : a.ldx, steps));
        if (BACK) {
            DEF_TRY(rows_map(maps.x, dtype, a.x, a.T, a.C, a.ldx, steps));
            DEF_TRY(rows_map(maps.y, dtype, a.y, a.T, a.C, a.ldy, steps));
        }
    }
    const bool handed = (BACK ? a.dh0 : a.h_last) != nullptr;
    cudaError_t err = cudaSuccess;
    by_dtype(dtype, [&](auto type) {
        using E = decltype(type);
        // `after`: the launch may overlap the end of the one before, which finds the parts' maps
        auto launch = [&](auto kernel, int smem, int ranks, int parts, bool after, auto... args) {
            cudaLaunchConfig_t cfg = {};
            cfg.gridDim = dim3((unsigned)(p.tiles * ranks), (unsigned)parts);
            cfg.blockDim = dim3(32 * deft::kRecWarps);
            cfg.dynamicSmemBytes = (size_t)smem;
            cfg.stream = stream;
            cudaLaunchAttribute attr[2];
            attr[0].id = cudaLaunchAttributeClusterDimension;
            attr[0].val.clusterDim.x = (unsigned)ranks;
            attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
            attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
            attr[1].val.programmaticStreamSerializationAllowed = 1;
            cfg.attrs = ranks > 1 ? attr : attr + 1;
            cfg.numAttrs = (ranks > 1 ? 1 : 0) + (after ? 1 : 0);
            if (err == cudaSuccess) err = cudaLaunchKernelEx(&cfg, kernel, a, ranks, args...);
        };
        if (streamed) {
            constexpr int smem = deft::StreamBlock<E, BACK>::smem, part_smem = deft::StreamBlock<E, BACK>::part_smem;
            constexpr auto part = deft::recurrence_stream_kernel<E, BACK, true, false>;
            if (p.parts > 1 && (err = allow_smem<part>(part_smem)) != cudaSuccess) return;
            const auto both = [&](auto is_handed) {
                constexpr auto whole = deft::recurrence_stream_kernel<E, BACK, false, decltype(is_handed)::value>;
                if ((err = allow_smem<whole>(smem)) != cudaSuccess) return;
                if (p.parts > 1) launch(part, part_smem, 1, p.parts - 1, false, maps);
                launch(whole, smem, p.ranks, p.parts, p.parts > 1, maps);
            };
            by_alignment(handed, both);
            return;
        }
        auto both = [&](auto v) {
            constexpr int V = decltype(v)::value ? 2 : 1;
            if (p.parts > 1) launch(deft::recurrence_kernel<E, V, BACK, true, false>, 0, 1, p.parts - 1, false);
            by_alignment(handed, [&](auto is_handed) { launch(deft::recurrence_kernel<E, V, BACK, false, decltype(is_handed)::value>, 0, p.ranks, p.parts, false); });
        };
        if constexpr (sizeof(E) == 2) by_alignment(pairs, both);
        else both(Is<false>());
    });
    if (err != cudaSuccess) {
        cudaGetLastError();
        return cuda_fail(err, what);
    }
    return DEF_OK;
}

// Whether two elements at a time can be read and written.
bool even(const void *p, int64_t ld, int64_t es) { return ((uintptr_t)p & (unsigned)(2 * es - 1)) == 0 && ld % 2 == 0; }

int check_sequences(int64_t T, int64_t sequences, const int64_t *offsets) {
    if (T > kMostSteps) return fail(DEF_ERR_ARG, "T must be at most 2^30 (got %lld)", (long long)T);
    if (sequences < 1 || sequences > kMostSteps) return fail(DEF_ERR_ARG, "sequences must be in [1, 2^30] (got %lld)", (long long)sequences);
    if (!offsets && T % sequences) return fail(DEF_ERR_ARG, "without offsets, sequences must divide T (got %lld sequences, %lld rows)", (long long)sequences, (long long)T);
    return DEF_OK;
}

}  // namespace

extern "C" int def_recurrence_workspace(int32_t dtype, int64_t T, int64_t C, int64_t *bytes_out) {
    if (!bytes_out) return fail(DEF_ERR_NULL, "bytes_out must not be NULL");
    DEF_TRY(check_rows(dtype, T, C, "C"));
    DEF_TRY(check_sequences(T, 1, nullptr));
    *bytes_out = recurrence_need(dtype, T, C);
    return DEF_OK;
}

extern "C" int def_recurrence_forward(int32_t dtype, int64_t T, int64_t C, int64_t sequences, const int64_t *offsets, const void *x,
                                      int64_t ldx, const void *gate, int64_t ldg, const float *h0, void *y, int64_t ldy, float *h_last,
                                      void *workspace, int64_t workspace_bytes, void *cuda_stream) {
    int64_t need = 0;
    DEF_TRY(def_recurrence_workspace(dtype, T, C, &need));
    DEF_TRY(check_sequences(T, sequences, offsets));
    if (T > 0 && (!x || !gate || !y)) return fail(DEF_ERR_NULL, "x, gate and y must not be NULL");
    DEF_TRY(check_stride(x, ldx, C, T, "x"));
    DEF_TRY(check_stride(gate, ldg, C, T, "gate"));
    DEF_TRY(check_stride(y, ldy, C, T, "y"));
    if (need > 0 && !workspace) return fail(DEF_ERR_NULL, "workspace must not be NULL");
    if (workspace_bytes < need) return fail(DEF_ERR_ARG, "the workspace must have %lld bytes (got %lld)", (long long)need, (long long)workspace_bytes);
    const int es = element_size(dtype);
    const View views[] = {rows_view(x, "x", T, C, ldx, es, false), rows_view(y, "y", T, C, ldy, es, true), rows_view(gate, "gate", T, C, ldg, es, false),
                          {offsets, "offsets", 1, (sequences + 1) * 8, (sequences + 1) * 8, 8, false}, floats_view(h0, "h0", sequences * C, false),
                          floats_view(h_last, "h_last", sequences * C, true), {workspace, "workspace", need > 0 ? 1 : 0, need, need, 16, true}};
    DEF_TRY(check_views(views, 0, 1));
    if (T == 0 && !h_last) return DEF_OK;
    if (const int sms = sm_count(); sms < 0) return sms;
    deft::Recurrence a = {};
    a.x = x; a.gate = gate; a.y = y;
    a.ldx = ldx; a.ldg = ldg; a.ldy = ldy;
    a.h0 = h0; a.h_last = h_last; a.offsets = offsets; a.sequences = sequences;
    a.T = (int)T; a.C = (int)C; a.each = (int)(T / sequences); a.summary = (float2 *)workspace;
    const bool pairs = C % 2 == 0 && even(x, ldx, es) && even(gate, ldg, es) && even(y, ldy, es);
    const bool streamed = T > kFewSteps && pairs && mapped(x, ldx, T, es) && mapped(gate, ldg, T, es);
    return recurrence<false>(dtype, a, pairs && es == 2, streamed, (cudaStream_t)cuda_stream, "def_recurrence_forward");
}

extern "C" int def_recurrence_backward(int32_t dtype, int64_t T, int64_t C, int64_t sequences, const int64_t *offsets, const void *dy,
                                       int64_t lddy, const float *dh_last, const void *x, int64_t ldx, const void *gate, int64_t ldg,
                                       const void *y, int64_t ldy, const float *h0, void *dx, int64_t lddx, void *dgate, int64_t lddg,
                                       float *dh0, void *workspace, int64_t workspace_bytes, void *cuda_stream) {
    int64_t need = 0;
    DEF_TRY(def_recurrence_workspace(dtype, T, C, &need));
    DEF_TRY(check_sequences(T, sequences, offsets));
    if (T > 0 && (!dy || !x || !gate || !y || !dx || !dgate)) return fail(DEF_ERR_NULL, "dy, x, gate, y, dx and dgate must not be NULL");
    DEF_TRY(check_stride(dy, lddy, C, T, "dy"));
    DEF_TRY(check_stride(x, ldx, C, T, "x"));
    DEF_TRY(check_stride(gate, ldg, C, T, "gate"));
    DEF_TRY(check_stride(y, ldy, C, T, "y"));
    DEF_TRY(check_stride(dx, lddx, C, T, "dx"));
    DEF_TRY(check_stride(dgate, lddg, C, T, "dgate"));
    if (need > 0 && !workspace) return fail(DEF_ERR_NULL, "workspace must not be NULL");
    if (workspace_bytes < need) return fail(DEF_ERR_ARG, "the workspace must have %lld bytes (got %lld)", (long long)need, (long long)workspace_bytes);
    const int es = element_size(dtype);
    const View views[] = {rows_view(dy, "dy", T, C, lddy, es, false), rows_view(x, "x", T, C, ldx, es, false), rows_view(gate, "gate", T, C, ldg, es, false),
                          rows_view(y, "y", T, C, ldy, es, false), rows_view(dx, "dx", T, C, lddx, es, true), rows_view(dgate, "dgate", T, C, lddg, es, true),
                          {offsets, "offsets", 1, (sequences + 1) * 8, (sequences + 1) * 8, 8, false}, floats_view(h0, "h0", sequences * C, false),
                          floats_view(dh_last, "dh_last", sequences * C, false), floats_view(dh0, "dh0", sequences * C, true),
                          {workspace, "workspace", need > 0 ? 1 : 0, need, need, 16, true}};
    DEF_TRY(check_views(views));
    if (T == 0 && !dh0) return DEF_OK;
    if (const int sms = sm_count(); sms < 0) return sms;
    deft::Recurrence a = {};
    a.x = x; a.gate = gate; a.dy = dy; a.y = const_cast<void *>(y); a.dx = dx; a.dgate = dgate;
    a.ldx = ldx; a.ldg = ldg; a.ldy = ldy; a.lddy = lddy; a.lddx = lddx; a.lddg = lddg;
    a.h0 = h0; a.dh_last = dh_last; a.dh0 = dh0; a.offsets = offsets; a.sequences = sequences;
    a.T = (int)T; a.C = (int)C; a.each = (int)(T / sequences); a.summary = (float2 *)workspace;
    const bool pairs = C % 2 == 0 && even(dy, lddy, es) && even(x, ldx, es) && even(gate, ldg, es) && even(y, ldy, es) && even(dx, lddx, es) && even(dgate, lddg, es);
    const bool streamed = T > kFewSteps && pairs && mapped(dy, lddy, T, es) && mapped(x, ldx, T, es) && mapped(gate, ldg, T, es) && mapped(y, ldy, T, es);
    return recurrence<true>(dtype, a, pairs && es == 2, streamed, (cudaStream_t)cuda_stream, "def_recurrence_backward");
}
