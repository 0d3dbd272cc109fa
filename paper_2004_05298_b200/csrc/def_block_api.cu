// C boundary of the operators between a model's input and its gradient rows (see include/def_train.h): recurrence over tokens.
#include "def_recurrence_kernels.cuh"
#include "def_train_checks.cuh"

// ---------------------------------------------------------------------------
// Recurrence
// ---------------------------------------------------------------------------
namespace {

constexpr int64_t kMostSteps = (int64_t)1 << 30;

// How a call is cut: channels per CTA, CTAs of a cluster along time, parts of time.
struct RecurrencePlan {
    int lanes, tiles, ranks, parts, part_steps;
};
RecurrencePlan recurrence_plan(int64_t T, int64_t C, int lanes) {
    RecurrencePlan p;
    p.lanes = lanes;
    p.tiles = (int)ceil_div(C, 32 * lanes);
    const int64_t blocks = ceil_div(T, deft::kRecSteps);
    p.ranks = 1;
    p.parts = 1;
    while (p.ranks < deft::kMostCluster && p.ranks * 2 <= blocks && (int64_t)p.tiles * p.ranks < 2 * kUsualSms) p.ranks *= 2;
    int64_t each = blocks;
    if ((int64_t)p.tiles * p.ranks < kUsualSms / 2 && blocks > p.ranks) {
        p.ranks = 1;
        const int64_t want = ceil_div(3 * kUsualSms, p.tiles), most = want < deft::kMostParts ? want : (int64_t)deft::kMostParts;
        each = ceil_div(blocks, blocks < most ? blocks : most);
        p.parts = (int)ceil_div(blocks, each);
    }
    p.part_steps = (int)((each > 0 ? each : 1) * deft::kRecSteps);
    return p;
}
int64_t recurrence_bytes(const RecurrencePlan &p, int64_t C) { return p.parts > 1 ? (int64_t)p.parts * C * 8 : 0; }

// Two 16-bit elements at a time need even strides, an even width and 4-byte bases; the workspace is sized for either way.
int64_t recurrence_need(int32_t dtype, int64_t T, int64_t C) {
    const int64_t one = recurrence_bytes(recurrence_plan(T, C, 1), C), two = recurrence_bytes(recurrence_plan(T, C, 2), C);
    return element_size(dtype) == 2 && two > one ? two : one;
}

template <bool BACK> int recurrence(int32_t dtype, deft::Recurrence a, bool pairs, cudaStream_t stream, const char *what) {
    const RecurrencePlan p = recurrence_plan(a.T, a.C, pairs ? 2 : 1);
    a.tiles = p.tiles;
    a.parts = p.parts;
    a.part_steps = p.part_steps;
    cudaError_t err = cudaSuccess;
    by_dtype(dtype, [&](auto type) {
        using E = decltype(type);
        auto launch = [&](auto kernel, int ranks, int parts) {
            cudaLaunchConfig_t cfg = {};
            cfg.gridDim = dim3((unsigned)(p.tiles * ranks), (unsigned)parts);
            cfg.blockDim = dim3(32 * deft::kRecWarps);
            cfg.stream = stream;
            cudaLaunchAttribute attr[1];
            attr[0].id = cudaLaunchAttributeClusterDimension;
            attr[0].val.clusterDim.x = (unsigned)ranks;
            attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
            cfg.attrs = attr;
            cfg.numAttrs = ranks > 1 ? 1 : 0;
            if (err == cudaSuccess) err = cudaLaunchKernelEx(&cfg, kernel, a, ranks);
        };
        auto both = [&](auto v) {
            constexpr int V = decltype(v)::value ? 2 : 1;
            if (p.parts > 1) launch(deft::recurrence_kernel<E, V, BACK, true>, 1, p.parts - 1);
            launch(deft::recurrence_kernel<E, V, BACK, false>, p.ranks, p.parts);
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

bool even(const void *p, int64_t ld) { return ((uintptr_t)p & 3u) == 0 && ld % 2 == 0; }

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
    const bool pairs = es == 2 && C % 2 == 0 && even(x, ldx) && even(gate, ldg) && even(y, ldy);
    return recurrence<false>(dtype, a, pairs, (cudaStream_t)cuda_stream, "def_recurrence_forward");
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
    const bool pairs = es == 2 && C % 2 == 0 && even(dy, lddy) && even(x, ldx) && even(gate, ldg) && even(y, ldy) && even(dx, lddx) && even(dgate, lddg);
    return recurrence<true>(dtype, a, pairs, (cudaStream_t)cuda_stream, "def_recurrence_backward");
}
