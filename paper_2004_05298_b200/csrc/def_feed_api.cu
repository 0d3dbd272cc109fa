// C boundary of the gated feed-forward block (see include/def_train.h).
#include <algorithm>
#include <type_traits>

#include "def_feed_kernels.cuh"
#include "def_product_launch.cuh"

namespace {

constexpr int64_t kShortSums = 1024;          // terms up to which chains are 4 stages
// Stages of 64 terms after which a sum that is stored in 16 bits moves on to registers.  The matrix unit truncates: sums of one sign
// came out 1.6 to 1.7 2^-24 low for every 16 terms, 4096 terms of fp16 2.5 10^-5, 32768 of bf16 2.1 10^-4, each a 19th of half a step of
// the type, and without a limit 2^17 terms 8.3 10^-4.  Shorter sums stay where they are until their end: emptying costs 2 to 5 %
// (8192 x 4096 x 20480 bf16, 950 to 1001 us against 996 to 1015 with 64 stages, 1071 to 1080 with 16).
template <typename E> constexpr int kLongChain = std::is_same_v<E, __half> ? 64 : 512;

// Two products, one after the other, and their operands; the parts of cut tiles come first in the workspace.
struct FeedPlan {
    Operand a1, b1, a2, b2;
    deft::Product first, second;
    int64_t parts;
    int64_t bytes() const { return parts + a1.bytes + b1.bytes + a2.bytes + b2.bytes; }
    void put(void *workspace) {
        first.parts = second.parts = (float *)workspace;
        char *at = (char *)workspace + parts;
        for (Operand *o : {&a1, &b1, &a2, &b2}) place(*o, at);
    }
};
// x [T, C] and w_in [2F, C]; h [T, F] and w_down [O, F] (w_down NULL: without the second product).
FeedPlan feed_plan(int32_t dtype, int64_t T, int64_t C, int64_t F, int64_t O, const void *x, int64_t ldx, const void *w_in, const void *w_down, const void *h,
                   int64_t ldh) {
    FeedPlan p = {operand(dtype, x, T, C, ldx), operand(dtype, w_in, 2 * F, C, C)};
    p.first = product_of(dtype, T, ceil_div(F, deft::kTileRows), C, deft::kTileRows, (int)F);
    p.parts = plan_cuts(p.first);
    if (w_down) {
        p.a2 = operand(dtype, h, T, F, ldh);
        p.b2 = operand(dtype, w_down, O, F, F);
        p.second = product_of(dtype, T, ceil_div(O, deft::kTileCols), F, deft::kTileCols, deft::kTileRows);
        p.parts = std::max(p.parts, plan_cuts(p.second));
    }
    return p;
}
// How few tokens without checkpoints are worked on: as columns of products whose rows are the weights (16 bits, in place), or
// against rows of the weights read by warps (fp32, or rows off 16-byte boundaries).  Against the products of more tokens, us: columns, 2048
// x 5632 bf16, 1 token 21.6 against 44.0, 16 24 against 38, 32 27.3 against 38.1, 512 x 1408 32 tokens 15.3 against 24.8 (33 tokens: 38.1
// and 25.1; wider columns are not built); rows, 2048 x 5632 fp32, 1 token 33.5 against 203, 8 89 against 180, 512 x 1408 8 tokens 21.3
// against 52 (9 tokens: 184 and 52; longer runs of tokens are not built).
enum class Few { no, columns, rows };
Few few_tokens(int32_t dtype, int64_t T, bool checkpoints, const FeedPlan &p) {
    const bool copied = p.a1.copy || p.b1.copy || p.a2.copy || p.b2.copy;
    if (checkpoints) return Few::no;
    if (element_size(dtype) == 2 && !copied && T <= deft::kMostTokens) return Few::columns;
    return T <= deft::kFewTokens ? Few::rows : Few::no;
}
// dout [T, O] and w_down [O, F]; dboth [T, 2F] and w_in [2F, C] (w_in NULL: without the second product).
FeedPlan back_plan(int32_t dtype, int64_t T, int64_t C, int64_t F, int64_t O, const void *dout, int64_t lddout, const void *w_in, const void *w_down,
                   const void *dboth, int64_t lddb) {
    FeedPlan p = {operand(dtype, dout, T, O, lddout), operand(dtype, w_down, O, F, F)};
    p.first = product_of(dtype, T, ceil_div(F, deft::kTileCols), O, deft::kTileCols, deft::kTileRows);
    p.parts = plan_cuts(p.first);
    if (w_in) {
        p.a2 = operand(dtype, dboth, T, 2 * F, lddb);
        p.b2 = operand(dtype, w_in, 2 * F, C, C);
        p.second = product_of(dtype, T, ceil_div(C, deft::kTileCols), 2 * F, deft::kTileCols, deft::kTileRows);
        p.parts = std::max(p.parts, plan_cuts(p.second));
    }
    return p;
}
int check_feed(int32_t dtype, int64_t T, int64_t C, int64_t F, int64_t O) {
    DEF_TRY(check_rows(dtype, T, C, "C"));
    DEF_TRY(check_rows(dtype, T, F, "F"));
    DEF_TRY(check_rows(dtype, T, O, "O"));
    if (T > (int64_t)1 << 30 || F > (int64_t)1 << 29) return fail(DEF_ERR_ARG, "T must be at most 2^30 and F at most 2^29");
    return DEF_OK;
}
int check_workspace(const void *workspace, int64_t bytes, int64_t need) {
    if (need > 0 && !workspace) return fail(DEF_ERR_NULL, "workspace must not be NULL");
    if (bytes < need) return fail(DEF_ERR_ARG, "the workspace must have %lld bytes (got %lld)", (long long)need, (long long)bytes);
    return DEF_OK;
}
// Tokens as N: k is cut so that there are about two CTAs per SM.
template <typename E, bool GATED>
cudaError_t launch_tokens(int64_t T, int64_t rows, int64_t k, E *out, int64_t ldo, const CUtensorMap &map_w, const CUtensorMap &map_x, bool after, cudaStream_t stream) {
    const int64_t tiles = ceil_div(rows, deft::kTileRows), blocks = ceil_div(k, deft::kTileK);
    const int64_t splits = std::max<int64_t>(1, std::min<int64_t>({deft::kMostSplit, 2 * kUsualSms / tiles, blocks / 2}));
    const deft::TokenProduct p = {(int)T, (int)blocks, std::is_same_v<E, __nv_bfloat16>, kLongChain<E>, rows, ldo};
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)tiles, (unsigned)splits);
    cfg.blockDim = dim3(192);
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = attr[0].val.clusterDim.z = 1;
    attr[0].val.clusterDim.y = (unsigned)splits;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = after ? 2 : 1;
    auto launch = [&](auto columns) {
        constexpr int N = decltype(columns)::value, smem = deft::TokenShape<GATED, N>::smem;
        cfg.dynamicSmemBytes = smem;
        const cudaError_t err = allow_smem<deft::token_product_kernel<E, GATED, N>>(smem);
        return err == cudaSuccess ? cudaLaunchKernelEx(&cfg, deft::token_product_kernel<E, GATED, N>, p, out, map_w, map_x) : err;
    };
    return T <= 16 ? launch(std::integral_constant<int, 16>()) : launch(std::integral_constant<int, 32>());
}
// A product whose result is rounded to E.
template <bool BN, typename E, typename EPILOGUE>
int launch_rounded(const deft::Product &p, const EPILOGUE &epilogue, const CUtensorMap &map_a, const CUtensorMap &map_b, cudaStream_t stream, const char *what) {
    if constexpr (sizeof(E) == 4) {
        return launch_product<BN, 8>(p, epilogue, map_a, map_b, stream, what);
    } else {
        const int longest = p.whole > 0 ? p.blocks : (int)ceil_div(p.blocks, p.cuts);
        return longest <= kLongChain<E> ? launch_product<BN, 0>(p, epilogue, map_a, map_b, stream, what)
                                        : launch_product<BN, kLongChain<E>>(p, epilogue, map_a, map_b, stream, what);
    }
}
int token_box(int64_t T) { return T <= 16 ? 16 : 32; }
template <typename E, bool GATED>
cudaError_t launch_rows(const deft::FewTokens<E> &a, bool after, cudaStream_t stream) {
    const bool aligned = a.cols % 8 == 0 && wide(a.x, a.tokens > 1 ? a.ldx : 8, sizeof(E)) && wide(a.w, 8, sizeof(E));
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)ceil_div(a.rows, deft::kFewWarps));
    cfg.blockDim = dim3(32 * deft::kFewWarps);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = after ? 1 : 0;
    cudaError_t err = cudaSuccess;
    auto launch = [&](auto tokens) {
        constexpr int N = decltype(tokens)::value;
        err = aligned ? cudaLaunchKernelEx(&cfg, deft::few_tokens_kernel<E, N, GATED, true>, a) : cudaLaunchKernelEx(&cfg, deft::few_tokens_kernel<E, N, GATED, false>, a);
    };
    if (a.tokens <= 1) launch(std::integral_constant<int, 1>());
    else if (a.tokens <= 2) launch(std::integral_constant<int, 2>());
    else if (a.tokens <= 4) launch(std::integral_constant<int, 4>());
    else launch(std::integral_constant<int, 8>());
    return err;
}
View weights_view(const void *p, const char *name, int64_t rows, int64_t cols, int64_t es) { return rows_view(p, name, p ? 1 : 0, rows * cols, rows * cols, es, false); }

}  // namespace

extern "C" int def_feed_forward_workspace(int32_t dtype, int64_t T, int64_t C, int64_t F, int64_t O, const void *x, int64_t ldx, const void *w_in,
                                          const void *w_down, const void *h, int64_t ldh, int64_t *bytes_out) {
    if (!bytes_out) return fail(DEF_ERR_NULL, "bytes_out must not be NULL");
    DEF_TRY(check_feed(dtype, T, C, F, O));
    DEF_TRY(check_stride(x, ldx, C, T, "x"));
    DEF_TRY(check_stride(h, ldh, F, T, "h"));
    *bytes_out = feed_plan(dtype, T, C, F, O, x, ldx, w_in, w_down, h, ldh).bytes();
    return DEF_OK;
}

extern "C" int def_feed_forward(int32_t dtype, int64_t T, int64_t C, int64_t F, int64_t O, const void *x, int64_t ldx, const void *w_in, const void *w_down,
                                void *h, int64_t ldh, void *out, int64_t ldout, int8_t *gate_q, uint8_t *gate_e, int8_t *up_q, uint8_t *up_e,
                                void *workspace, int64_t workspace_bytes, void *cuda_stream) {
    int64_t need = 0;
    DEF_TRY(def_feed_forward_workspace(dtype, T, C, F, O, x, ldx, w_in, w_down, h, ldh, &need));
    if (T == 0) return DEF_OK;
    if (!x || !w_in || !h) return fail(DEF_ERR_NULL, "x, w_in and h must not be NULL");
    if (!w_down != !out) return fail(DEF_ERR_NULL, "w_down and out must both be given or both be NULL");
    DEF_TRY(check_pair(gate_q, gate_e, "gate"));
    DEF_TRY(check_pair(up_q, up_e, "up"));
    if (!gate_q != !up_q) return fail(DEF_ERR_NULL, "the checkpoints of gate and up must both be given or both be NULL");
    DEF_TRY(check_stride(out, ldout, O, T, "out"));
    DEF_TRY(check_workspace(workspace, workspace_bytes, need));
    const int es = element_size(dtype);
    const View views[] = {rows_view(x, "x", T, C, ldx, es, false), weights_view(w_in, "w_in", 2 * F, C, es), weights_view(w_down, "w_down", O, F, es),
                          rows_view(h, "h", T, F, ldh, es, true), rows_view(out, "out", T, O, ldout, es, true), q_view(gate_q, "gate_q", T, F, true),
                          e_view(gate_e, "gate_e", T, F, true), q_view(up_q, "up_q", T, F, true), e_view(up_e, "up_e", T, F, true),
                          {workspace, "workspace", need > 0 ? 1 : 0, need, need, 16, true}};
    DEF_TRY(check_views(views));
    if (const int sms = sm_count(); sms < 0) return sms;
    const cudaStream_t stream = (cudaStream_t)cuda_stream;
    FeedPlan p = feed_plan(dtype, T, C, F, O, x, ldx, w_in, w_down, h, ldh);
    const Few few = few_tokens(dtype, T, gate_q != nullptr, p);
    if (few == Few::columns) {
        const bool half = dtype == DEF_DTYPE_F16;
        CUtensorMap map_x, map_in, map_h, map_down;
        // the plan's strides: those by which it says that nothing has to be copied (a single row has any)
        DEF_TRY(operand_map(map_x, half, x, C, T, 1, p.a1.ld, token_box(T)));
        DEF_TRY(operand_map(map_in, half, w_in, C, 2 * F, 1, p.b1.ld, deft::kTileRows));
        if (out) {
            DEF_TRY(operand_map(map_h, half, h, F, T, 1, p.a2.ld, token_box(T)));
            DEF_TRY(operand_map(map_down, half, w_down, F, O, 1, p.b2.ld, deft::kTileRows));
        }
        cudaError_t err = cudaSuccess;
        by_dtype(dtype, [&](auto type) {
            using E = decltype(type);
            if constexpr (sizeof(E) == 2) {
                err = launch_tokens<E, true>(T, F, C, (E *)h, ldh, map_in, map_x, false, stream);
                if (err == cudaSuccess && out) err = launch_tokens<E, false>(T, O, F, (E *)out, ldout, map_down, map_h, true, stream);
            }
        });
        if (err == cudaSuccess) return DEF_OK;
        cudaGetLastError();
        return cuda_fail(err, "def_feed_forward");
    }
    if (few == Few::rows) {
        cudaError_t err = cudaSuccess;
        by_dtype(dtype, [&](auto type) {
            using E = decltype(type);
            err = launch_rows<E, true>({(const E *)x, (const E *)w_in, (E *)h, ldx, ldh, F, C, (int)T}, false, stream);
            if (err == cudaSuccess && out) err = launch_rows<E, false>({(const E *)h, (const E *)w_down, (E *)out, ldh, ldout, O, F, (int)T}, true, stream);
        });
        if (err == cudaSuccess) return DEF_OK;
        cudaGetLastError();
        return cuda_fail(err, "def_feed_forward");
    }
    p.put(workspace);
    // The maps first: nothing is launched where the driver refuses one.
    CUtensorMap map_x, map_in, map_h, map_down;
    DEF_TRY(operand_map(map_x, dtype, p.a1, false));
    DEF_TRY(operand_map(map_in, dtype, p.b1, false));
    if (w_down) {
        DEF_TRY(operand_map(map_h, dtype, p.a2, false));
        DEF_TRY(operand_map(map_down, dtype, p.b2, false));
    }
    DEF_TRY(fill({p.a1, p.b1, p.b2}, dtype, {x, w_in, w_down}, {ldx, C, F}, stream, "def_feed_forward (copies)"));
    int rc = DEF_OK;
    by_dtype(dtype, [&](auto type) {
        using E = decltype(type);
        const deft::StoreGated<E> store = {(E *)h, ldh, T, F, q_stride(F), e_stride(F), gate_q, up_q, gate_e, up_e, wide(h, ldh, es)};
        // What a checkpoint keeps goes by the sums' last bits.  A chain of 4 stages against 8, 777 terms: checkpoints in fp16 are
        // 0.8 against 1.2 10^-4 off (plain fp32 sums: 0.9), 4096 terms: bf16 0.8 against 1.1 (1.2) at 1169 against 1050 us.  h has the
        // same bits with and without checkpoints, so the chains are the same, too.
        rc = C <= kShortSums ? launch_product<false, 4>(p.first, store, map_x, map_in, stream, "def_feed_forward")
                             : launch_product<false, 8>(p.first, store, map_x, map_in, stream, "def_feed_forward");
    });
    if (rc != DEF_OK || !w_down) return rc;
    DEF_TRY(fill({p.a2}, dtype, {h}, {ldh}, stream, "def_feed_forward (h)"));
    by_dtype(dtype, [&](auto type) {
        using E = decltype(type);
        const deft::StoreRows<E> store = {(E *)out, ldout, T, O, wide(out, ldout, es)};
        rc = launch_rounded<false, E>(p.second, store, map_h, map_down, stream, "def_feed_forward (out)");
    });
    return rc;
}

extern "C" int def_feed_forward_backward_workspace(int32_t dtype, int64_t T, int64_t C, int64_t F, int64_t O, const void *dout, int64_t lddout, const void *w_in,
                                                   const void *w_down, const void *dboth, int64_t lddb, int64_t *bytes_out) {
    if (!bytes_out) return fail(DEF_ERR_NULL, "bytes_out must not be NULL");
    DEF_TRY(check_feed(dtype, T, C, F, O));
    DEF_TRY(check_stride(dout, lddout, O, T, "dout"));
    DEF_TRY(check_stride(dboth, lddb, 2 * F, T, "dboth"));
    *bytes_out = back_plan(dtype, T, C, F, O, dout, lddout, w_in, w_down, dboth, lddb).bytes();
    return DEF_OK;
}

extern "C" int def_feed_forward_backward(int32_t dtype, int64_t T, int64_t C, int64_t F, int64_t O, const void *dout, int64_t lddout, const void *w_in,
                                         const void *w_down, const int8_t *gate_q, const uint8_t *gate_e, const int8_t *up_q, const uint8_t *up_e,
                                         void *dboth, int64_t lddb, void *dx, int64_t lddx, void *h_out, int64_t ldh, int8_t *h_q, uint8_t *h_e,
                                         void *workspace, int64_t workspace_bytes, void *cuda_stream) {
    int64_t need = 0;
    DEF_TRY(def_feed_forward_backward_workspace(dtype, T, C, F, O, dout, lddout, w_in, w_down, dboth, lddb, &need));
    if (T == 0) return DEF_OK;
    if (!dout || !w_down || !gate_q || !gate_e || !up_q || !up_e || !dboth)
        return fail(DEF_ERR_NULL, "dout, w_down, the checkpoints of gate and up, and dboth must not be NULL");
    if (!w_in != !dx) return fail(DEF_ERR_NULL, "w_in and dx must both be given or both be NULL");
    DEF_TRY(check_pair(h_q, h_e, "h"));
    DEF_TRY(check_stride(dx, lddx, C, T, "dx"));
    DEF_TRY(check_stride(h_out, ldh, F, T, "h_out"));
    DEF_TRY(check_workspace(workspace, workspace_bytes, need));
    const int es = element_size(dtype);
    const View views[] = {rows_view(dout, "dout", T, O, lddout, es, false), weights_view(w_in, "w_in", 2 * F, C, es), weights_view(w_down, "w_down", O, F, es),
                          q_view(gate_q, "gate_q", T, F, false), e_view(gate_e, "gate_e", T, F, false), q_view(up_q, "up_q", T, F, false),
                          e_view(up_e, "up_e", T, F, false), rows_view(dboth, "dboth", T, 2 * F, lddb, es, true), rows_view(dx, "dx", T, C, lddx, es, true),
                          rows_view(h_out, "h_out", T, F, ldh, es, true), q_view(h_q, "h_q", T, F, true), e_view(h_e, "h_e", T, F, true),
                          {workspace, "workspace", need > 0 ? 1 : 0, need, need, 16, true}};
    DEF_TRY(check_views(views));
    if (const int sms = sm_count(); sms < 0) return sms;
    const cudaStream_t stream = (cudaStream_t)cuda_stream;
    FeedPlan p = back_plan(dtype, T, C, F, O, dout, lddout, w_in, w_down, dboth, lddb);
    p.put(workspace);
    CUtensorMap map_a, map_down, map_both, map_in;
    DEF_TRY(operand_map(map_a, dtype, p.a1, false));
    DEF_TRY(operand_map(map_down, dtype, p.b1, true));
    if (dx) {
        DEF_TRY(operand_map(map_both, dtype, p.a2, false));
        DEF_TRY(operand_map(map_in, dtype, p.b2, true));
    }
    DEF_TRY(fill({p.a1, p.b1, p.b2}, dtype, {dout, w_down, w_in}, {lddout, F, C}, stream, "def_feed_forward_backward (copies)"));
    int rc = DEF_OK;
    by_dtype(dtype, [&](auto type) {
        using E = decltype(type);
        E *dgate = (E *)dboth, *dup = dgate + F;
        const deft::StoreGatedBack<E> store = {dgate, dup, (E *)h_out, lddb, ldh, T, F, q_stride(F), e_stride(F), gate_q, up_q, gate_e, up_e, h_q, h_e,
                                               wide(dgate, lddb, es) && wide(dup, lddb, es), wide(h_out, ldh, es)};
        rc = launch_rounded<true, E>(p.first, store, map_a, map_down, stream, "def_feed_forward_backward");
    });
    if (rc != DEF_OK || !dx) return rc;
    DEF_TRY(fill({p.a2}, dtype, {dboth}, {lddb}, stream, "def_feed_forward_backward (dboth)"));
    by_dtype(dtype, [&](auto type) {
        using E = decltype(type);
        const deft::StoreRows<E> store = {(E *)dx, lddx, T, C, wide(dx, lddx, es)};
        rc = launch_rounded<true, E>(p.second, store, map_both, map_in, stream, "def_feed_forward_backward (dx)");
    });
    return rc;
}
