// C boundary of the orthogonalised update (see include/def_train.h).
#include <algorithm>
#include <cmath>

#include "def_orthogonal_kernels.cuh"
#include "def_product_launch.cuh"

namespace {

constexpr int64_t kMostSide = (int64_t)1 << 16, kMostMatrices = (int64_t)1 << 16;

// Two buffers of X and one of A and B each, as two pieces of rows padded to 32 elements; the parts of cut tiles in what the
// documented size leaves beside them.
struct OrthogonalPlan {
    int64_t m, n, ldm, ldn, parts, sums, x, square;        // bytes of: parts, sums, one buffer of X, one of A
    deft::Product gram, polynomial, update;
    int64_t bytes() const { return parts + sums + 2 * x + 2 * square; }
};
deft::Product piece_product(int64_t batch, int64_t m, int64_t n, int64_t k, bool triangle) {
    deft::Product p = {};
    p.tiles_m = (int)ceil_div(m, 2 * deft::kTileRows);
    p.tiles_n = (int)ceil_div(n, deft::kTileCols);
    p.batch = (int)batch;
    p.blocks = (int)ceil_div(k, deft::kTileK);
    p.pairs = 3;                                           // lo hi, hi lo, hi hi
    p.planes_a = p.planes_b = 2;
    p.order_a = 0x001u;
    p.order_b = 0x010u;
    p.triangle = triangle;
    p.step_n = deft::kTileCols;
    p.second = deft::kTileRows;
    return p;
}
OrthogonalPlan orthogonal_plan(int64_t batch, int64_t rows, int64_t cols) {
    OrthogonalPlan p = {};
    p.m = std::min(rows, cols);
    p.n = std::max(rows, cols);
    p.ldm = ceil_div(p.m, 32) * 32;
    p.ldn = ceil_div(p.n, 32) * 32;
    p.sums = batch * deft::kNormParts64 * 8;
    p.x = batch * 2 * p.m * p.ldn * 2;
    p.square = batch * 2 * p.m * p.ldm * 2;
    p.gram = piece_product(batch, p.m, p.m, p.n, true);
    p.polynomial = piece_product(batch, p.m, p.m, p.m, true);
    p.update = piece_product(batch, p.m, p.n, p.m, false);
    const int64_t most = std::min(kMostPartBytes, batch * (16 * (p.m + 8) * (p.n + p.m + 16) + 8192) - p.bytes());
    for (deft::Product *q : {&p.gram, &p.polynomial, &p.update}) p.parts = std::max(p.parts, plan_cuts(*q, most, 2));
    return p;
}
// Stages in a chain of the matrix unit.  What the chains lose against fp32 sums decides: relative error of five steps with 4, 2
// and 1 of them, beside that of the same steps in plain fp32, 10^-6:
//     128 x 128  2.3, 2.3, 1.6 (1.4)     512 x 512  3.6, 2.5, 1.6 (2.3)     1024 x 1024  4.0, 2.2, 1.4 (2.7)     1500 x 3000  3.5, 2.0, 1.3 (2.7)
//     2048 x 4096  3.4, 1.9, 1.3 (2.9)   100 x 8000  3.1, 3.4, 2.2 (1.3)    4096 x 10240  3.3, 1.9, 1.4 (3.8)
// 4096 x 10240 takes 7.9, 9.2 and 10.3 ms (calls back to back, one set of inputs), 512 x 512 260, 262 and 270 us (before joins read
// several parts at once: 209 with 2 stages now).
int piece_chain(int64_t m) { return m < 384 ? 1 : m < 1280 ? 2 : 4; }
template <bool BN, typename EPILOGUE>
int launch_pieces(int64_t m, const deft::Product &p, const EPILOGUE &epilogue, const CUtensorMap &map_a, const CUtensorMap &map_b, cudaStream_t stream, const char *what) {
    const int chain = piece_chain(m);
    return chain == 1   ? launch_product<BN, 1>(p, epilogue, map_a, map_b, stream, what)
           : chain == 2 ? launch_product<BN, 2>(p, epilogue, map_a, map_b, stream, what)
                        : launch_product<BN, 4>(p, epilogue, map_a, map_b, stream, what);
}
int check_matrices(int32_t dtype, int64_t batch, int64_t rows, int64_t cols) {
    if (!element_size(dtype)) return fail(DEF_ERR_ARG, "dtype must be one of DEF_DTYPE_F32, _BF16, _F16 (got %d)", dtype);
    if (batch < 0 || batch > kMostMatrices) return fail(DEF_ERR_ARG, "batch must be in [0, 2^16] (got %lld)", (long long)batch);
    if (rows < 1 || cols < 1 || rows > kMostSide || cols > kMostSide)
        return fail(DEF_ERR_ARG, "rows and cols must be in [1, 2^16] (got %lld, %lld)", (long long)rows, (long long)cols);
    return DEF_OK;
}
// Whether the steps keep the singular values of X below 4 and those of B below 16, whatever matrix they start from (norm 1 at
// most): then the entries are, too, which is what the pieces have room for.
bool polynomials_stay(const float *coeffs, int steps) {
    double top = 1.;                                       // singular values of X are in [0, top]
    for (int i = 0; i < steps; ++i, coeffs += 3) {
        const double a = coeffs[0], b = coeffs[1], c = coeffs[2], most = top * top;
        const auto factor = [&](double t) { return a + t * (b + t * c); };             // of the singular value whose square is t
        double largest = 0., next = 0.;
        const auto look = [&](double t) {
            if (!(t >= 0.)) t = 0.;
            if (t > most) t = most;
            largest = std::max(largest, std::abs(factor(t)));
            next = std::max(next, std::sqrt(t) * std::abs(factor(t)));
        };
        look(0.);
        look(most);
        if (c != 0.) {
            look(-b / (2. * c));                           // extremes of the factor, and of s times it
            const double root = 9. * b * b - 20. * a * c;
            if (root >= 0.) {
                look((-3. * b + std::sqrt(root)) / (10. * c));
                look((-3. * b - std::sqrt(root)) / (10. * c));
            }
        } else if (b != 0.) {
            look(-a / (3. * b));
        }
        top = next * 1.00001;                              // what 22 bits may add
        if (!(largest * 1.001 < 16.) || !(top < 4.)) return false;
    }
    return true;
}
// Matrices as a view: `batch` runs that each span a whole matrix.
View matrices_view(const void *p, const char *name, int64_t batch, int64_t rows, int64_t cols, int64_t ld, int64_t stride, int64_t es, bool written) {
    const int64_t width = ((rows - 1) * ld + cols) * es;
    return {p, name, batch, width, batch > 1 ? stride * es : width, (unsigned)es, written};
}
// The same as rows of one pitch, where the distance between matrices allows it: columns of one buffer beside each other are apart.
View matrix_rows_view(const void *p, const char *name, int64_t batch, int64_t rows, int64_t cols, int64_t ld, int64_t stride, int64_t es, bool written) {
    if (batch > 1 && stride % ld != 0) return matrices_view(p, name, batch, rows, cols, ld, stride, es, written);
    return rows_view(p, name, batch > 1 ? (batch - 1) * (stride / ld) + rows : rows, cols, ld, es, written);
}
int check_layout(const char *name, int64_t batch, int64_t rows, int64_t cols, int64_t ld, int64_t stride) {
    if (ld < cols) return fail(DEF_ERR_ARG, "the row stride of %s must be at least its width (got %lld)", name, (long long)ld);
    if (ld > ((int64_t)1 << 40)) return fail(DEF_ERR_ARG, "the rows of %s reach too far", name);
    if (batch > 1 && stride < (rows - 1) * ld + cols) return fail(DEF_ERR_ARG, "the matrices of %s overlap (stride %lld)", name, (long long)stride);
    if (batch > 1 && stride > ((int64_t)1 << 60) / batch / 4) return fail(DEF_ERR_ARG, "the matrices of %s reach too far", name);
    return DEF_OK;
}

}  // namespace

extern "C" int def_orthogonalize_workspace(int64_t batch, int64_t rows, int64_t cols, int64_t *bytes_out) {
    if (!bytes_out) return fail(DEF_ERR_NULL, "bytes_out must not be NULL");
    DEF_TRY(check_matrices(DEF_DTYPE_F32, batch, rows, cols));
    *bytes_out = batch ? orthogonal_plan(batch, rows, cols).bytes() : 0;
    return DEF_OK;
}

extern "C" int def_orthogonalize(int32_t dtype, int64_t batch, int64_t rows, int64_t cols, const void *x, int64_t ldx, int64_t stride_x, void *out,
                                 int64_t ldo, int64_t stride_o, const float *coeffs, int32_t steps, float eps, float scale, void *workspace,
                                 int64_t workspace_bytes, void *cuda_stream) {
    DEF_TRY(check_matrices(dtype, batch, rows, cols));
    if (steps < 1 || steps > DEF_ORTHOGONALIZE_MAX_STEPS) return fail(DEF_ERR_ARG, "steps must be in [1, %d] (got %d)", DEF_ORTHOGONALIZE_MAX_STEPS, steps);
    if (!coeffs) return fail(DEF_ERR_NULL, "coeffs must not be NULL");
    for (int i = 0; i < 3 * steps; ++i)
        if (!(std::abs(coeffs[i]) <= 8.f) && !(std::abs(coeffs[i]) <= 64.f && polynomials_stay(coeffs, steps)))
            return fail(DEF_ERR_ARG, "coefficients must be within 8 of 0, or within 64 where singular values stay below 4 (got %g)", (double)coeffs[i]);
    if (!(eps >= 0.f) || !(eps <= 1e30f)) return fail(DEF_ERR_ARG, "eps must be a finite number that is not negative");
    if (!(scale >= -1e30f && scale <= 1e30f)) return fail(DEF_ERR_ARG, "scale must be a finite number");
    if (batch == 0) return DEF_OK;
    if (!x || !out) return fail(DEF_ERR_NULL, "x and out must not be NULL");
    DEF_TRY(check_layout("x", batch, rows, cols, ldx, stride_x));
    DEF_TRY(check_layout("out", batch, rows, cols, ldo, stride_o));
    OrthogonalPlan p = orthogonal_plan(batch, rows, cols);
    if (!workspace) return fail(DEF_ERR_NULL, "workspace must not be NULL");
    if (workspace_bytes < p.bytes()) return fail(DEF_ERR_ARG, "the workspace must have %lld bytes (got %lld)", (long long)p.bytes(), (long long)workspace_bytes);
    const int es = element_size(dtype);
    const bool same = x == out && (rows == 1 || ldx == ldo) && (batch == 1 || stride_x == stride_o);
    const View in_view = matrices_view(x, "x", batch, rows, cols, ldx, stride_x, es, false), out_view = matrices_view(out, "out", batch, rows, cols, ldo, stride_o, es, true),
               work_view = {workspace, "workspace", 1, p.bytes(), p.bytes(), 16, true};
    const View first[] = {in_view, work_view}, second[] = {out_view, work_view};
    DEF_TRY(check_views(first));
    DEF_TRY(check_views(second));
    if (!same && share_bytes(in_view, out_view) &&
        share_bytes(matrix_rows_view(x, "x", batch, rows, cols, ldx, stride_x, es, false), matrix_rows_view(out, "out", batch, rows, cols, ldo, stride_o, es, true)))
        return fail(DEF_ERR_ALIAS, "x and out overlap");
    if (const int sms = sm_count(); sms < 0) return sms;
    const cudaStream_t stream = (cudaStream_t)cuda_stream;
    char *at = (char *)workspace;
    p.gram.parts = p.polynomial.parts = p.update.parts = (float *)at;
    at += p.parts;
    double *sums = (double *)at;
    at += p.sums;
    __half *xs[2] = {(__half *)at, (__half *)(at + p.x)};
    at += 2 * p.x;
    __half *gram = (__half *)at, *poly = (__half *)(at + p.square);
    const int64_t plane_x = p.m * p.ldn, plane_a = p.m * p.ldm;
    // The maps first: nothing is launched where the driver refuses one.
    CUtensorMap x_rows[2], x_cols[2], gram_rows, poly_rows;
    for (int i = 0; i < 2; ++i) {
        DEF_TRY(operand_map(x_rows[i], true, xs[i], p.n, p.m, 2 * batch, p.ldn, deft::kTileRows));
        DEF_TRY(operand_map(x_cols[i], true, xs[i], p.n, p.m, 2 * batch, p.ldn, deft::kTileK));
    }
    DEF_TRY(operand_map(gram_rows, true, gram, p.m, p.m, 2 * batch, p.ldm, deft::kTileRows));
    DEF_TRY(operand_map(poly_rows, true, poly, p.m, p.m, 2 * batch, p.ldm, deft::kTileRows));

    const bool tall = rows > cols;
    const deft::Matrices in = {x, ldx, stride_x, rows, cols, batch};
    const int parts = (int)std::min<int64_t>(deft::kNormParts64, ceil_div(rows, 8));
    by_dtype(dtype, [&](auto type) {
        using E = decltype(type);
        deft::square_sum_kernel<E><<<dim3((unsigned)parts, (unsigned)std::min<int64_t>(batch, 65535)), 256, 0, stream>>>(in, sums);
        const dim3 grid((unsigned)ceil_div(tall ? cols : p.ldn, deft::kPackTile), (unsigned)ceil_div(tall ? p.ldn : rows, deft::kPackTile), (unsigned)std::min<int64_t>(batch, 65535));
        if (tall) deft::pack_pieces_kernel<E, true><<<grid, 256, 0, stream>>>(in, sums, parts, eps, xs[0], p.ldn, plane_x);
        else deft::pack_pieces_kernel<E, false><<<grid, 256, 0, stream>>>(in, sums, parts, eps, xs[0], p.ldn, plane_x);
    });
    DEF_TRY(launched("def_orthogonalize (pieces)"));
    const float down = 1.f / deft::kPieceScale;
    for (int i = 0; i < steps; ++i) {
        const float *k = coeffs + 3 * i;
        const int from = i & 1, to = from ^ 1;
        const deft::StoreSymmetric first = {gram, nullptr, p.ldm, plane_a, p.m, down, 0.f, 0.f};
        const deft::StoreSymmetric second = {poly, gram, p.ldm, plane_a, p.m, k[2] * down, k[1], k[0] * deft::kPieceScale};
        DEF_TRY((launch_pieces<false>(p.m, p.gram, first, x_rows[from], x_rows[from], stream, "def_orthogonalize (gram)")));
        DEF_TRY((launch_pieces<false>(p.m, p.polynomial, second, gram_rows, gram_rows, stream, "def_orthogonalize (polynomial)")));
        if (i + 1 < steps) {
            const deft::StorePieces third = {xs[to], p.ldn, plane_x, p.m, p.n, down};
            DEF_TRY((launch_pieces<true>(p.m, p.update, third, poly_rows, x_cols[from], stream, "def_orthogonalize (update)")));
        } else {
            int rc = DEF_OK;
            by_dtype(dtype, [&](auto type) {
                using E = decltype(type);
                bool aligned = wide(out, ldo, es) && (batch == 1 || stride_o * es % 16 == 0);
                const deft::StoreUpdate<E> last = {(E *)out, ldo, stride_o, p.m, p.n, scale * down * down, tall, aligned};
                rc = launch_pieces<true>(p.m, p.update, last, poly_rows, x_cols[from], stream, "def_orthogonalize (out)");
            });
            if (rc != DEF_OK) return rc;
        }
    }
    return DEF_OK;
}
