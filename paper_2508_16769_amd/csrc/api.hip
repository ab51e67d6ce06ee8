// C ABI entry points: host-side argument validation, then the kernel launchers.
#include "dr_internal.h"

#include <cstring>

namespace drc {

static thread_local char g_err[512] = "";

void set_error(const char* fmt, ...) {
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(g_err, sizeof(g_err), fmt, ap);
    va_end(ap);
}

int fail(int code, const char* fmt, ...) {
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(g_err, sizeof(g_err), fmt, ap);
    va_end(ap);
    return code;
}

int hip_fail(hipError_t e, const char* what) {
    snprintf(g_err, sizeof(g_err), "HIP error %d (%s) in %s", (int)e, hipGetErrorString(e), what);
    return DR_ERR_HIP;
}

int check_csr(const dr_csr* A, const char* name, bool need_vals) {
    DRC_REQUIRE(A != nullptr, "%s: null dr_csr", name);
    DRC_REQUIRE(A->n_rows >= 0 && A->n_cols >= 0 && A->nnz >= 0, "%s: negative dimension", name);
    DRC_REQUIRE(A->n_rows < (int64_t(1) << 31) - 1 && A->n_cols < (int64_t(1) << 31) - 1,
                "%s: more than 2^31-2 rows or columns", name);
    DRC_REQUIRE(A->nnz < (int64_t(1) << 31), "%s: nnz >= 2^31", name);
    DRC_REQUIRE(A->rowptr != nullptr, "%s: null rowptr", name);
    DRC_REQUIRE(A->nnz == 0 || A->colidx != nullptr, "%s: null colidx", name);
    DRC_REQUIRE(!need_vals || A->nnz == 0 || A->vals != nullptr, "%s: null vals", name);
    DRC_REQUIRE(A->nnz == 0 || A->n_cols > 0, "%s: edges but no columns", name);
    return DR_OK;
}

static int check_dk(int32_t D, int32_t k, const char* fn) {
    DRC_REQUIRE(D >= 1, "%s: D must be >= 1 (got %d)", fn, D);
    DRC_REQUIRE(k >= 1, "%s: k must be >= 1 (got %d)", fn, k);
    DRC_REQUIRE(k <= D, "%s: k (%d) exceeds D (%d)", fn, k, D);
    if (D > DR_MAX_D) return fail(DR_ERR_UNSUPPORTED, "%s: D = %d exceeds DR_MAX_D = %d", fn, D, DR_MAX_D);
    return DR_OK;
}

}  // namespace drc

using namespace drc;

extern "C" {

const char* dr_last_error(void) { return g_err; }

int dr_abi_version(void) { return 2; }

int dr_topk(const float* X, int64_t n, int32_t D, int32_t k, float* vals, uint16_t* idx, void* stream) {
    if (int rc = check_dk(D, k, "dr_topk")) return rc;
    DRC_REQUIRE(n >= 0, "dr_topk: negative row count");
    DRC_REQUIRE(n < (int64_t(1) << 31), "dr_topk: more than 2^31-1 rows");
    if (n == 0) return DR_OK;
    DRC_REQUIRE(X && vals && idx, "dr_topk: null pointer");
    DRC_REQUIRE(aligned(X, 4) && aligned(vals, 4) && aligned(idx, 2), "dr_topk: misaligned pointer");
    return launch_topk(X, n, D, k, vals, idx, as_stream(stream));
}

int dr_spmm_fwd(const dr_csr* A, const float* xs_vals, const uint16_t* xs_idx, int32_t D, int32_t k, float* H,
                void* stream) {
    if (int rc = check_csr(A, "dr_spmm_fwd: A", true)) return rc;
    if (int rc = check_dk(D, k, "dr_spmm_fwd")) return rc;
    if (A->n_rows == 0) return DR_OK;
    DRC_REQUIRE(H != nullptr, "dr_spmm_fwd: null H");
    DRC_REQUIRE(A->nnz == 0 || (xs_vals && xs_idx), "dr_spmm_fwd: null CBSR operand");
    DRC_REQUIRE(aligned(H, 4) && aligned(xs_vals, 4) && aligned(xs_idx, 2), "dr_spmm_fwd: misaligned pointer");
    DRC_REQUIRE(A->n_cols * (int64_t)k < (int64_t(1) << 31), "dr_spmm_fwd: N*k >= 2^31");
    return launch_spmm_fwd(A, xs_vals, xs_idx, D, k, H, as_stream(stream));
}

int dr_spmm_bwd(const dr_csr* At, const float* dH, const uint16_t* xs_idx, int32_t D, int32_t k, float* dXs,
                int accumulate, void* stream) {
    if (int rc = check_csr(At, "dr_spmm_bwd: At", true)) return rc;
    if (int rc = check_dk(D, k, "dr_spmm_bwd")) return rc;
    if (At->n_rows == 0) return DR_OK;
    DRC_REQUIRE(dXs != nullptr && xs_idx != nullptr, "dr_spmm_bwd: null dXs or xs_idx");
    DRC_REQUIRE(At->nnz == 0 || dH != nullptr, "dr_spmm_bwd: null dH");
    DRC_REQUIRE(aligned(dH, 4) && aligned(dXs, 4) && aligned(xs_idx, 2), "dr_spmm_bwd: misaligned pointer");
    DRC_REQUIRE(At->n_cols * (int64_t)D < (int64_t(1) << 32), "dr_spmm_bwd: M*D >= 2^32");
    return launch_spmm_bwd(At, dH, xs_idx, D, k, dXs, accumulate, as_stream(stream));
}

static int check_classes(const dr_degree_classes* c, int32_t D, const char* fn) {
    DRC_REQUIRE(c != nullptr, "%s: null degree classes", fn);
    DRC_REQUIRE(c->t1 >= 0 && c->t1 <= c->t2, "%s: class boundaries must satisfy 0 <= t1 <= t2 (got %d, %d)", fn, c->t1, c->t2);
    DRC_REQUIRE(c->k3 >= 1 && c->k2 >= c->k3 && c->k1 >= c->k2, "%s: widths must satisfy k1 >= k2 >= k3 >= 1 (got %d, %d, %d)", fn,
                c->k1, c->k2, c->k3);
    if (int rc = check_dk(D, c->k1, fn)) return rc;
    if (c->k1 > 64) return fail(DR_ERR_UNSUPPORTED, "%s: k1 = %d exceeds 64", fn, c->k1);
    return DR_OK;
}

int dr_topk_ranked(const float* X, int64_t n, int32_t D, int32_t k, float* vals, uint16_t* idx, void* stream) {
    if (int rc = check_dk(D, k, "dr_topk_ranked")) return rc;
    DRC_REQUIRE(n >= 0 && n < (int64_t(1) << 31), "dr_topk_ranked: n out of range");
    if (n == 0) return DR_OK;
    DRC_REQUIRE(X && vals && idx, "dr_topk_ranked: null pointer");
    DRC_REQUIRE(aligned(X, 4) && aligned(vals, 4) && aligned(idx, 2), "dr_topk_ranked: misaligned pointer");
    DRC_REQUIRE(n * (int64_t)D < (int64_t(1) << 33) && n * (int64_t)k < (int64_t(1) << 31), "dr_topk_ranked: n*D or n*k too large");
    return launch_topk_ranked(X, n, D, k, vals, idx, as_stream(stream));
}

int dr_spmm_fwd_adaptive(const dr_csr* A, const float* xr_vals, const uint16_t* xr_idx, int32_t D,
                         const dr_degree_classes* cls, float* H, void* stream) {
    if (int rc = check_csr(A, "dr_spmm_fwd_adaptive: A", true)) return rc;
    if (int rc = check_classes(cls, D, "dr_spmm_fwd_adaptive")) return rc;
    if (A->n_rows == 0) return DR_OK;
    DRC_REQUIRE(H != nullptr, "dr_spmm_fwd_adaptive: null H");
    DRC_REQUIRE(A->nnz == 0 || (xr_vals && xr_idx), "dr_spmm_fwd_adaptive: null CBSR operand");
    DRC_REQUIRE(aligned(H, 4) && aligned(xr_vals, 4) && aligned(xr_idx, 2), "dr_spmm_fwd_adaptive: misaligned pointer");
    DRC_REQUIRE(A->n_cols * (int64_t)cls->k1 < (int64_t(1) << 31), "dr_spmm_fwd_adaptive: N*k1 >= 2^31");
    return launch_spmm_fwd_adaptive(A, xr_vals, xr_idx, D, cls, H, as_stream(stream));
}

int dr_degree_edge_classes(const dr_csr* At, const int32_t* A_rowptr, const dr_degree_classes* cls, uint8_t* edge_class,
                           void* stream) {
    if (int rc = check_csr(At, "dr_degree_edge_classes: At", false)) return rc;
    DRC_REQUIRE(cls != nullptr && cls->t1 >= 0 && cls->t1 <= cls->t2, "dr_degree_edge_classes: class boundaries must satisfy 0 <= t1 <= t2");
    if (At->nnz == 0) return DR_OK;
    DRC_REQUIRE(A_rowptr != nullptr && edge_class != nullptr, "dr_degree_edge_classes: null pointer");
    return launch_edge_classes(At, A_rowptr, cls, edge_class, as_stream(stream));
}

int dr_spmm_bwd_adaptive(const dr_csr* At, const uint8_t* edge_class, const float* dH, const uint16_t* xr_idx, int32_t D,
                         const dr_degree_classes* cls, float* dXr, int accumulate, void* stream) {
    if (int rc = check_csr(At, "dr_spmm_bwd_adaptive: At", true)) return rc;
    if (int rc = check_classes(cls, D, "dr_spmm_bwd_adaptive")) return rc;
    if (At->n_rows == 0) return DR_OK;
    DRC_REQUIRE(dXr != nullptr && xr_idx != nullptr, "dr_spmm_bwd_adaptive: null dXr or xr_idx");
    DRC_REQUIRE(At->nnz == 0 || (dH != nullptr && edge_class != nullptr), "dr_spmm_bwd_adaptive: null dH or edge_class");
    DRC_REQUIRE(aligned(dH, 4) && aligned(dXr, 4) && aligned(xr_idx, 2), "dr_spmm_bwd_adaptive: misaligned pointer");
    DRC_REQUIRE(At->n_cols < (int64_t(1) << 30), "dr_spmm_bwd_adaptive: 2^30 or more destinations");
    DRC_REQUIRE(At->n_cols * (int64_t)D < (int64_t(1) << 32), "dr_spmm_bwd_adaptive: M*D >= 2^32");
    return launch_spmm_bwd_adaptive(At, edge_class, dH, xr_idx, D, cls, dXr, accumulate, as_stream(stream));
}

static int check_rows(int64_t n, int32_t D, const char* fn) {
    DRC_REQUIRE(n >= 0, "%s: negative row count", fn);
    DRC_REQUIRE(n < (int64_t(1) << 31), "%s: more than 2^31-1 rows", fn);
    DRC_REQUIRE(D >= 1, "%s: D must be >= 1 (got %d)", fn, D);
    if (D > DR_MAX_D) return fail(DR_ERR_UNSUPPORTED, "%s: D = %d exceeds DR_MAX_D = %d", fn, D, DR_MAX_D);
    return DR_OK;
}

static int check_act8(const dr_act8* c, const char* fn, const char* name) {
    DRC_REQUIRE(c != nullptr && c->q != nullptr && c->scale != nullptr, "%s: null checkpoint (%s)", fn, name);
    DRC_REQUIRE(aligned(c->scale, 8), "%s: scales of checkpoint %s must be 8-byte aligned", fn, name);
    return DR_OK;
}

static int check_workspace(const void* ws, size_t have, size_t need, const char* fn) {
    DRC_REQUIRE(ws != nullptr, "%s: null workspace", fn);
    DRC_REQUIRE(aligned(ws, 256), "%s: workspace must be 256-byte aligned", fn);
    if (have < need) return fail(DR_ERR_WORKSPACE, "%s: workspace has %zu bytes, needs %zu", fn, have, need);
    return DR_OK;
}

size_t dr_act8_scale_bytes(int64_t n, int32_t D) {
    if (n < 0 || D < 1) return 0;
    return (size_t)((n + 7) / 8) * act_groups(D) * 8;
}

int dr_act8_pack(const float* X, int64_t n, int32_t D, const dr_act8* out, void* stream) {
    DRC_TRY(check_rows(n, D, "dr_act8_pack"));
    if (n == 0) return DR_OK;
    DRC_REQUIRE(X != nullptr, "dr_act8_pack: null pointer");
    DRC_REQUIRE(aligned(X, 4), "dr_act8_pack: misaligned pointer");
    DRC_TRY(check_act8(out, "dr_act8_pack", "out"));
    return launch_act8_pack(X, n, D, *out, as_stream(stream));
}

int dr_act8_unpack(const dr_act8* in, int64_t n, int32_t D, float* X, void* stream) {
    DRC_TRY(check_rows(n, D, "dr_act8_unpack"));
    if (n == 0) return DR_OK;
    DRC_REQUIRE(X != nullptr, "dr_act8_unpack: null pointer");
    DRC_REQUIRE(aligned(X, 4), "dr_act8_unpack: misaligned pointer");
    DRC_TRY(check_act8(in, "dr_act8_unpack", "in"));
    return launch_act8_unpack(*in, n, D, X, as_stream(stream));
}

size_t dr_act8_wgrad_workspace_bytes(int64_t n, int32_t D, int32_t F) {
    if (n < 0 || D < 1 || F < 1) return 0;
    return act8_wgrad_workspace(n, D, F);
}

int dr_act8_wgrad(const dr_act8* A, int64_t n, int32_t D, const float* dZ, int32_t F, float* dW, int accumulate, void* workspace,
                  size_t workspace_bytes, void* stream) {
    DRC_TRY(check_rows(n, D, "dr_act8_wgrad"));
    DRC_REQUIRE(F >= 1, "dr_act8_wgrad: F must be >= 1 (got %d)", F);
    if (F > DR_MAX_D) return fail(DR_ERR_UNSUPPORTED, "dr_act8_wgrad: F = %d exceeds DR_MAX_D = %d", F, DR_MAX_D);
    DRC_REQUIRE(dW != nullptr, "dr_act8_wgrad: null dW");
    if (n > 0) {
        DRC_TRY(check_act8(A, "dr_act8_wgrad", "A"));
        DRC_REQUIRE(dZ != nullptr, "dr_act8_wgrad: null dZ");
    }
    DRC_REQUIRE(aligned(dZ, 4) && aligned(dW, 4), "dr_act8_wgrad: misaligned pointer");
    DRC_TRY(check_workspace(workspace, workspace_bytes, act8_wgrad_workspace(n, D, F), "dr_act8_wgrad"));
    return launch_act8_wgrad(n > 0 ? *A : dr_act8{}, n, D, dZ, F, dW, accumulate != 0, workspace, as_stream(stream));
}

static int check_block(const dr_block* b, int32_t D, const char* fn) {
    DRC_REQUIRE(b != nullptr, "%s: null block", fn);
    DRC_REQUIRE(b->norm == DR_ROWNORM_RMS || b->norm == DR_ROWNORM_LAYER, "%s: unknown norm %d", fn, b->norm);
    DRC_REQUIRE(b->eps >= 1.17549435e-38f && b->eps < 1e30f, "%s: eps must be positive and a normal number", fn);
    DRC_REQUIRE(b->gate_cols == 0 || b->gate_cols == 1 || b->gate_cols == D, "%s: gate_cols = %d is not 0, 1 or D = %d", fn, b->gate_cols, D);
    DRC_REQUIRE(aligned(b->w_after, 4) && aligned(b->b_after, 4) && aligned(b->scale, 4) && aligned(b->w_before, 4) && aligned(b->b_before, 4),
                "%s: misaligned parameter vector", fn);
    return DR_OK;
}

int dr_block_fwd(const dr_block* block, int64_t n, int32_t D, const float* X, const float* Y, const float* G, float* X_out, float* N,
                 const dr_block_saved* saved, void* stream) {
    DRC_TRY(check_rows(n, D, "dr_block_fwd"));
    DRC_TRY(check_block(block, D, "dr_block_fwd"));
    if (n == 0) return DR_OK;
    const dr_block_saved S = saved ? *saved : dr_block_saved{};
    DRC_REQUIRE(X != nullptr, "dr_block_fwd: null X");
    DRC_REQUIRE(Y != nullptr || N != nullptr, "dr_block_fwd: neither Y nor N");
    DRC_REQUIRE((Y != nullptr) == (X_out != nullptr), "dr_block_fwd: Y and X_out must both be given or both be NULL");
    DRC_REQUIRE((G != nullptr) == (block->gate_cols != 0), "dr_block_fwd: G and gate_cols = %d do not match", block->gate_cols);
    DRC_REQUIRE(Y != nullptr || (G == nullptr && S.y.q == nullptr && S.g.q == nullptr && S.stats_after == nullptr),
                "dr_block_fwd: a gate, statistics or checkpoints of a layer's output without Y");
    DRC_REQUIRE(N != nullptr || S.stats_before == nullptr, "dr_block_fwd: statistics of a norm in front without N");
    DRC_REQUIRE(S.g.q == nullptr || block->gate_cols == D, "dr_block_fwd: a checkpoint of G needs gate_cols = D");
    DRC_REQUIRE(X_out == nullptr || X_out != N, "dr_block_fwd: X_out and N are the same");
    DRC_REQUIRE(G == nullptr || block->gate_cols == D || (G != X_out && G != N), "dr_block_fwd: a gate of one column is no room for X_out or N");
    DRC_REQUIRE(aligned(X, 4) && aligned(Y, 4) && aligned(G, 4) && aligned(X_out, 4) && aligned(N, 4) && aligned(S.stats_after, 4) &&
                    aligned(S.stats_before, 4),
                "dr_block_fwd: misaligned pointer");
    if (S.x.q) DRC_TRY(check_act8(&S.x, "dr_block_fwd", "x"));
    if (S.y.q) DRC_TRY(check_act8(&S.y, "dr_block_fwd", "y"));
    if (S.g.q) DRC_TRY(check_act8(&S.g, "dr_block_fwd", "g"));
    return launch_block_fwd(BlockFwd{*block, n, D, X, Y, G, X_out, N, S}, as_stream(stream));
}

size_t dr_block_bwd_workspace_bytes(int64_t n, int32_t D) {
    if (n < 0 || D < 1) return 0;
    return block_bwd_workspace(n, D);
}

int dr_block_bwd(const dr_block* block, int64_t n, int32_t D, const float* dX_out, const float* dN, const float* X_out, const float* Y,
                 const float* G, const dr_block_saved* saved, const dr_block_grads* grads, void* workspace, size_t workspace_bytes,
                 void* stream) {
    DRC_TRY(check_rows(n, D, "dr_block_bwd"));
    DRC_TRY(check_block(block, D, "dr_block_bwd"));
    DRC_REQUIRE(grads != nullptr, "dr_block_bwd: null grads");
    const dr_block_saved S = saved ? *saved : dr_block_saved{};
    const dr_block_grads& g = *grads;
    const bool after = Y != nullptr || S.y.q != nullptr, gated = G != nullptr || S.g.q != nullptr;
    if (n > 0) {
        DRC_REQUIRE(dX_out != nullptr || dN != nullptr, "dr_block_bwd: neither dX_out nor dN");
        DRC_REQUIRE(Y == nullptr || S.y.q == nullptr, "dr_block_bwd: Y and its checkpoint are both given");
        DRC_REQUIRE(G == nullptr || S.g.q == nullptr, "dr_block_bwd: G and its checkpoint are both given");
        DRC_REQUIRE(X_out == nullptr || S.x.q == nullptr, "dr_block_bwd: X_out and its checkpoint are both given");
        DRC_REQUIRE(dN == nullptr || X_out != nullptr || S.x.q != nullptr, "dr_block_bwd: dN without X_out or its checkpoint");
        DRC_REQUIRE(dN == nullptr || S.stats_before != nullptr, "dr_block_bwd: dN without saved.stats_before");
        DRC_REQUIRE(!after || S.stats_after != nullptr, "dr_block_bwd: Y without saved.stats_after");
        DRC_REQUIRE(gated == (block->gate_cols != 0) && (after || !gated), "dr_block_bwd: G and gate_cols = %d do not match", block->gate_cols);
        DRC_REQUIRE(S.g.q == nullptr || block->gate_cols == D, "dr_block_bwd: a checkpoint of G needs gate_cols = D");
        DRC_REQUIRE(after || (!g.dY && !g.dG && !g.dw_after && !g.db_after && !g.dscale), "dr_block_bwd: gradients behind the layer without Y");
        DRC_REQUIRE(gated || !g.dG, "dr_block_bwd: dG without G");
        const bool row_gate = gated && block->gate_cols != D;
        DRC_REQUIRE(!row_gate || (G != g.dX && G != g.dY), "dr_block_bwd: a gate of one column is no room for dX or dY");
        DRC_REQUIRE(!row_gate || !g.dG || (g.dG != dX_out && g.dG != dN && g.dG != X_out && g.dG != Y),
                    "dr_block_bwd: a dG of one column takes no other tensor's place than G's");
        if (S.x.q) DRC_TRY(check_act8(&S.x, "dr_block_bwd", "x"));
        if (S.y.q) DRC_TRY(check_act8(&S.y, "dr_block_bwd", "y"));
        if (S.g.q) DRC_TRY(check_act8(&S.g, "dr_block_bwd", "g"));
    }
    DRC_REQUIRE((g.dX == nullptr || (g.dX != g.dY && g.dX != g.dG)) && (g.dY == nullptr || g.dY != g.dG),
                "dr_block_bwd: two of dX, dY and dG are the same");
    DRC_REQUIRE(aligned(dX_out, 4) && aligned(dN, 4) && aligned(X_out, 4) && aligned(Y, 4) && aligned(G, 4) && aligned(S.stats_after, 4) &&
                    aligned(S.stats_before, 4) && aligned(g.dX, 4) && aligned(g.dY, 4) && aligned(g.dG, 4) && aligned(g.dw_after, 4) &&
                    aligned(g.db_after, 4) && aligned(g.dscale, 4) && aligned(g.dw_before, 4) && aligned(g.db_before, 4),
                "dr_block_bwd: misaligned pointer");
    DRC_TRY(check_workspace(workspace, workspace_bytes, block_bwd_workspace(n, D), "dr_block_bwd"));
    return launch_block_bwd(BlockBwd{*block, n, D, dX_out, dN, X_out, Y, G, S, g, nullptr, 0}, workspace, as_stream(stream));
}

size_t dr_csr_transpose_workspace_bytes(int64_t n_rows, int64_t n_cols, int64_t nnz) {
    (void)n_rows;
    if (n_cols < 0 || nnz < 0) return 0;
    return csr_transpose_workspace(n_cols, nnz);
}

int dr_csr_transpose(const dr_csr* A, int32_t* t_rowptr, int32_t* t_colidx, float* t_vals, void* workspace,
                     size_t workspace_bytes, void* stream) {
    if (int rc = check_csr(A, "dr_csr_transpose: A", false)) return rc;
    DRC_REQUIRE(t_rowptr != nullptr, "dr_csr_transpose: null t_rowptr");
    DRC_REQUIRE(A->nnz == 0 || t_colidx != nullptr, "dr_csr_transpose: null t_colidx");
    DRC_REQUIRE((A->vals == nullptr) == (t_vals == nullptr) || A->nnz == 0,
                "dr_csr_transpose: vals and t_vals must both be given or both be NULL");
    size_t need = dr_csr_transpose_workspace_bytes(A->n_rows, A->n_cols, A->nnz);
    DRC_REQUIRE(workspace != nullptr, "dr_csr_transpose: null workspace");
    DRC_REQUIRE(aligned(workspace, 256), "dr_csr_transpose: workspace must be 256-byte aligned");
    if (workspace_bytes < need)
        return fail(DR_ERR_WORKSPACE, "dr_csr_transpose: workspace has %zu bytes, needs %zu", workspace_bytes, need);
    const TransposeJob job{A, t_rowptr, t_colidx, t_vals, workspace};
    return launch_csr_transposes(&job, 1, as_stream(stream));
}

size_t dr_csr_normalize_workspace_bytes(int mode, int64_t n_rows, int64_t n_cols, int64_t nnz) {
    (void)n_rows;
    if (n_cols < 0 || nnz < 0) return 0;
    return csr_normalize_workspace(mode, n_cols, nnz);
}

int dr_csr_normalize(int mode, int64_t n_rows, int64_t n_cols, int64_t nnz, const int32_t* rowptr,
                     const int32_t* colidx, float* vals_out, void* workspace, size_t workspace_bytes,
                     void* stream) {
    DRC_REQUIRE(mode == DR_NORM_MEAN || mode == DR_NORM_SYM, "dr_csr_normalize: unknown mode %d", mode);
    dr_csr A{n_rows, n_cols, nnz, rowptr, colidx, nullptr};
    if (int rc = check_csr(&A, "dr_csr_normalize", false)) return rc;
    if (nnz == 0) return DR_OK;
    DRC_REQUIRE(vals_out != nullptr, "dr_csr_normalize: null vals_out");
    size_t need = dr_csr_normalize_workspace_bytes(mode, n_rows, n_cols, nnz);
    if (need > 0) {
        DRC_REQUIRE(workspace != nullptr, "dr_csr_normalize: null workspace");
        DRC_REQUIRE(aligned(workspace, 256), "dr_csr_normalize: workspace must be 256-byte aligned");
        if (workspace_bytes < need)
            return fail(DR_ERR_WORKSPACE, "dr_csr_normalize: workspace has %zu bytes, needs %zu", workspace_bytes,
                        need);
    }
    return launch_csr_normalize(mode, n_rows, n_cols, nnz, rowptr, colidx, vals_out, workspace, as_stream(stream));
}

int dr_csr_normalize_noalloc(int mode, int64_t n_rows, int64_t n_cols, int64_t nnz, const int32_t* rowptr,
                             const int32_t* colidx, float* vals_out, void* stream) {
    DRC_REQUIRE(mode == DR_NORM_MEAN || mode == DR_NORM_SYM, "dr_csr_normalize_noalloc: unknown mode %d", mode);
    dr_csr A{n_rows, n_cols, nnz, rowptr, colidx, nullptr};
    if (int rc = check_csr(&A, "dr_csr_normalize_noalloc", false)) return rc;
    if (nnz == 0) return DR_OK;
    DRC_REQUIRE(vals_out != nullptr, "dr_csr_normalize_noalloc: null vals_out");
    if (mode == DR_NORM_SYM && n_cols > DR_NOALLOC_MAX_COLS)
        return fail(DR_ERR_UNSUPPORTED, "dr_csr_normalize_noalloc: n_cols = %lld exceeds DR_NOALLOC_MAX_COLS = %d",
                    (long long)n_cols, DR_NOALLOC_MAX_COLS);
    return launch_csr_normalize_noalloc(mode, n_rows, n_cols, nnz, rowptr, colidx, vals_out, as_stream(stream));
}

}  // extern "C"
