// C ABI of the operators around a linear layer (see include/mxfp4.h): argument checks on the host, then launches.
#include <hip/hip_runtime.h>
#include <math.h>

#include "../../include/mxfp4.h"
#include "layer_ops.h"
#include "mxfp4_internal.h"

namespace {

using namespace mxfp4;

bool known_type(int dtype) { return dtype == MXFP4_OUT_BF16 || dtype == MXFP4_OUT_FP32; }
size_t element(int dtype) { return dtype == MXFP4_OUT_FP32 ? 4 : 2; }
bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
bool flag(int v) { return v == 0 || v == 1; }
constexpr int64_t MOST = int64_t(1) << 40;      // rows, tokens, strides
constexpr int64_t FURTHEST = int64_t(1) << 58;  // elements from the first to the last of a tensor, along each of its axes: offsets in bytes stay below 2^63
constexpr int64_t MOST_POSITIONS = int64_t(1) << 31;  // of a rotary table
// whether the last of n things that lie `stride` elements apart is within that (n, stride >= 0)
bool in_reach(int64_t n, int64_t stride) { return n < 2 || stride <= FURTHEST / (n - 1); }

// a matrix that a call reads or writes: its rows do not overlap, its elements lie at multiples of their size
int check_matrix(const void *p, int64_t ld, int64_t rows, int64_t cols, int dtype)
{
    if (ld < cols || ld > MOST || !in_reach(rows, ld)) return MXFP4_ESHAPE;
    return aligned(p, element(dtype)) ? MXFP4_OK : MXFP4_EALIGN;
}

int check_norm_cfg(const mxfp4_norm_cfg *cfg, int x_dtype, int branch_dtype)
{
    if (!cfg || !known_type(x_dtype) || !known_type(branch_dtype)) return MXFP4_EINVAL;
    if (!(cfg->eps >= 0.0f) || !isfinite(cfg->eps) || !isfinite(cfg->residual_scale) || !isfinite(cfg->branch_scale) ||
        !isfinite(cfg->weight_offset))
        return MXFP4_EINVAL;
    return flag(cfg->post_norm) && flag(cfg->accumulate) ? MXFP4_OK : MXFP4_EINVAL;
}

struct Operand {
    const void *p;
    int64_t ld;
    int dtype;
};
// those that are there
template <int N>
int check_matrices(const Operand (&list)[N], int64_t rows, int64_t cols)
{
    for (const Operand &m : list)
        if (m.p)
            if (const int rc = check_matrix(m.p, m.ld, rows, cols, m.dtype)) return rc;
    return MXFP4_OK;
}

int check_gate(const void *gate, int64_t ld_gate, int64_t rows, int64_t cols, int branch_dtype)
{
    if (!gate) return MXFP4_OK;
    if (ld_gate == 0) return aligned(gate, 4) ? MXFP4_OK : MXFP4_EALIGN;
    return check_matrix(gate, ld_gate, rows, cols, branch_dtype);
}

NormArgs norm_args(const mxfp4_norm_cfg *cfg, int64_t rows, int64_t cols, int x_dtype, int branch_dtype)
{
    NormArgs a;
    a.rows = rows;
    a.cols = (int)cols;
    a.eps = cfg->eps;
    a.alpha = cfg->residual_scale;
    a.beta = cfg->branch_scale;
    a.offset = cfg->weight_offset;
    a.post = cfg->post_norm;
    a.accumulate = cfg->accumulate;
    a.x_fp32 = x_dtype == MXFP4_OUT_FP32;
    a.branch_fp32 = branch_dtype == MXFP4_OUT_FP32;
    return a;
}

// Sizes of an update that are not too large: a launch has one tile of at least 64 x 64 per workgroup, of 256 threads, and fewer than 2^32 threads.
bool ortho_sizes(int64_t batch, int64_t N, int64_t K)
{
    return batch <= 65535 && N <= ORTHO_MAX && K <= ORTHO_MAX && batch * ((N + 63) / 64) * ((K + 63) / 64) < (int64_t(1) << 24);
}

// Whether the singular values of X stay in range: those of the first X are at most 1, and every step takes [0, most] into the polynomial's range over it,
// whose extremes lie at its ends or where its derivative a + 3 b t + 5 c t^2 (t = s^2) vanishes.  They have to stay below what the fp16 scales of X (and so
// of its square A, and of P A) and of Q leave room for.  joined: whether those of the P of two and three steps, multiplied, do too (else steps stay single also where joining is asked for).
bool coefficients_in_range(const mxfp4_muon_cfg *cfg, bool &joined)
{
    const double a = cfg->a, b = cfg->b, c = cfg->c;
    if (!isfinite(a) || !isfinite(b) || !isfinite(c)) return false;
    double most = 1.0, largest_p = 0.0;
    for (int step = 0; step < cfg->steps; ++step) {
        double roots[4] = {most * most, 0.0, 0.0, 0.0};
        const double half = 1.5 * b, under = half * half - 5.0 * c * a;
        if (under >= 0.0) {  // (the form of the roots in which nothing cancels, however small c is)
            const double q = -(half + copysign(sqrt(under), half));
            if (c != 0.0) roots[1] = q / (5.0 * c);
            if (q != 0.0) roots[2] = a / q;
        }
        if (c != 0.0) roots[3] = -b / (2.0 * c);  // where b t + c t^2 is extreme
        double next = 0.0, largest_q = 0.0;
        for (double t : roots) {
            if (!(t >= 0.0) || t > most * most) continue;
            const double q = b * t + c * t * t;
            next = fmax(next, sqrt(t) * fabs(a + q));
            largest_q = fmax(largest_q, fabs(q));
            largest_p = fmax(largest_p, fabs(a + q));
        }
        largest_p = fmax(largest_p, fabs(a));
        if (!(next <= 1.9) || !(largest_q <= 15.0)) return false;
        most = fmax(most, next);
    }
    joined = largest_p * largest_p <= 15.0;  // (and those of three below 60)
    return true;
}

}  // namespace

extern "C" {

int mxfp4_residual_norm_fwd(const void *x, int64_t ld_x, const void *o, int64_t ld_o, const void *gate, int64_t ld_gate,
                            const float *w_post, const float *w_pre, int64_t rows, int64_t cols, int x_dtype, int branch_dtype,
                            const mxfp4_norm_cfg *cfg, void *x_out, int64_t ld_x_out, void *h, int64_t ld_h, float *rstd,
                            void *hip_stream)
{
    int rc = check_norm_cfg(cfg, x_dtype, branch_dtype);
    if (rc != MXFP4_OK) return rc;
    if (rows < 0 || cols < 1 || rows > MOST || cols > NORM_MAX_COLS) return MXFP4_ESHAPE;
    if (w_post && !cfg->post_norm) return MXFP4_EINVAL;
    if (rows == 0) return MXFP4_OK;
    if (!o && (gate || w_post || cfg->post_norm)) return MXFP4_EINVAL;
    if (w_pre && !h) return MXFP4_EINVAL;
    if (!x || (!x_out && !h)) return MXFP4_EINVAL;
    const Operand list[] = {{x, ld_x, x_dtype}, {o, ld_o, branch_dtype}, {x_out, ld_x_out, x_dtype}, {h, ld_h, branch_dtype}};
    if ((rc = check_matrices(list, rows, cols)) != MXFP4_OK || (rc = check_gate(gate, ld_gate, rows, cols, branch_dtype)) != MXFP4_OK) return rc;
    if (!aligned(w_post, 4) || !aligned(w_pre, 4) || !aligned(rstd, 4)) return MXFP4_EALIGN;
    if (!device_ok()) return MXFP4_EDEVICE;
    NormArgs a = norm_args(cfg, rows, cols, x_dtype, branch_dtype);
    a.x = x; a.ld_x = ld_x;
    a.o = o; a.ld_o = ld_o;
    a.gate = gate; a.ld_gate = ld_gate;
    a.w_post = w_post; a.w_pre = w_pre;
    a.x_out = x_out; a.ld_x_out = ld_x_out;
    a.h = h; a.ld_h = ld_h;
    a.rstd = rstd;
    return launch_norm_fwd(a, static_cast<hipStream_t>(hip_stream)) == hipSuccess ? MXFP4_OK : MXFP4_EDEVICE;
}

size_t mxfp4_residual_norm_workspace_bytes(int64_t rows, int64_t cols)
{
    if (rows < 0 || cols < 1 || rows > MOST || cols > NORM_MAX_COLS) return 0;
    return (size_t)norm_parts(rows) * (size_t)cols * 2 * sizeof(float);
}

int mxfp4_residual_norm_bwd(const void *dx_out, int64_t ld_dx_out, const void *dh, int64_t ld_dh, const void *x_out, int64_t ld_x_out,
                            const void *o, int64_t ld_o, const void *gate, int64_t ld_gate, const float *w_post, const float *w_pre,
                            const float *rstd, int64_t rows, int64_t cols, int x_dtype, int branch_dtype, const mxfp4_norm_cfg *cfg,
                            void *dx, int64_t ld_dx, void *d_o, int64_t ld_do, void *dgate, int64_t ld_dgate, float *dw_post,
                            float *dw_pre, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    int rc = check_norm_cfg(cfg, x_dtype, branch_dtype);
    if (rc != MXFP4_OK) return rc;
    if (rows < 0 || cols < 1 || rows > MOST || cols > NORM_MAX_COLS) return MXFP4_ESHAPE;
    if (!dx && !d_o && !dgate && !dw_post && !dw_pre) return MXFP4_OK;
    const bool vector_gate = gate && ld_gate == 0;
    if ((w_post && !cfg->post_norm) || (dw_post && !cfg->post_norm) || (dgate && !gate)) return MXFP4_EINVAL;
    const bool sums = dw_post || dw_pre || (dgate && vector_gate);
    if (rows > 0) {
        if (!dx_out && !dh) return MXFP4_EINVAL;
        if (!dh && (dw_pre || w_pre)) return MXFP4_EINVAL;
        if (dh && (!x_out || !rstd)) return MXFP4_EINVAL;
        if (!o && ((cfg->post_norm && (d_o || dw_post)) || dgate)) return MXFP4_EINVAL;
        if (cfg->post_norm && (d_o || dw_post || dgate) && !rstd) return MXFP4_EINVAL;
        const Operand list[] = {{dx_out, ld_dx_out, x_dtype}, {dh, ld_dh, branch_dtype}, {x_out, ld_x_out, x_dtype},
                                {o, ld_o, branch_dtype}, {dx, ld_dx, x_dtype}, {d_o, ld_do, branch_dtype}};
        if ((rc = check_matrices(list, rows, cols)) != MXFP4_OK || (rc = check_gate(gate, ld_gate, rows, cols, branch_dtype)) != MXFP4_OK) return rc;
        if (dgate && !vector_gate && (rc = check_matrix(dgate, ld_dgate, rows, cols, branch_dtype)) != MXFP4_OK) return rc;
        if (sums && !workspace) return MXFP4_EINVAL;
        if (sums && workspace_bytes < mxfp4_residual_norm_workspace_bytes(rows, cols)) return MXFP4_EWORKSPACE;
    }
    if (!aligned(w_post, 4) || !aligned(w_pre, 4) || !aligned(rstd, 4) || !aligned(dw_post, 4) || !aligned(dw_pre, 4) ||
        (vector_gate && !aligned(dgate, 4)) || (sums && !aligned(workspace, 16)))
        return MXFP4_EALIGN;
    if (rows == 0 && !sums) return MXFP4_OK;
    if (!device_ok()) return MXFP4_EDEVICE;
    NormArgs a = norm_args(cfg, rows, cols, x_dtype, branch_dtype);
    a.dx_out = dx_out; a.ld_dx_out = ld_dx_out;
    a.dh = dh; a.ld_dh = ld_dh;
    a.x = x_out; a.ld_x = ld_x_out;
    a.o = o; a.ld_o = ld_o;
    a.gate = gate; a.ld_gate = ld_gate;
    a.w_post = w_post; a.w_pre = w_pre;
    a.rstd = const_cast<float *>(rstd);
    a.dx = dx; a.ld_dx = ld_dx;
    a.d_o = d_o; a.ld_do = ld_do;
    a.dgate = dgate; a.ld_dgate = ld_dgate;
    a.dw_post = dw_post; a.dw_pre = dw_pre;
    a.partial = static_cast<float *>(workspace);
    if (a.post && !a.rstd) a.post = 0;  // (dx alone: the norm behind the block plays no part)
    return launch_norm_bwd(a, static_cast<hipStream_t>(hip_stream)) == hipSuccess ? MXFP4_OK : MXFP4_EDEVICE;
}

int mxfp4_rope_table(float *table, int64_t positions, int64_t rot_dim, const mxfp4_rope_cfg *cfg, void *hip_stream)
{
    if (!cfg || cfg->scaling < MXFP4_ROPE_SCALE_NONE || cfg->scaling > MXFP4_ROPE_SCALE_WAVELENGTH) return MXFP4_EINVAL;
    if (!isfinite(cfg->base) || !(cfg->base > 1.0) || !isfinite(cfg->attention_factor) || cfg->attention_factor < 0.0) return MXFP4_EINVAL;
    if (cfg->scaling != MXFP4_ROPE_SCALE_NONE && (!isfinite(cfg->factor) || !(cfg->factor >= 1.0))) return MXFP4_EINVAL;
    if (cfg->scaling >= MXFP4_ROPE_SCALE_YARN &&
        (!isfinite(cfg->low) || !isfinite(cfg->high) || !(cfg->low > 0.0) || !(cfg->high > cfg->low) || !isfinite(cfg->original_positions) ||
         !(cfg->original_positions > 0.0)))
        return MXFP4_EINVAL;
    if (positions < 0 || positions > MOST_POSITIONS || rot_dim < 2 || rot_dim % 2 != 0 || rot_dim > 65536) return MXFP4_ESHAPE;
    if (positions == 0) return MXFP4_OK;
    if (!table) return MXFP4_EINVAL;
    if (!aligned(table, 16)) return MXFP4_EALIGN;
    if (!device_ok()) return MXFP4_EDEVICE;
    const RopeTableArgs a{table, positions, (int)rot_dim, cfg->base, cfg->factor, cfg->low, cfg->high, cfg->original_positions,
                          cfg->attention_factor, cfg->scaling};
    return launch_rope_table(a, static_cast<hipStream_t>(hip_stream)) == hipSuccess ? MXFP4_OK : MXFP4_EDEVICE;
}

int mxfp4_rope(const void *x, int64_t x_token, int64_t x_head, void *out, int64_t out_token, int64_t out_head, int64_t tokens,
               int64_t heads, int64_t head_dim, int64_t rot_dim, int dtype, int layout, int inverse, const int32_t *positions,
               int64_t first_position, const float *table, int64_t table_positions, void *hip_stream)
{
    if (!known_type(dtype) || !flag(inverse) || (layout != MXFP4_ROPE_HALF && layout != MXFP4_ROPE_PAIRS)) return MXFP4_EINVAL;
    if (tokens < 0 || heads < 0 || tokens > MOST || heads > (1 << 20) || head_dim < 2 || head_dim > 65536 || rot_dim < 2 || rot_dim % 2 != 0 ||
        rot_dim > head_dim || table_positions < 0 || table_positions > MOST_POSITIONS)
        return MXFP4_ESHAPE;
    if (tokens == 0 || heads == 0) return MXFP4_OK;
    if (!x || !out || !table) return MXFP4_EINVAL;
    if (x_token < 0 || x_head < 0 || out_token < 0 || out_head < 0 || x_token > MOST || x_head > MOST || out_token > MOST || out_head > MOST)
        return MXFP4_ESHAPE;
    if (!in_reach(tokens, x_token) || !in_reach(tokens, out_token) || !in_reach(heads, x_head) || !in_reach(heads, out_head) ||
        tokens > FURTHEST / (heads * head_dim))
        return MXFP4_ESHAPE;
    // heads of the output must not overlap: token by token, or head by head
    const bool by_token = (heads == 1 || out_head >= head_dim) && (tokens == 1 || out_token >= (heads - 1) * out_head + head_dim);
    const bool by_head = (tokens == 1 || out_token >= head_dim) && (heads == 1 || out_head >= (tokens - 1) * out_token + head_dim);
    if (!by_token && !by_head) return MXFP4_ESHAPE;
    if (x == out && ((tokens > 1 && x_token != out_token) || (heads > 1 && x_head != out_head))) return MXFP4_EINVAL;
    if (!aligned(x, element(dtype)) || !aligned(out, element(dtype)) || !aligned(positions, 4) || !aligned(table, 16)) return MXFP4_EALIGN;
    if (!device_ok()) return MXFP4_EDEVICE;
    // (further from the table than there are tokens none of them is in it; the sum of position and token stays in range)
    const int64_t first = first_position < -2 * MOST ? -2 * MOST : first_position > 2 * MOST ? 2 * MOST : first_position;
    const RopeArgs a{x, out, x_token, x_head, out_token, out_head, tokens, (int)heads, (int)head_dim, (int)rot_dim,
                     dtype == MXFP4_OUT_FP32, layout == MXFP4_ROPE_PAIRS, inverse, positions, first, table, table_positions};
    return launch_rope(a, static_cast<hipStream_t>(hip_stream)) == hipSuccess ? MXFP4_OK : MXFP4_EDEVICE;
}

size_t mxfp4_orthogonalize_workspace_bytes(int64_t batch, int64_t N, int64_t K)
{
    if (batch < 1 || N < 1 || K < 1 || !ortho_sizes(batch, N, K)) return 0;
    return ortho_workspace_bytes(batch, N, K);
}

int mxfp4_orthogonalize(const void *g, int64_t ld_g, int64_t g_matrix, float *momentum, void *out, int64_t ld_out, int64_t out_matrix,
                        int64_t batch, int64_t N, int64_t K, int g_dtype, const mxfp4_muon_cfg *cfg, void *workspace,
                        size_t workspace_bytes, void *hip_stream)
{
    if (!cfg || !known_type(g_dtype) || !flag(cfg->nesterov) || !flag(cfg->join_steps) || cfg->steps < 1 || cfg->steps > 64) return MXFP4_EINVAL;
    if (!(cfg->eps > 0.0f) || !isfinite(cfg->eps) || !isfinite(cfg->momentum) || !isfinite(cfg->out_scale)) return MXFP4_EINVAL;
    bool joined = false;
    if (!coefficients_in_range(cfg, joined)) return MXFP4_EINVAL;
    if (batch < 0 || N < 0 || K < 0 || !ortho_sizes(batch, N, K)) return MXFP4_ESHAPE;
    if (batch == 0 || N == 0 || K == 0) return MXFP4_OK;
    if (!g || !out || !workspace) return MXFP4_EINVAL;
    int rc;
    if ((rc = check_matrix(g, ld_g, N, K, g_dtype)) != MXFP4_OK || (rc = check_matrix(out, ld_out, N, K, MXFP4_OUT_BF16)) != MXFP4_OK) return rc;
    if (batch > 1 && (g_matrix < 0 || g_matrix > MOST || out_matrix < (N - 1) * ld_out + K || out_matrix > MOST)) return MXFP4_ESHAPE;
    if (workspace_bytes < ortho_workspace_bytes(batch, N, K)) return MXFP4_EWORKSPACE;
    if (!aligned(workspace, 256) || !aligned(momentum, 4)) return MXFP4_EALIGN;
    if (!device_ok()) return MXFP4_EDEVICE;
    OrthoArgs a{};
    a.g = g;
    a.momentum = momentum;
    a.out = out;
    a.batch = batch;
    a.N = N;
    a.K = K;
    a.ld_g = ld_g;
    a.ld_out = ld_out;
    a.g_matrix = g_matrix;
    a.out_matrix = out_matrix;
    a.g_fp32 = g_dtype == MXFP4_OUT_FP32;
    a.nesterov = cfg->nesterov;
    a.steps = cfg->steps;
    a.joined = cfg->join_steps && joined;
    a.mu = cfg->momentum;
    a.a = cfg->a;
    a.b = cfg->b;
    a.c = cfg->c;
    a.eps = cfg->eps;
    a.out_scale = cfg->out_scale;
    a.workspace = static_cast<uint8_t *>(workspace);
    return launch_orthogonalize(a, static_cast<hipStream_t>(hip_stream)) == hipSuccess ? MXFP4_OK : MXFP4_EDEVICE;
}

}  // extern "C"
