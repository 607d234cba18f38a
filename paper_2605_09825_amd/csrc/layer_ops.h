// Launch interface of the operators around a linear layer: residual norm, rotary positions, orthogonalised updates.  As in
// mxfp4_internal.h, every launcher assumes that its caller has checked the arguments, and returns the launch's hipError_t.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace mxfp4 {

struct NormArgs {  // elements of x, x_out, dx_out, dx: fp32 if x_fp32, else bf16; of o, h, dh, d_o, a gate per row: branch_fp32
    const void *x = nullptr, *o = nullptr, *gate = nullptr;   // forward: the residual; backward: x_out of the forward pass
    const void *dx_out = nullptr, *dh = nullptr;              // backward
    const float *w_post = nullptr, *w_pre = nullptr;
    float *rstd = nullptr;                                    // [2][rows]: written by the forward pass, read by the backward one
    void *x_out = nullptr, *h = nullptr;                      // forward
    void *dx = nullptr, *d_o = nullptr, *dgate = nullptr;     // backward
    float *dw_post = nullptr, *dw_pre = nullptr;
    float *partial = nullptr;                                 // backward: sums over rows for dw_post (and a vector's dgate), dw_pre: [2][parts][cols]
    int64_t ld_x = 0, ld_o = 0, ld_gate = 0, ld_x_out = 0, ld_h = 0, ld_dx_out = 0, ld_dh = 0, ld_dx = 0, ld_do = 0, ld_dgate = 0;
    int64_t rows = 0;
    int cols = 0;
    float eps = 0, alpha = 1, beta = 1, offset = 0;
    int post = 0, accumulate = 0, x_fp32 = 0, branch_fp32 = 0;
};
constexpr int64_t NORM_MAX_COLS = 16384;
int64_t norm_parts(int64_t rows);  // rows of partial sums that the backward launch writes
hipError_t launch_norm_fwd(const NormArgs &a, hipStream_t st);
hipError_t launch_norm_bwd(const NormArgs &a, hipStream_t st);

struct RopeTableArgs {
    float *table;  // [positions][rot / 2][2]: cos, sin
    int64_t positions;
    int rot;
    double base, factor, low, high, original, attention;
    int scaling;
};
hipError_t launch_rope_table(const RopeTableArgs &a, hipStream_t st);

struct RopeArgs {
    const void *x;
    void *out;
    int64_t x_token, x_head, out_token, out_head;  // strides in elements
    int64_t tokens;
    int heads, dim, rot;
    int fp32, pairs_layout, inverse;
    const int32_t *positions;  // null: first, first + 1, ...
    int64_t first;
    const float *table;
    int64_t table_positions;
};
hipError_t launch_rope(const RopeArgs &a, hipStream_t st);

struct OrthoArgs {
    const void *g;     // [batch][N][ld_g], fp32 if g_fp32, else bf16
    float *momentum;   // [batch][N][K] dense, or null
    void *out;         // bf16 [batch][N][ld_out]
    int64_t batch, N, K, ld_g, ld_out, g_matrix, out_matrix;  // ..._matrix: elements from one matrix to the next
    int g_fp32, nesterov, steps;
    bool joined;       // two and three steps in one: asked for, and within what the coefficients allow
    float mu, a, b, c, eps, out_scale;
    uint8_t *workspace;
};
constexpr int64_t ORTHO_MAX = 1 << 20;  // rows or columns of a matrix
size_t ortho_workspace_bytes(int64_t batch, int64_t N, int64_t K);
hipError_t launch_orthogonalize(const OrthoArgs &a, hipStream_t st);

}  // namespace mxfp4
