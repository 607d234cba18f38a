// Norms behind one block and before the next, with the block's gate and the residual sum between them:
//     n  = o r(o) (w_post + offset)            r(v) = (mean(v^2) + eps)^(-1/2)        (n = o without the norm behind the block)
//     x' = alpha x + beta gate n               h = x' r(x') (w_pre + offset)
// and their gradients.  With u the gradient of x' by both of its uses, ^ for v r(v) and the means over a row,
//     u = dx' + r(x') (dh w_pre - x'^ mean(dh w_pre x'^))         dx = alpha u
//     dn = beta gate u       do = r(o) (dn w_post - o^ mean(dn w_post o^))
//     dgate = beta u n       dw_post = sum over rows of dn o^     dw_pre = sum over rows of dh x'^
// With one gate for all rows, S = sum over rows of beta u o^ gives both dw_post = gate S and dgate = (w_post + offset) S.
//
// Memory is what bounds all of it: forward 57 us for 8192 x 4096 in bf16 (268 MB, 4.7 TB/s; a large copy here 4.9), backward 83 us (403 MB, 4.85
// TB/s; 4 us of it the sums' own launch), 38 us for 4010 x 1440 with 32-bit x and a gate per row (127 MB, 3.4 TB/s: four rounds of rows, of which the
// first waits for memory, and the second launch), 4.3 us of the chip's time for 24 x 4096.  A row lives in the registers of one workgroup (for short
// rows: of one or two of its waves), so that every tensor is read and written once; the sums of a row are the only thing that its lanes exchange.  All
// arithmetic is in fp32; h is formed from the unrounded x'.
#include "layer_ops.h"
#include "vector_io.h"

namespace mxfp4 {
namespace {

// Sum over the W waves that share a row, the same bits in all of them.  slots: 2 * W floats of the row's own; phase alternates, so that
// one barrier is enough: the slots of one sum are overwritten two barriers later.
template <int W>
__device__ __forceinline__ float row_sum(float v, float *slots, int phase, int wave)
{
    v = wave_sum(v);
    if (W == 1) return v;
    float *s = slots + (phase & 1) * W;
    if ((threadIdx.x & 63) == 0) s[wave] = v;
    lds_barrier();
    float t = 0.0f;
#pragma unroll
    for (int i = 0; i < W; ++i) t += s[i];
    return t;
}

typedef float v4 __attribute__((ext_vector_type(4)));

// Eight values of a lane as two vectors in LDS, `apart` vectors from each other.
__device__ __forceinline__ void put(v4 *p, int apart, const float (&f)[8])
{
    p[0] = v4{f[0], f[1], f[2], f[3]};
    p[apart] = v4{f[4], f[5], f[6], f[7]};
}
__device__ __forceinline__ void add_to(v4 *p, int apart, const float (&f)[8])
{
    p[0] += v4{f[0], f[1], f[2], f[3]};
    p[apart] += v4{f[4], f[5], f[6], f[7]};
}
__device__ __forceinline__ void add_from(const v4 *p, int apart, float (&f)[8])
{
    const v4 a = p[0], b = p[apart];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        f[e] += a[e];
        f[4 + e] += b[e];
    }
}

// W waves per row, NV vectors of 8 elements per lane, R rows at a time in a workgroup
template <typename X, typename O, int W, int NV, int R>
__global__ __launch_bounds__(64 * W *R) void norm_fwd_kernel(const NormArgs a)
{
    __shared__ float slots[R][2 * W];
    const int sub = threadIdx.x / (64 * W), t = threadIdx.x % (64 * W), wave = t >> 6;
    const bool row_gate = a.gate && a.ld_gate;
    int phase = 0;
    for (int64_t first = (int64_t)blockIdx.x * R; first < a.rows; first += (int64_t)gridDim.x * R) {
        const int64_t row = first + sub;
        const bool on = row < a.rows;
        Raw8<X> x[NV];
        Raw8<O> o[NV], gate[NV];
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int c = (v * 64 * W + t) * 8, n = on ? a.cols - c : 0;
            x[v].load(reinterpret_cast<const X *>(a.x) + row * a.ld_x + c, n);
            o[v].load(reinterpret_cast<const O *>(a.o) + row * a.ld_o + c, a.o ? n : 0);
            if (row_gate) gate[v].load(reinterpret_cast<const O *>(a.gate) + row * a.ld_gate + c, n);
        }
        float r = 1.0f;
        if (a.post) {
            float s = 0.0f;
#pragma unroll
            for (int v = 0; v < NV; ++v)
#pragma unroll
                for (int e = 0; e < 8; ++e) s = fmaf(o[v].get(e), o[v].get(e), s);
            r = rsqrtf(row_sum<W>(s, slots[sub], phase++, wave) / a.cols + a.eps);
            if (a.rstd && on && t == 0) a.rstd[row] = r;
        }
        float y[NV][8], s = 0.0f;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int c = (v * 64 * W + t) * 8, n = on ? a.cols - c : 0;
            Raw8<float> w, g;
            if (a.post && a.w_post) w.load(a.w_post + c, n);
            if (a.gate && !row_gate) g.load(reinterpret_cast<const float *>(a.gate) + c, n);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                float z = o[v].get(e) * r;
                if (a.post && a.w_post) z *= w.get(e) + a.offset;
                if (a.gate) z *= row_gate ? gate[v].get(e) : g.get(e);
                y[v][e] = fmaf(a.beta, z, a.alpha * x[v].get(e));
                if (c + e < a.cols && on) s = fmaf(y[v][e], y[v][e], s);
            }
            if (a.x_out) store8(reinterpret_cast<X *>(a.x_out) + row * a.ld_x_out + c, y[v], n);
        }
        if (!a.h) continue;
        r = rsqrtf(row_sum<W>(s, slots[sub], phase++, wave) / a.cols + a.eps);
        if (a.rstd && on && t == 0) a.rstd[a.rows + row] = r;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int c = (v * 64 * W + t) * 8, n = on ? a.cols - c : 0;
            Raw8<float> w;
            if (a.w_pre) w.load(a.w_pre + c, n);
#pragma unroll
            for (int e = 0; e < 8; ++e) y[v][e] *= a.w_pre ? r * (w.get(e) + a.offset) : r;
            store8(reinterpret_cast<O *>(a.h) + row * a.ld_h + c, y[v], n);
        }
    }
}

// The backward pass walks rows with R of them at a time in a workgroup: the sums over rows stay in its registers, are added over the R at the end, and
// leave once, as one row of partial sums.  AHEAD: the next row is on its way while one is worked on.  Rows of more than 8192 columns leave
// no registers for that, nor for the sums of the weights' gradients, which lie in LDS there, each lane's own.
enum NormGate { GATE_NONE = 0, GATE_VECTOR = 1, GATE_ROWS = 2 };

template <typename X, typename O, int NV, int GATE>
struct NormRow {
    Raw8<X> x[NV], dxo[NV];
    Raw8<O> o[NV], dh[NV], gate[GATE == GATE_ROWS ? NV : 1];
    float r_post, r_pre;
    __device__ __forceinline__ void load(const NormArgs &a, int64_t row, int t, int lanes)
    {
        const bool on = row < a.rows;
        r_post = a.post && on ? a.rstd[row] : 1.0f;
        r_pre = a.dh && on ? a.rstd[a.rows + row] : 0.0f;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int c = (v * lanes + t) * 8, n = on ? a.cols - c : 0;
            dh[v].load(reinterpret_cast<const O *>(a.dh) + row * a.ld_dh + c, a.dh ? n : 0);
            x[v].load(reinterpret_cast<const X *>(a.x) + row * a.ld_x + c, a.dh ? n : 0);
            dxo[v].load(reinterpret_cast<const X *>(a.dx_out) + row * a.ld_dx_out + c, a.dx_out ? n : 0);
            o[v].load(reinterpret_cast<const O *>(a.o) + row * a.ld_o + c, a.o ? n : 0);
            if (GATE == GATE_ROWS) gate[v].load(reinterpret_cast<const O *>(a.gate) + row * a.ld_gate + c, n);
        }
    }
};

template <typename X, typename O, int W, int NV, int R, int GATE>
__global__ __launch_bounds__(64 * W *R) void norm_bwd_kernel(const NormArgs a)
{
    constexpr int LANES = 64 * W;
    constexpr bool SUMS_IN_LDS = NV > 1, AHEAD = NV == 1 && (W < 16 || sizeof(X) + sizeof(O) == 4);
    // [dw_post (or S), dw_pre][vector][lane] of a workgroup's own sums; at the end, those of one of its R rows after the other
    constexpr int HELD = SUMS_IN_LDS || R > 1 ? 2 * NV * LANES * 8 : 1;
    __shared__ float slots[R][2 * W];
    __shared__ __attribute__((aligned(16))) float held[HELD];
    const int sub = threadIdx.x / LANES, t = threadIdx.x % LANES, wave = t >> 6;
    const auto mine = [&](int which, int v) -> v4 * { return reinterpret_cast<v4 *>(held) + ((which * NV + v) * 2 * LANES + t); };
    float s_post[SUMS_IN_LDS ? 1 : NV][8] = {}, s_pre[SUMS_IN_LDS ? 1 : NV][8] = {};
    float w_post[SUMS_IN_LDS ? 1 : NV][8], w_pre[SUMS_IN_LDS ? 1 : NV][8], vector[SUMS_IN_LDS ? 1 : NV][8];
    const auto weights = [&](const float *from, int v, float offset, float (&to)[8]) {
        const int c = (v * LANES + t) * 8;
        Raw8<float> w;
        if (from) w.load(from + c, a.cols - c);
#pragma unroll
        for (int e = 0; e < 8; ++e) to[e] = from ? w.get(e) + offset : 1.0f;
    };
    const float *gate_vector = GATE == GATE_VECTOR ? reinterpret_cast<const float *>(a.gate) : nullptr;
    if constexpr (SUMS_IN_LDS) {
#pragma unroll
        for (int k = 0; k < 2 * NV; ++k) {
            mine(k / NV, k % NV)[0] = v4{};
            mine(k / NV, k % NV)[LANES] = v4{};
        }
    } else {
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            weights(a.w_post, v, a.offset, w_post[v]);
            weights(a.w_pre, v, a.offset, w_pre[v]);
            weights(gate_vector, v, 0.0f, vector[v]);
        }
    }
    int phase = 0;
    NormRow<X, O, NV, GATE> now, next;
    if (AHEAD) now.load(a, (int64_t)blockIdx.x * R + sub, t, LANES);
    for (int64_t first = (int64_t)blockIdx.x * R; first < a.rows; first += (int64_t)gridDim.x * R) {
        const int64_t row = first + sub;
        const bool on = row < a.rows;
        if (AHEAD)
            next.load(a, row + (int64_t)gridDim.x * R, t, LANES);
        else
            now.load(a, row, t, LANES);
        float u[NV][8], s = 0.0f;
        if (a.dh) {
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                float w[8];
                if (SUMS_IN_LDS) weights(a.w_pre, v, a.offset, w);
                float add[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float g = now.dh[v].get(e), hat = now.x[v].get(e) * now.r_pre;
                    add[e] = g * hat;
                    u[v][e] = g * (SUMS_IN_LDS ? w[e] : w_pre[SUMS_IN_LDS ? 0 : v][e]);
                    s = fmaf(u[v][e], hat, s);
                    if (!SUMS_IN_LDS) s_pre[SUMS_IN_LDS ? 0 : v][e] += add[e];
                }
                if (SUMS_IN_LDS && a.dw_pre) add_to(mine(1, v), LANES, add);
            }
            s = row_sum<W>(s, slots[sub], phase++, wave) / a.cols;
        }
        float q = 0.0f;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int c = (v * LANES + t) * 8, n = on ? a.cols - c : 0;
            float w[8], g[8];
            if (SUMS_IN_LDS) {
                weights(a.w_post, v, a.offset, w);
                if (GATE == GATE_VECTOR) weights(gate_vector, v, 0.0f, g);
            }
            float dx[8], dg[8], add[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                float d = now.dxo[v].get(e);
                if (a.dh) d += now.r_pre * (u[v][e] - now.x[v].get(e) * now.r_pre * s);
                dx[e] = a.alpha * d;
                d *= a.beta;
                const float hat = now.o[v].get(e) * now.r_post, wp = SUMS_IN_LDS ? w[e] : w_post[SUMS_IN_LDS ? 0 : v][e];
                if (GATE == GATE_ROWS) {
                    dg[e] = d * (hat * wp);
                    d *= now.gate[GATE == GATE_ROWS ? v : 0].get(e);
                }
                add[e] = d * hat;
                if (GATE == GATE_VECTOR) d *= SUMS_IN_LDS ? g[e] : vector[SUMS_IN_LDS ? 0 : v][e];
                if (!SUMS_IN_LDS) s_post[SUMS_IN_LDS ? 0 : v][e] += add[e];
                u[v][e] = d * wp;
                q = fmaf(u[v][e], hat, q);
            }
            if (SUMS_IN_LDS) add_to(mine(0, v), LANES, add);
            if (a.dx) store8(reinterpret_cast<X *>(a.dx) + row * a.ld_dx + c, dx, n);
            if (GATE == GATE_ROWS && a.dgate) store8(reinterpret_cast<O *>(a.dgate) + row * a.ld_dgate + c, dg, n);
        }
        if (a.d_o) {
            if (a.post) q = row_sum<W>(q, slots[sub], phase++, wave) / a.cols;
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                const int c = (v * LANES + t) * 8, n = on ? a.cols - c : 0;
                if (a.post)
#pragma unroll
                    for (int e = 0; e < 8; ++e) u[v][e] = now.r_post * (u[v][e] - now.o[v].get(e) * now.r_post * q);
                store8(reinterpret_cast<O *>(a.d_o) + row * a.ld_do + c, u[v], n);
            }
        }
        if (AHEAD) now = next;
    }
    // the other rows' sums to the first one's lanes
    for (int k = 1; k < R; ++k) {
        lds_barrier();
        if (sub == k)
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                put(mine(0, v), LANES, s_post[SUMS_IN_LDS ? 0 : v]);
                put(mine(1, v), LANES, s_pre[SUMS_IN_LDS ? 0 : v]);
            }
        lds_barrier();
        if (sub == 0)
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                add_from(mine(0, v), LANES, s_post[SUMS_IN_LDS ? 0 : v]);
                add_from(mine(1, v), LANES, s_pre[SUMS_IN_LDS ? 0 : v]);
            }
    }
    if (sub) return;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int c = (v * LANES + t) * 8, n = a.cols - c;
        float *to = a.partial + (int64_t)blockIdx.x * a.cols + c;
        const int64_t next_vector = (int64_t)gridDim.x * a.cols;
        float post[8] = {}, pre[8] = {};
        if (SUMS_IN_LDS) {
            add_from(mine(0, v), LANES, post);
            add_from(mine(1, v), LANES, pre);
        }
        if (a.dw_post || (GATE == GATE_VECTOR && a.dgate)) store8(to, SUMS_IN_LDS ? post : s_post[SUMS_IN_LDS ? 0 : v], n);
        if (a.dw_pre) store8(to + next_vector, SUMS_IN_LDS ? pre : s_pre[SUMS_IN_LDS ? 0 : v], n);
    }
}

// Partial sums to the vectors (blockIdx.y 0: dw_post and a vector's dgate, 1: dw_pre): a wave's lanes are columns, its 16 waves take every 16th
// part, in the order of the parts.
__global__ __launch_bounds__(1024) void norm_sums_kernel(const NormArgs a, int64_t parts)
{
    __shared__ float sums[16][64];
    const bool vector_gate = a.gate && !a.ld_gate;
    float *dgate = vector_gate ? static_cast<float *>(a.dgate) : nullptr;
    if (blockIdx.y ? !a.dw_pre : !a.dw_post && !dgate) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = blockIdx.x * 64 + lane;
    const float *p = a.partial + (int64_t)blockIdx.y * parts * a.cols + c;
    float s = 0.0f;
    if (c < a.cols) {
#pragma unroll 8
        for (int64_t i = wave; i < parts; i += 16) s += p[i * a.cols];
    }
    sums[wave][lane] = s;
    __syncthreads();
    if (wave || c >= a.cols) return;
    s = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i) s += sums[i][lane];
    const auto write = [&](float *out, float v) {
        if (out) out[c] = a.accumulate ? out[c] + v : v;
    };
    if (blockIdx.y) {
        write(a.dw_pre, s);
    } else {
        write(a.dw_post, vector_gate ? s * static_cast<const float *>(a.gate)[c] : s);
        write(dgate, a.w_post ? s * (a.w_post[c] + a.offset) : s);
    }
}

constexpr int64_t MAX_GROUPS = 1 << 20;  // beyond that a workgroup takes several rows, so that the grid stays within what HIP launches

template <typename F>
hipError_t with_types(const NormArgs &a, F f)
{
    if (a.x_fp32) return a.branch_fp32 ? f(float{}, float{}) : f(float{}, uint16_t{});
    return a.branch_fp32 ? f(uint16_t{}, float{}) : f(uint16_t{}, uint16_t{});
}

template <typename X, typename O, int W, int NV, int R>
hipError_t fwd(const NormArgs &a, hipStream_t st)
{
    const int64_t groups = (a.rows + R - 1) / R;
    hipLaunchKernelGGL((norm_fwd_kernel<X, O, W, NV, R>), dim3((uint32_t)(groups < MAX_GROUPS ? groups : MAX_GROUPS)), dim3(64 * W * R), 0, st, a);
    return hipGetLastError();
}

// Workgroups of the backward pass, and so rows of partial sums: few rows get a workgroup each, many are walked by a workgroup of 8 to 16 waves on each
// compute unit (8192 x 4096: 512 workgroups of eight waves took 118 us, and wrote and read twice the partial sums).  Both launches together, a workgroup per row
// against walked (us, bf16, one gate): 256 rows of 64 columns 8.9 / 12.7, of 1440 10.6 / 13.2, of 4096 14.4 / 15.2; 512 rows 9.7 / 13.0, 13.3 / 13.4, 20.2 / 16.8;
// 1024 rows 11.4 / 12.4, 19.1 / 14.8, 28.6 / 19.4; 2048 rows 14.7 / 12.9, 27.8 / 18.7, 47.9 / 25.5.  One limit for all widths: rows of 4096 columns would change over at
// about 300, rows of up to 512 columns at about 1000 (in between they lose 1 to 3 us).
constexpr int64_t FEW_ROWS = 512, MANY_GROUPS = 256;

template <typename X, typename O, int W, int NV>
hipError_t bwd(const NormArgs &a, hipStream_t st)
{
    const auto launch = [&](auto gate) {
        // (16 waves leave 128 registers each, 12 leave 170, which rows of 32-bit elements take twice: 4010 x 1440 with a gate per row 44 us with 8)
        constexpr int GATE = decltype(gate)::value, WAVES = sizeof(X) + sizeof(O) == 4 || W > 12 ? 16 : 12, R = WAVES / W;
        if (a.rows <= FEW_ROWS)
            hipLaunchKernelGGL((norm_bwd_kernel<X, O, W, NV, 1, GATE>), dim3((uint32_t)a.rows), dim3(64 * W), 0, st, a);
        else
            hipLaunchKernelGGL((norm_bwd_kernel<X, O, W, NV, R, GATE>), dim3(MANY_GROUPS), dim3(64 * W * R), 0, st, a);
        return hipGetLastError();
    };
    if (!a.gate) return launch(std::integral_constant<int, GATE_NONE>{});
    return a.ld_gate ? launch(std::integral_constant<int, GATE_ROWS>{}) : launch(std::integral_constant<int, GATE_VECTOR>{});
}

}  // namespace

int64_t norm_parts(int64_t rows) { return rows <= FEW_ROWS ? rows : MANY_GROUPS; }

// f(waves per row, vectors per lane): 512 columns to a wave, and beyond 8192 columns two vectors to a lane
template <typename F>
hipError_t with_shape(int cols, F f)
{
    using std::integral_constant;
    if (cols <= 512) return f(integral_constant<int, 1>{}, integral_constant<int, 1>{});
    if (cols <= 1024) return f(integral_constant<int, 2>{}, integral_constant<int, 1>{});
    if (cols <= 1536) return f(integral_constant<int, 3>{}, integral_constant<int, 1>{});
    if (cols <= 2048) return f(integral_constant<int, 4>{}, integral_constant<int, 1>{});
    if (cols <= 3072) return f(integral_constant<int, 6>{}, integral_constant<int, 1>{});
    if (cols <= 4096) return f(integral_constant<int, 8>{}, integral_constant<int, 1>{});
    if (cols <= 6144) return f(integral_constant<int, 12>{}, integral_constant<int, 1>{});
    if (cols <= 8192) return f(integral_constant<int, 16>{}, integral_constant<int, 1>{});
    return f(integral_constant<int, 16>{}, integral_constant<int, 2>{});
}

hipError_t launch_norm_fwd(const NormArgs &a, hipStream_t st)
{
    return with_types(a, [&](auto x, auto o) {
        return with_shape(a.cols, [&](auto waves, auto vectors) {
            constexpr int W = decltype(waves)::value, R = W < 4 ? 4 / W : 1;  // four waves in a workgroup at least
            return fwd<decltype(x), decltype(o), W, decltype(vectors)::value, R>(a, st);
        });
    });
}

hipError_t launch_norm_bwd(const NormArgs &a, hipStream_t st)
{
    const int64_t parts = norm_parts(a.rows);
    if (parts) {
        const hipError_t e = with_types(a, [&](auto x, auto o) {
            return with_shape(a.cols, [&](auto waves, auto vectors) {
                return bwd<decltype(x), decltype(o), decltype(waves)::value, decltype(vectors)::value>(a, st);
            });
        });
        if (e != hipSuccess) return e;
    }
    if (!a.dw_post && !a.dw_pre && !(a.gate && !a.ld_gate && a.dgate)) return hipSuccess;
    hipLaunchKernelGGL(norm_sums_kernel, dim3((a.cols + 63) / 64, 2), dim3(1024), 0, st, a, parts);
    return hipGetLastError();
}

}  // namespace mxfp4
