// Rotary positions: pairs (u, v) of a head's first `rot` elements become (u cos - v sin, v cos + u sin), with the angle position * frequency
// of the pair.  Pairs are elements i and i + rot / 2 ("half") or 2 i and 2 i + 1 ("pairs").  The gradient turns the other way (inverse); an
// attention factor, which the table holds with cos and sin, multiplies in both.
//
// Memory bound: each head is read and written once (8192 tokens x 40 heads of 128 in bf16 36 us, 172 MB at 4.7 TB/s; 4010 x 32 in 32 bits, half of each
// head turned, 27 us at 4.9; 24 tokens 3.4).  cos and sin come from a table in fp32, one row per position, built once in 64 bits:
// angles of 10^5 radians would lose three digits in fp32.  A wave takes one token and walks its heads, so that a lane keeps the table values
// of its elements in registers for all of them.
#include "launch_limits.h"
#include "layer_ops.h"
#include "vector_io.h"

#include <type_traits>

namespace mxfp4 {
namespace {

__global__ __launch_bounds__(256) void rope_table_kernel(const RopeTableArgs a)
{
    const int pairs = a.rot / 2;
    const int i = blockIdx.y * 64 + (threadIdx.x & 63);
    if (i >= pairs) return;
    constexpr double TWO_PI = 6.283185307179586476925;
    double base = a.base, magnitude = a.attention;
    if (a.scaling == 2 && a.rot > 2) base *= pow(a.factor, (double)a.rot / (a.rot - 2));  // NTK-aware base
    double f = pow(base, -2.0 * i / a.rot);
    if (a.scaling == 1) {  // positions interpolated linearly
        f /= a.factor;
    } else if (a.scaling == 3) {
        // YaRN: pairs that turn more than `high` times over the original context keep their frequency, those that turn less than `low`
        // times are interpolated, a ramp over the pair's number between them; attention is sharpened by 0.1 ln(factor) + 1
        const double per = a.rot / (2.0 * log(base));
        double from = floor(per * log(a.original / (a.high * TWO_PI))), to = ceil(per * log(a.original / (a.low * TWO_PI)));
        from = fmax(from, 0.0);
        to = fmin(to, a.rot - 1.0);
        const double ramp = fmin(fmax((i - from) / fmax(to - from, 1e-3), 0.0), 1.0);
        f = f / a.factor * ramp + f * (1.0 - ramp);
        if (magnitude == 0.0) magnitude = 0.1 * log(a.factor) + 1.0;
    } else if (a.scaling == 4) {
        // by wavelength: longer than original / low interpolated, shorter than original / high kept, a smooth step between them
        const double turns = a.original * f / TWO_PI;
        const double keep = fmin(fmax((turns - a.low) / (a.high - a.low), 0.0), 1.0);
        f = f / a.factor * (1.0 - keep) + f * keep;
    }
    if (magnitude == 0.0) magnitude = 1.0;
    for (int64_t position = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); position < a.positions; position += (int64_t)gridDim.x * 4) {
        double s, c;
        sincos(position * f, &s, &c);
        a.table[2 * (position * pairs + i)] = (float)(c * magnitude);
        a.table[2 * (position * pairs + i) + 1] = (float)(s * magnitude);
    }
}

__device__ __forceinline__ int64_t position_of(const RopeArgs &a, int64_t token)
{
    return a.positions ? (int64_t)a.positions[token] : a.first + token;
}

// Any sizes, strides and alignment: a thread per pair, then one per element that is not turned.  A position outside the table gives NaN.
template <typename T>
__global__ __launch_bounds__(256) void rope_any_kernel(const RopeArgs a)
{
    const int pairs = a.rot / 2, rest = a.x == a.out ? 0 : a.dim - a.rot, units = pairs + rest;
    for (int64_t k = (int64_t)blockIdx.x * 256 + threadIdx.x; k < a.tokens * a.heads * units; k += (int64_t)gridDim.x * 256) {
        const int unit = (int)(k % units);
        const int64_t th = k / units, token = th / a.heads;
        const int head = (int)(th - token * a.heads);
        const T *x = static_cast<const T *>(a.x) + token * a.x_token + head * a.x_head;
        T *out = static_cast<T *>(a.out) + token * a.out_token + head * a.out_head;
        if (unit >= pairs) {
            out[a.rot + unit - pairs] = x[a.rot + unit - pairs];
            continue;
        }
        const int64_t position = position_of(a, token);
        float c = __builtin_nanf(""), s = c;
        if (position >= 0 && position < a.table_positions) {
            c = a.table[2 * (position * pairs + unit)];
            s = a.table[2 * (position * pairs + unit) + 1];
        }
        if (a.inverse) s = -s;
        const int iu = a.pairs_layout ? 2 * unit : unit, iv = a.pairs_layout ? iu + 1 : unit + pairs;
        if constexpr (std::is_same<T, float>::value) {
            const float u = x[iu], v = x[iv];
            out[iu] = u * c - v * s;
            out[iv] = v * c + u * s;
        } else {
            const float u = bf16_to_f32(x[iu]), v = bf16_to_f32(x[iv]);
            out[iu] = bf16_bits(u * c - v * s);
            out[iv] = bf16_bits(v * c + u * s);
        }
    }
}

// The sizes that models have: 16 bytes at a time.  A head is `units` lanes wide: `turned` of them take 16 bytes of u and of v (half) or of pairs as
// they lie, the rest copy what is not turned; the wave's 64 lanes hold 64 / units heads, and walk the token's heads that many at a time, DEEP of
// these steps under way together.  A lane's table values stay in its registers.
template <typename T>
struct RopeVec;
template <>
struct RopeVec<uint16_t> {
    static constexpr int N = 8;
    Vec16 v;
    __device__ __forceinline__ float get(int e) const { return e & 1 ? __uint_as_float(v.v[e >> 1] & 0xFFFF0000u) : __uint_as_float(v.v[e >> 1] << 16); }
    __device__ __forceinline__ void set(const float (&f)[8])
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) v.v[i] = bf16_pair(f[2 * i], f[2 * i + 1]);
    }
};
template <>
struct RopeVec<float> {
    static constexpr int N = 4;
    struct __attribute__((packed, aligned(4))) { uint32_t v[4]; } v;
    __device__ __forceinline__ float get(int e) const { return __uint_as_float(v.v[e]); }
    __device__ __forceinline__ void set(const float (&f)[4])
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) v.v[i] = __float_as_uint(f[i]);
    }
};

constexpr int DEEP = 4;

template <typename T, bool PAIRS>
__global__ __launch_bounds__(256) void rope_kernel(const RopeArgs a, const int units, const int turned, const int splits)
{
    using V = RopeVec<T>;
    constexpr int N = V::N, ANGLES = PAIRS ? N / 2 : N;
    const int lane = threadIdx.x & 63;
    const int64_t job = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6), token = job / splits;
    if (token >= a.tokens) return;
    const int split = (int)(job - token * splits), at_once = 64 / units;
    const int in_step = lane / units, unit = lane - in_step * units;
    if (in_step >= at_once) return;
    const bool turns = unit < turned;
    const int pairs = a.rot / 2;
    float c[ANGLES], s[ANGLES];
    if (turns) {
        const int64_t position = position_of(a, token);
        if (position >= 0 && position < a.table_positions) {
            const float4 *from = reinterpret_cast<const float4 *>(a.table + 2 * (position * pairs + unit * ANGLES));
#pragma unroll
            for (int i = 0; i < ANGLES / 2; ++i) {
                const float4 t = from[i];
                c[2 * i] = t.x;
                s[2 * i] = a.inverse ? -t.y : t.y;
                c[2 * i + 1] = t.z;
                s[2 * i + 1] = a.inverse ? -t.w : t.w;
            }
        } else {
#pragma unroll
            for (int i = 0; i < ANGLES; ++i) c[i] = s[i] = __builtin_nanf("");
        }
    }
    const int first = turns ? unit * N : a.rot + (unit - turned) * N;
    const T *x = static_cast<const T *>(a.x) + token * a.x_token + first;
    T *out = static_cast<T *>(a.out) + token * a.out_token + first;
    for (int head = split * at_once + in_step; head < a.heads; head += DEEP * splits * at_once) {
        V u[DEEP], v[DEEP];
#pragma unroll
        for (int k = 0; k < DEEP; ++k) {
            const int h = head + k * splits * at_once;
            if (h >= a.heads) break;
            u[k] = *reinterpret_cast<const V *>(x + h * a.x_head);
            if (!PAIRS && turns) v[k] = *reinterpret_cast<const V *>(x + h * a.x_head + pairs);
        }
#pragma unroll
        for (int k = 0; k < DEEP; ++k) {
            const int h = head + k * splits * at_once;
            if (h >= a.heads) break;
            if (turns) {
                float p[N], q[N];
                if (PAIRS) {
#pragma unroll
                    for (int e = 0; e < N; e += 2) {
                        p[e] = u[k].get(e) * c[e / 2] - u[k].get(e + 1) * s[e / 2];
                        p[e + 1] = u[k].get(e + 1) * c[e / 2] + u[k].get(e) * s[e / 2];
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < N; ++e) {
                        p[e] = u[k].get(e) * c[e % ANGLES] - v[k].get(e) * s[e % ANGLES];
                        q[e] = v[k].get(e) * c[e % ANGLES] + u[k].get(e) * s[e % ANGLES];
                    }
                    v[k].set(q);
                    *reinterpret_cast<V *>(out + h * a.out_head + pairs) = v[k];
                }
                u[k].set(p);
            }
            *reinterpret_cast<V *>(out + h * a.out_head) = u[k];
        }
    }
}

// Waves that share a token's heads: enough to fill the chip, as far as there are heads.
constexpr int64_t ROPE_WAVES = 256 * 16;

template <typename T>
hipError_t rope(const RopeArgs &a, hipStream_t st)
{
    constexpr int N = RopeVec<T>::N;
    const int per = a.pairs_layout ? a.rot : a.rot / 2, rest = a.x == a.out ? 0 : a.dim - a.rot;
    const int units = per / N + rest / N;
    if (per % N == 0 && rest % N == 0 && units <= 64) {
        const int steps = (a.heads + 64 / units - 1) / (64 / units);
        const int64_t wanted = (ROPE_WAVES + a.tokens - 1) / a.tokens;
        const int splits = wanted < steps ? (int)wanted : steps;
        const int64_t groups = (a.tokens * splits + 3) / 4;
        if (grid_fits(groups, 256)) {
            if (a.pairs_layout)
                hipLaunchKernelGGL((rope_kernel<T, true>), dim3((uint32_t)groups), dim3(256), 0, st, a, units, per / N, splits);
            else
                hipLaunchKernelGGL((rope_kernel<T, false>), dim3((uint32_t)groups), dim3(256), 0, st, a, units, per / N, splits);
            return hipGetLastError();
        }
    }
    const int64_t n = a.tokens * a.heads * (a.rot / 2 + rest), groups = (n + 255) / 256;
    hipLaunchKernelGGL(rope_any_kernel<T>, dim3((uint32_t)(groups < (1 << 20) ? groups : 1 << 20)), dim3(256), 0, st, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_rope_table(const RopeTableArgs &a, hipStream_t st)
{
    const int64_t groups = (a.positions + 3) / 4;
    hipLaunchKernelGGL(rope_table_kernel, dim3((uint32_t)(groups < 4096 ? groups : 4096), (a.rot / 2 + 63) / 64), dim3(256), 0, st, a);
    return hipGetLastError();
}

hipError_t launch_rope(const RopeArgs &a, hipStream_t st) { return a.fp32 ? rope<float>(a, st) : rope<uint16_t>(a, st); }

}  // namespace mxfp4
