// Orthogonalised updates: momentum, then Newton-Schulz products on the matrix cores.
//     M = mu M + G,  U = G + mu M (Nesterov), M, or G without momentum,  X = U / (|U| + eps)      (|.|: root of the sum of squares)
//     `steps` times:  A = X X^T,  Q = b A + c A A,  X = P X with P = a I + Q
// X is taken with fewer rows than columns (m <= n), so that A and Q are the small ones: G^T is worked on where G has more rows.
//
// Two and three steps in one, on request.  The matrix of the next step is known without its X: A' = P A P, and X'' = P' P X.  That takes three more products
// of m x m matrices (B = a A + A Q, A' = a B + Q B, T = P' P) and saves a product with X, its X X^T, and X's way to memory and back.  All m x m matrices
// are polynomials in A: symmetric, and half of each product is enough.  So five steps, taken as three and two, take 2 x 3 m^2 n + 14 m^3 operations, as single
// ones 5 x 3 m^2 n + 5 m^3: they are joined where X is so much wider than tall that this pays (joined_steps_pay).  A's small eigenvalues, from which the
// steps bring a direction up, lose accuracy in the rounding of its large ones (each step multiplies them by a^2; X X^T of the X that is really there does
// not drift): two and three steps lose some of it, which is why a caller has to ask for them, and longer runs would lose most.  Three only at the start,
// where the trace of A is 1: its rounding is 1.6e-4 / sqrt(m) at most there, against each eigenvalue that still has to grow.  The last two steps are joined
// rather than two before the last: a step behind may double what they leave.
//
// Types.  The products are of fp16 operands with fp32 sums; every operand has a fixed power of two as its scale, chosen so that the largest
// singular value that X may reach fits (checked on the host for the coefficients given) and fp16's 11 bits hold all the way down to elements 2^-28 of it.
// What the polynomial carries from step to step is kept more exactly than that: X as two fp16 words (hi + lo / 2048, 22 bits), of which the product takes
// the first and the term with P's diagonal both, and the diagonals of all m x m matrices apart in fp32 (the products see zeros there), where nearly all of a
// nearly orthogonal matrix's A and Q is.  Relative error of the result before its rounding to bf16 (1.7e-3 by itself), five steps, 512 rows and more, singular
// values 1 / i, 1 / i^2, exponential over nine decades, of noise, and of noise below sixteen directions or one: single steps 1e-4 to 9e-4, joined ones 3e-4 to
// 4e-3 (1024 x 4096 with 1 / i^2: 1.3e-4 and 1.6e-3, noise 3.0e-4 and 2.6e-4).  With X rounded to fp16 in every step 1.2e-3 to 2.4e-3, and 2.4e-2 where a few
// directions hold nearly all of the gradient: the small ones, which each step multiplies by a, drown in the rounding of the large ones.  With bf16 1e-2.
//
// Layout.  Rows and columns are padded with zeros to whole 64s in the workspace, which the products turn into zeros again; nothing in the products' loops is
// ragged.  X X^T and the m x m products take two operands whose rows lie along the contraction; in P X the second one's columns do, and its
// fragments come out of LDS by transposing reads.
#include "layer_ops.h"
#include "vector_io.h"

#include <type_traits>

namespace mxfp4 {
namespace {

typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef _Float16 v4h __attribute__((ext_vector_type(4)));
typedef short v4s __attribute__((ext_vector_type(4)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));

constexpr float SX = 16384.0f, SA = 16384.0f, SQ = 4096.0f, ST = 1024.0f, LO = 2048.0f;  // scales of X; of A, B; of Q, T; of three steps' T; of lo against hi

// What a matrix of the batch has in the workspace, and where.
struct OrthoLayout {
    int64_t m, n, mp, np;                     // mp, np: padded
    size_t xh[2], xlo, s[4], d[4];            // X's first words (read, written), its second ones; symmetric matrices, their diagonals
    size_t squares, sums, arrived, total;     // arrived: counters of the tiles of X X^T that are worked on in pieces
};
constexpr int SUM_GROUPS = 512;  // most partial sums of squares per matrix

OrthoLayout ortho_layout(int64_t N, int64_t K)
{
    OrthoLayout l;
    l.m = N < K ? N : K;
    l.n = N < K ? K : N;
    l.mp = (l.m + 63) / 64 * 64;
    l.np = (l.n + 63) / 64 * 64;
    size_t at = 0;
    const auto take = [&](size_t bytes) {
        const size_t here = at;
        at = (at + bytes + 255) / 256 * 256;
        return here;
    };
    const size_t x = (size_t)l.mp * l.np * 2, s = (size_t)l.mp * l.mp * 2;
    l.xh[0] = take(x);
    l.xh[1] = take(x);
    l.xlo = take(x);
    for (int i = 0; i < 3; ++i) l.s[i] = take(s);
    l.s[3] = l.xh[1];  // used before anything is written there
    for (int i = 0; i < 4; ++i) l.d[i] = take((size_t)l.mp * 4);
    l.squares = take((size_t)(l.np / 32) * l.mp * 4);  // [pieces of a row][mp]: sums of squares of X's rows, as its writers had them
    l.sums = take(SUM_GROUPS * 8);
    const int64_t blocks = l.mp / 64;
    l.arrived = take(blocks * (blocks + 1) / 2 * 4);
    l.total = at;
    return l;
}

// ---- momentum and the sum of squares --------------------------------------------------------------------------------------------

// The update that is orthogonalised, of eight elements; m: the momentum after this step.
template <typename G>
__device__ __forceinline__ void update_of(const Raw8<G> &g, const float (&m)[8], bool has, bool nesterov, float mu, float (&u)[8])
{
#pragma unroll
    for (int e = 0; e < 8; ++e) u[e] = !has ? g.get(e) : nesterov ? fmaf(mu, m[e], g.get(e)) : m[e];
}

// Squares are summed in fp64: gradients of any scale that fp32 holds neither vanish nor overflow.
template <typename G>
__global__ __launch_bounds__(256) void ortho_momentum_kernel(const OrthoArgs p, uint8_t *workspace, const OrthoLayout l, int counters)
{
    const int64_t matrix = blockIdx.y, vectors = (p.K + 7) / 8;
    if (blockIdx.x == 0)
        for (int i = threadIdx.x; i < counters; i += 256) reinterpret_cast<uint32_t *>(workspace + matrix * l.total + l.arrived)[i] = 0;
    const G *g = static_cast<const G *>(p.g) + matrix * p.g_matrix;
    float *mom = p.momentum ? p.momentum + matrix * p.N * p.K : nullptr;
    double s = 0.0;
    for (int64_t v = (int64_t)blockIdx.x * 256 + threadIdx.x; v < p.N * vectors; v += (int64_t)gridDim.x * 256) {
        const int64_t row = v / vectors, c = (v - row * vectors) * 8;
        const int n = (int)(p.K - c < 8 ? p.K - c : 8);
        Raw8<G> gv;
        gv.load(g + row * p.ld_g + c, n);
        float m[8] = {}, u[8];
        if (mom) {
            Raw8<float> mv;
            mv.load(mom + row * p.K + c, n);
#pragma unroll
            for (int e = 0; e < 8; ++e) m[e] = fmaf(p.mu, mv.get(e), gv.get(e));
            store8(mom + row * p.K + c, m, n);
        }
        update_of(gv, m, mom != nullptr, p.nesterov, p.mu, u);
#pragma unroll
        for (int e = 0; e < 8; ++e) s = fma((double)u[e], (double)u[e], s);
    }
    __shared__ double sums[4];
    for (int d = 1; d < 64; d <<= 1) s += __shfl_xor(s, d);
    if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x == 0)
        reinterpret_cast<double *>(workspace + matrix * l.total + l.sums)[blockIdx.x] = sums[0] + sums[1] + sums[2] + sums[3];
}

// ---- X = U / (|U| + eps) as fp16 words -------------------------------------------------------------------------------------------

// hi in the low half, lo in the high one
__device__ __forceinline__ uint32_t words_of(float x)
{
    const _Float16 hi = (_Float16)x, lo = (_Float16)((x - (float)hi) * LO);
    return __builtin_bit_cast(uint16_t, hi) | (uint32_t)__builtin_bit_cast(uint16_t, lo) << 16;
}

// A workgroup takes 64 x 64 elements of the padded X; where X is U^T they are turned in LDS.
template <typename G>
__global__ __launch_bounds__(256) void ortho_split_kernel(const OrthoArgs p, uint8_t *workspace, const OrthoLayout l, int sums)
{
    __shared__ float tile[64][65];
    __shared__ double part[4];
    const int64_t matrix = blockIdx.z;
    uint8_t *ws = workspace + matrix * l.total;
    {
        const double *all = reinterpret_cast<const double *>(ws + l.sums);
        double s = 0.0;
        for (int i = threadIdx.x; i < sums; i += 256) s += all[i];
        for (int d = 1; d < 64; d <<= 1) s += __shfl_xor(s, d);
        if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = s;
        __syncthreads();
    }
    const double scale = (double)SX / (sqrt(part[0] + part[1] + part[2] + part[3]) + (double)p.eps);  // (may be beyond fp32, where U is tiny)
    const bool flipped = p.N > p.K;
    const int64_t row0 = (int64_t)blockIdx.y * 64, col0 = (int64_t)blockIdx.x * 64;  // of U
    const G *g = static_cast<const G *>(p.g) + matrix * p.g_matrix;
    const float *mom = p.momentum ? p.momentum + matrix * p.N * p.K : nullptr;
    const int r = threadIdx.x >> 3, c = (threadIdx.x & 7) * 8;
    const bool momentum_alone = mom && !p.nesterov;  // is U: G is not read again (4096 x 14336 142 -> 90 us)
    const auto write = [&](const float (&x)[8], int64_t row, int64_t col, int piece) {  // of X; eight lanes have 64 elements of a row
        uint32_t w[8];
        float square = 0.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            w[e] = words_of(x[e]);
            square = fmaf(x[e], x[e], square);
        }
        uint4 hi, lo;
        uint32_t *ph = &hi.x, *pl = &lo.x;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            ph[e] = (w[2 * e] & 0xFFFF) | w[2 * e + 1] << 16;
            pl[e] = w[2 * e] >> 16 | (w[2 * e + 1] & 0xFFFF0000u);
        }
        const int64_t at = (row * l.np + col) * 2;
        *reinterpret_cast<uint4 *>(ws + l.xh[0] + at) = hi;
        *reinterpret_cast<uint4 *>(ws + l.xlo + at) = lo;
        for (int d = 1; d < 8; d <<= 1) square += __shfl_xor(square, d);
        if (c == 0) reinterpret_cast<float *>(ws + l.squares)[(int64_t)piece * l.mp + row] = square;
    };
#pragma unroll
    for (int half = 0; half < 64; half += 32) {
        const int64_t row = row0 + r + half;
        const int64_t left = row < p.N ? p.K - (col0 + c) : 0;
        const int n = (int)(left < 0 ? 0 : left < 8 ? left : 8);
        Raw8<G> gv;
        gv.load(g + row * p.ld_g + col0 + c, momentum_alone ? 0 : n);
        float m[8] = {}, u[8];
        if (mom) {
            Raw8<float> mv;
            mv.load(mom + row * p.K + col0 + c, n);
#pragma unroll
            for (int e = 0; e < 8; ++e) m[e] = mv.get(e);
        }
        update_of(gv, m, mom != nullptr, p.nesterov, p.mu, u);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            u[e] = e < n ? (float)(u[e] * scale) : 0.0f;
            if (flipped) tile[r + half][c + e] = u[e];
        }
        if (!flipped) write(u, row, col0 + c, blockIdx.x);
    }
    if (!flipped) return;
    __syncthreads();
#pragma unroll
    for (int half = 0; half < 64; half += 32) {
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = tile[c + e][r + half];
        write(x, col0 + r + half, row0 + c, blockIdx.y);
    }
}

// ---- the products ---------------------------------------------------------------------------------------------------------------

enum OrthoMode { GRAM = 0, SYMM = 1, APPLY = 2, LAST = 3 };  // A = X X^T; of two symmetric matrices; X = T X; the same, to the output

struct ProductArgs {
    uint8_t *workspace;
    OrthoLayout l;
    int from;                      // which of X's first words are read
    int stages;                    // of 64 along the contraction
    int pieces;                    // that the sums of squares of X's rows are in
    int blocks_u, blocks_v, tiles; // tiles of one matrix
    int tiles_all;                 // ... of the batch, and of all pieces
    int splits;                    // GRAM on the smallest tiles: pieces that the contraction is cut into
    uint8_t *partial;              // ... and their sums
    int p, r, to;                  // SYMM: to = cp p + cr r + cpr p r + one I; APPLY, LAST: p is T
    float p_scale, r_scale, to_scale, cp, cr, cpr, one;
    float p_unit;                  // APPLY, LAST: what a 1 in T stands for
    float out_scale;
    uint16_t *out;
    int64_t N, K, ld_out, out_matrix;
};

// Eight elements of the output's row, as far as it has them.
__device__ __forceinline__ void store_row(uint16_t *out, int64_t ld, int64_t rows, int64_t cols, int64_t row, int64_t col, const uint4 &t)
{
    if (row >= rows || col >= cols) return;
    uint16_t *here = out + row * ld + col;
    const Vec16 u = {{t.x, t.y, t.z, t.w}};
    if (col + 8 <= cols) {
        *reinterpret_cast<Vec16 *>(here) = u;
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (col + e < cols) here[e] = (uint16_t)(u.v[e >> 1] >> (16 * (e & 1)));
    }
}

// Each lane: 16 bytes from sbase + voff to LDS[lds + IMM + 16 * lane].  (One wait state between writing M0 and the load that reads it.)
template <int IMM>
__device__ __forceinline__ void dma16(uint32_t lds, uint32_t voff, const uint8_t *sbase)
{
    asm volatile("s_add_u32 m0, %0, %3\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(voff), "s"(sbase), "n"(IMM) : "memory", "scc");
}

// Of `things` spread evenly over `slots`: how many come before slot t.
constexpr int spread(int t, int things, int slots)
{
    const int k = (t * things + slots - 1) / slots;
    return k < things ? k : things;
}

// Vector memory operations issued behind the loads of strip t, when it is waited for: of `strips`, `depth` are loaded ahead, each with `loads`, and behind
// every strip's turn its stores follow the loads of the one that takes its place.  (Stores that a wave may skip are not counted:
// fewer are waited for then, never too few.)
constexpr int younger(int t, int strips, int depth, int loads, int stores)
{
    int n = 0;
    for (int k = t + 1; k < depth && k < strips; ++k) n += loads;
    for (int k = t < depth ? 0 : t - depth; k < t; ++k) n += (k + depth < strips && k + depth > t ? loads : 0) + stores;
    return n < 63 ? n : 63;
}
template <int N>
__device__ __forceinline__ void wait_loads()
{
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
// A loop whose counter is a constant in its body.
template <int I, int N, typename F>
__device__ __forceinline__ void unrolled(F &&f)
{
    if constexpr (I < N) {
        f(std::integral_constant<int, I>{});
        unrolled<I + 1, N>(f);
    }
}

template <bool FIRST, typename A, typename B>
__device__ __forceinline__ auto &either(A &a, B &b)
{
    if constexpr (FIRST)
        return a;
    else
        return b;
}

// A column of a triangle of tiles has tiles of all rows above it: bands of columns keep the 32 or so tiles that an XCD works on at a time nearly square.
constexpr int BAND = 6;

// A tile has TU x TV outputs, of rows u of the first operand and v of the second one.  Four waves (2 x 2) take 16 NU x 16 NV of them each, with
// V_MFMA_F32_16X16X32_F16, whose result has four consecutive u of one v in a lane: what lies along u in memory is written in whole rows.
// A stage is 64 elements (128 bytes, a cache line) of the contraction, brought to LDS without a way through registers; NBUF stages are on their way or
// in use.  Chunk c (16 bytes) of row r lies at place c ^ (r / 2 mod 8) of the row, so that 16 lanes of a fragment read touch every bank once, whether LDS
// takes lanes 0 .. 15 together or 0 .. 3, 12 .. 15, 20 .. 27 (c ^ r ^ (r / 8), which is free of conflicts in the first case only: 1 to 4 % slower).  A stage
// is two halves of one instruction's 32 elements; while one is multiplied, the fragments of the next are read, across the change of stage too: the one
// barrier of a stage stands between its halves, when all fragments of it are in registers, and behind it the loads of the stage NBUF further on may overwrite
// it.
// Where the first operand lies the other way (X in T X), a stage has 64 rows k of TU elements.  A transposing read takes 32 bytes from each of 16 rows;
// rows' 32-byte pieces are exchanged by x(k) so that these 16 touch every bank twice, which is the least for 512 bytes.
template <int NU, int NV, int NBUF>
struct Tile {
    static constexpr int TU = 32 * NU, TV = 32 * NV, STAGE = (TU + TV) * 128, LOADS = (TU + TV) / 32;
    // Outputs leave by way of LDS.  Strips of 16 v x 16 NU u of a wave, with what they are added to: DEPTH of them at a time.
    static constexpr int STRIP = 16 * 16 * NU * 2, DEPTH = NV < 3 ? NV : 3;  // (five or six: 1 to 2 % slower)
    static constexpr int TURN = (STRIP >> 9) % 4 == 0 ? 7 : 3;                      // 16-byte chunks of a strip's row v are exchanged by v & TURN
    static constexpr int PITCH = 16 * NV * 2 + 16, SLICE = 16 * NU * PITCH;         // a wave's outputs turned, rows along v
    static constexpr int MOST = 4 * SLICE > 8 * DEPTH * STRIP ? 4 * SLICE : 8 * DEPTH * STRIP;
    static constexpr int LDS = NBUF * STAGE > MOST ? NBUF * STAGE : MOST;
    static_assert(LDS <= 163840 && DEPTH >= 1, "LDS of a compute unit");
};

template <int NU, int NV, int NBUF, int MODE>
__global__ __launch_bounds__(256) void ortho_product_kernel(const ProductArgs p)
{
    using T = Tile<NU, NV, NBUF>;
    constexpr bool SYMMETRIC = MODE == GRAM || MODE == SYMM, ALONG = SYMMETRIC;  // ALONG: the first operand's rows lie along the contraction too
    __shared__ __attribute__((aligned(1024))) uint8_t smem[T::LDS];
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t *)smem;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l16 = lane & 15, lg = lane >> 4;

    // Workgroups go round robin over the 8 XCDs: each takes a run of neighbouring tiles, whose operands then meet in its L2.
    int id = blockIdx.x;
    {
        const int x = id & 7, per = p.tiles_all >> 3, rest = p.tiles_all & 7;
        id = x * per + (x < rest ? x : rest) + (id >> 3);
    }
    constexpr bool MAY_SPLIT = MODE == GRAM && NU == 2 && NV == 2;
    int piece = 0;
    if (MAY_SPLIT && p.splits > 1) {
        piece = __builtin_amdgcn_readfirstlane(id / (p.tiles_all / p.splits));
        id -= piece * (p.tiles_all / p.splits);
    }
    const int tile_of_all = id, matrix = __builtin_amdgcn_readfirstlane(id / p.tiles);
    id -= matrix * p.tiles;
    const int tile = id;
    int bu, bv;
    if (SYMMETRIC) {  // tiles on and to one side of the diagonal: bands of six columns, row by row, then the band's piece of the diagonal
        int first = 0;
        while ((first + BAND) * (first + BAND + 1) / 2 <= id) first += BAND;
        const int width = p.blocks_u - first < BAND ? p.blocks_u - first : BAND;
        int k = id - first * (first + 1) / 2;
        bv = k / width;
        bu = first + (k - bv * width);
        if (bv >= first) {
            k -= first * width;
            bu = 0;
            while ((bu + 1) * (bu + 2) / 2 <= k) ++bu;
            bv = first + k - bu * (bu + 1) / 2;
            bu += first;
        }
    } else {  // four rows of tiles at a time
        const int band = id / (4 * p.blocks_u), rows = p.blocks_v - 4 * band < 4 ? p.blocks_v - 4 * band : 4;
        const int k = id - band * 4 * p.blocks_u;
        bv = 4 * band + k % rows;
        bu = k / rows;
    }
    bu = __builtin_amdgcn_readfirstlane(bu);
    bv = __builtin_amdgcn_readfirstlane(bv);
    const int mp = (int)p.l.mp, np = (int)p.l.np;
    const int u0 = bu * T::TU, v0 = bv * T::TV, end_u = SYMMETRIC ? mp : np, end_v = mp;
    uint8_t *ws = p.workspace + matrix * p.l.total;
    const uint8_t *xh = ws + p.l.xh[p.from];
    const uint8_t *pu = MODE == SYMM ? ws + p.l.s[p.p] : xh, *pv = MODE == GRAM ? xh : ws + p.l.s[MODE == SYMM ? p.r : p.p];
    const uint32_t ld_u = (MODE == SYMM ? mp : np) * 2, ld_v = (MODE == GRAM ? np : mp) * 2;  // bytes
    pu += ALONG ? (int64_t)u0 * ld_u : (int64_t)u0 * 2;
    pv += (int64_t)v0 * ld_v;
    const int64_t step_u = ALONG ? 128 : 64 * (int64_t)ld_u;

    // This lane's part of a stage's loads.  What lies behind an operand's last row (or column) is that one again; such outputs are not stored.
    constexpr int ROW = T::TU * 2;  // bytes of a row k
    constexpr auto exchange = [](int k) { return ROW % 256 == 0 ? (k & 3) | (k >> 3 & 1) << 2 : (k >> 1 & 1) | (k >> 3 & 1) << 1; };
    // A wave loads NU groups (1 KB) of the first operand and NV of the second one.
    uint32_t voff[T::LOADS];
#pragma unroll
    for (int q = 0; q < T::LOADS; ++q) {
        const bool first = q < NU;
        const int g = first ? wave * NU + q : wave * NV + q - NU, r = lane >> 3;
        if (!ALONG && first) {
            const int at = (g * 64 + lane) * 16, k = at / ROW, piece = (at - k * ROW) >> 5;
            int u = (piece ^ exchange(k)) * 16 + (lane & 1) * 8;
            u = u < end_u - 8 - u0 ? u : end_u - 8 - u0;
            voff[q] = k * ld_u + u * 2;
        } else {
            int row = 8 * g + r;
            const int last = first ? end_u - 1 - u0 : end_v - 1 - v0;
            row = row < last ? row : last;
            voff[q] = row * (first ? ld_u : ld_v) + (((lane & 7) ^ (g & 1) << 2 ^ r >> 1) << 4);
        }
    }
    const uint32_t lds_u = lds0 + wave * NU * 1024, lds_v = lds0 + T::TU * 128 + wave * NV * 1024;
    // (pu, pv: the stage that is loaded next)
    const auto load = [&](auto which, uint32_t buf) __attribute__((always_inline)) {
        constexpr int q = decltype(which)::value;
        if constexpr (q < NU)
            dma16<q * 1024>(lds_u + buf, voff[q], pu);
        else
            dma16<(q - NU) * 1024>(lds_v + buf, voff[q], pv);
    };
    const auto next_stage = [&]() __attribute__((always_inline)) {
        pu += step_u;
        pv += 128;
    };

    const int wu = wave >> 1, wv = wave & 1;
    const auto along = [&](int row0, int kk, uint32_t buf) {  // 16 rows from row0 (whole 16s), 32 elements from 32 kk
        const int c = (kk * 4 + lg) ^ (l16 >> 1);
        return *reinterpret_cast<const v8h *>(smem + buf + row0 * 128 + l16 * 128 + c * 16);
    };
    uint32_t piece_at[NU];
#pragma unroll
    for (int t = 0; t < NU; ++t)
        piece_at[t] = lds0 + (8 * lg + (l16 >> 2)) * ROW + (((wu * NU + t) ^ exchange(8 * lg + (l16 >> 2))) << 5) + (l16 & 3) * 8;
    const auto across_k = [&](int t, int kk, uint32_t buf) {  // the same of 16 columns u: four rows k, and the next four
        typedef __attribute__((address_space(3))) v4s *Lds;
        const v4s a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(uintptr_t)(piece_at[t] + buf + kk * 32 * ROW));
        const v4s b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(uintptr_t)(piece_at[t] + buf + (kk * 32 + 4) * ROW));
        return __builtin_bit_cast(v8h, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
    };
    v8h fu[2][NU], fv[2][NV];
    const auto fragment = [&](int r, int set, uint32_t buf) {  // the r-th that a half needs
        if (r < NV)
            fv[set][r] = along(T::TU + wv * 16 * NV + 16 * r, set, buf);
        else if (ALONG)
            fu[set][r - NV] = along(wu * 16 * NU + 16 * (r - NV), set, buf);
        else
            fu[set][r - NV] = across_k(r - NV, set, buf);
    };

    int stages = p.stages;
    if (MAY_SPLIT && p.splits > 1) {
        const int each = p.stages / p.splits, longer = p.stages - each * p.splits;  // (the first ones have one more)
        const int first = __builtin_amdgcn_readfirstlane(piece * each + (piece < longer ? piece : longer));
        stages = __builtin_amdgcn_readfirstlane(each + (piece < longer));
        pu += first * step_u;
        pv += first * 128;
    }
#pragma unroll
    for (int s = 0; s < NBUF; ++s)
        if (s < stages) {
            unrolled<0, T::LOADS>([&](auto q) __attribute__((always_inline)) { load(q, s * T::STAGE); });
            next_stage();
        }

    // The diagonal of A is the sums of squares of X's rows, which were taken from both of its words: a thread has four rows of every fourth piece.
    v4f squares = {};
    const int sq_row = 4 * lane;
    if (MODE == GRAM && bu == bv && sq_row < T::TU && u0 + sq_row < mp) {
        const float *from = reinterpret_cast<const float *>(ws + p.l.squares) + u0 + sq_row;
#pragma unroll 8
        for (int k = wave; k < p.pieces; k += 4) squares += *reinterpret_cast<const v4f *>(from + (int64_t)k * mp);
    }

    v4f sums[NU][NV] = {};
    if (MODE != GRAM && stages >= NBUF)  // (the sums of squares are loads of their own)
        asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"((NBUF - 1) * T::LOADS) : "memory");
    else
        asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
#pragma unroll
    for (int r = 0; r < NU + NV; ++r) fragment(r, 0, 0);

    uint32_t cur = 0;
    // (one loop for all stages: with a second one for the last, without loads, the compiler moves sums from register to register in both)
    for (int left = stages; left > 0; --left) {
        const uint32_t nxt = cur + T::STAGE < NBUF * T::STAGE ? cur + T::STAGE : 0;
        const bool more = left > NBUF;
        unrolled<0, 2>([&](auto which) __attribute__((always_inline)) {
            constexpr int half = decltype(which)::value;
            if (half) {
                // all of this stage is in registers, of every wave behind the barrier, and the next one has arrived
                if (NBUF > 2 && left >= NBUF)
                    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((NBUF - 2) * T::LOADS) : "memory");
                else
                    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
            }
            constexpr int M = NU * NV, RUNS = T::LOADS > 4 ? 4 : 2;
            unrolled<0, M>([&](auto slot) __attribute__((always_inline)) {
                // in front of the t-th: fragment reads, over the first three quarters, and loads in a few runs
                constexpr int t = decltype(slot)::value;
#pragma unroll
                for (int r = spread(t, NU + NV, 3 * M / 4); r < spread(t + 1, NU + NV, 3 * M / 4); ++r) fragment(r, half ^ 1, half ? nxt : cur);
                if constexpr (half && spread(t, RUNS, M) < spread(t + 1, RUNS, M)) {
                    constexpr int run = spread(t, RUNS, M);
                    if (more)
                        unrolled<run * T::LOADS / RUNS, (run + 1) * T::LOADS / RUNS>([&](auto q) __attribute__((always_inline)) { load(q, cur); });
                }
                sums[t / NV][t % NV] = __builtin_amdgcn_mfma_f32_16x16x32_f16(fu[half][t / NV], fv[half][t % NV], sums[t / NV][t % NV], 0, 0, 0);
                __builtin_amdgcn_sched_barrier(0);
            });
        });
        next_stage();
        cur = nxt;
    }
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");

    // (apart, where they are changed once more before they are used: else the compiler moves the sums about in the loop, to where the code below wants
    // them, and that is a third slower)
    v4f apart[MAY_SPLIT ? NU : 1][MAY_SPLIT ? NV : 1];
    if constexpr (MAY_SPLIT)
#pragma unroll
        for (int t = 0; t < NU * NV; ++t) {
            apart[t / NV][t % NV] = sums[t / NV][t % NV];
            asm volatile("" : "+v"(apart[t / NV][t % NV]));
        }
    auto &acc = either<MAY_SPLIT>(apart, sums);
    if (MAY_SPLIT && p.splits > 1) {
        // Every piece writes its sums past the caches (agent scope: the XCDs' L2s are not coherent), waits until they are there, and counts itself; the last one
        // to do so reads them past the caches, adds them up in their order, and goes on.  Nobody waits for anybody.  Each word is coherent by itself, being an
        // atomic of agent scope on both sides; that the sums come before the count is not the language's memory model but gfx950's: such a store (SC1) is done, and
        // taken off vmcnt, when all XCDs can see it, every thread's are waited for in front of the barrier, and the count is behind that; the loads (SC1 too)
        // are issued when the count has come back.  The asm's memory clobbers keep the compiler to that order.  (With release and acquire in place of the wait every
        // piece writes back and empties its XCD's L2: 1024 x 4096 in three pieces 23 us where this took 17.)
        uint64_t *pieces = reinterpret_cast<uint64_t *>(p.partial) + ((int64_t)tile_of_all * p.splits * 256 + threadIdx.x) * 2;  // [16 x 16][tile][piece][thread][2]
        const int64_t next = 256 * 2;
#pragma unroll
        for (int t = 0; t < NU * NV; ++t)
#pragma unroll
            for (int e = 0; e < 2; ++e)
                __hip_atomic_store(pieces + ((int64_t)t * p.tiles_all + piece) * next + e,
                                   (uint64_t)__float_as_uint(acc[t / NV][t % NV][2 * e]) | (uint64_t)__float_as_uint(acc[t / NV][t % NV][2 * e + 1]) << 32,
                                   __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
        uint32_t *last = reinterpret_cast<uint32_t *>(smem);
        uint32_t *arrived = reinterpret_cast<uint32_t *>(ws + p.l.arrived) + tile;
        if (threadIdx.x == 0) {
            const uint32_t before = __hip_atomic_fetch_add(arrived, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            *last = before + 1 == (uint32_t)p.splits;
            if (before + 1 == (uint32_t)p.splits) *arrived = 0;  // for the next step's
        }
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        const bool mine = *last;
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        if (!mine) return;
#pragma unroll
        for (int t = 0; t < NU * NV; ++t) acc[t / NV][t % NV] = v4f{};
#pragma unroll 2
        for (int k = 0; k < p.splits; ++k) {
            uint64_t got[NU * NV][2];
#pragma unroll
            for (int t = 0; t < NU * NV; ++t)
#pragma unroll
                for (int e = 0; e < 2; ++e)
                    got[t][e] = __hip_atomic_load(pieces + ((int64_t)t * p.tiles_all + k) * next + e, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
#pragma unroll
            for (int t = 0; t < NU * NV; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[t / NV][t % NV][e] += __uint_as_float((uint32_t)(got[t][e >> 1] >> (32 * (e & 1))));
        }
    }
    // ---- outputs: a wave's strips of 16 v, rows along u, in the wave's own part of LDS ----
    // Strip t has two slots (hi and lo of X, or p and r) at ring + (t % DEPTH) * 2 * STRIP.
    constexpr int CHUNKS = 2 * NU, PER = NU / 2;  // 16-byte chunks of a row; a lane's chunks of a strip
    constexpr int ADDED = MODE == GRAM ? 0 : 2;   // matrices that outputs are made of beside the product
    const uint32_t ring = wave * (2 * T::DEPTH * T::STRIP);
    const int wave_u = u0 + wu * 16 * NU, wave_v = v0 + wv * 16 * NV;
    const uint8_t *added0 = MODE == SYMM ? ws + p.l.s[p.p] : xh, *added1 = MODE == SYMM ? ws + p.l.s[p.r] : ws + p.l.xlo;
    const int ld_out = SYMMETRIC ? mp : np;  // elements of a row of whatever is added and written (but the last output)
    const auto place = [&](int k, int &v, int &u) {  // of the lane's k-th chunk
        const int at = k * 64 + lane;
        v = at / CHUNKS;
        u = ((at - v * CHUNKS) ^ (v & T::TURN)) * 8;
    };
    const auto fetch = [&](int t) {
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            int v, u;
            place(k, v, u);
            v += wave_v + 16 * t;
            u += wave_u;
            v = v < end_v - 1 ? v : end_v - 1;
            u = u < end_u - 8 ? u : end_u - 8;
            const uint32_t at = ((uint32_t)(v - v0) * ld_out + (uint32_t)u) * 2;
            const int64_t base = (int64_t)v0 * ld_out * 2;
            const uint32_t slot = lds0 + ring + (t % T::DEPTH) * 2 * T::STRIP + k * 1024;
            dma16<0>(slot, at, added0 + base);
            dma16<T::STRIP>(slot, at, added1 + base);
        }
    };
    // (the diagonals first, and waited for: the compiler knows nothing of the loads above and would wait for all of them too)
    const float *dp = reinterpret_cast<const float *>(ws + p.l.d[p.p]), *dr = reinterpret_cast<const float *>(ws + p.l.d[p.r]);
    v4f dpu[NU];
    float dpv[NV], drv[NV];
    if (ADDED) {
#pragma unroll
        for (int t = 0; t < NV; ++t) {
            const int v = wave_v + 16 * t + l16;
            dpv[t] = v < mp ? dp[v] : 0.0f;
            if (MODE == SYMM) drv[t] = v < mp ? dr[v] : 0.0f;
        }
        if (MODE == SYMM)
#pragma unroll
            for (int t = 0; t < NU; ++t) {
                const int u = wave_u + 16 * t + 4 * lg;
                dpu[t] = u < mp ? *reinterpret_cast<const v4f *>(dp + u) : v4f{};
            }
#pragma unroll
        for (int t = 0; t < NV; ++t) {
            asm volatile("" : "+v"(dpv[t]));
            if (MODE == SYMM) asm volatile("" : "+v"(drv[t]));
        }
        if (MODE == SYMM)
#pragma unroll
            for (int t = 0; t < NU; ++t) asm volatile("" : "+v"(dpu[t]));
#pragma unroll
        for (int t = 0; t < T::DEPTH; ++t) fetch(t);
    }

    if (MODE == GRAM && bu == bv) {
        v4f *sums = reinterpret_cast<v4f *>(smem);
        sums[threadIdx.x] = squares;
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        if (wave == 0) {
            squares = (sums[lane] + sums[64 + lane]) + (sums[128 + lane] + sums[192 + lane]);
            squares *= 1.0f / (SX * SX);
            if (sq_row < T::TU && u0 + sq_row < mp) *reinterpret_cast<v4f *>(ws + p.l.d[p.to] + (size_t)(u0 + sq_row) * 4) = squares;
        }
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    }
    const bool turned = (SYMMETRIC && bu != bv) || (MODE == LAST && p.N > p.K);  // rows along v are written
    const bool straight = MODE != LAST || p.N <= p.K;                              // ... along u
    // The tile's rows as buffers: a store behind the last row or column gets an offset beyond them, and is dropped.
    constexpr int STORES = MODE == APPLY ? 2 * PER : PER;
    const int64_t rows_at = (int64_t)v0 * ld_out * 2;
    const uint32_t rows_bytes = (uint32_t)((end_v - v0 < T::TV ? end_v - v0 : T::TV) * (int64_t)ld_out * 2);
    // (so for the output too, if its rows are of whole 16 bytes at multiples of 4)
    const int64_t last_rows = p.N - v0 < T::TV ? p.N - v0 : T::TV;
    uint16_t *last_at = p.out + matrix * p.out_matrix + v0 * p.ld_out;
    const bool whole = MODE != LAST || (straight && p.K % 8 == 0 && p.ld_out % 2 == 0 && p.ld_out <= 1 << 22 && (reinterpret_cast<uintptr_t>(last_at) & 3) == 0 && last_rows > 0);
    const auto out0 = MODE == LAST ? __builtin_amdgcn_make_buffer_rsrc(last_at, 0, whole ? (uint32_t)(((last_rows - 1) * p.ld_out + p.K) * 2) : 0, 0x00020000)
                                   : __builtin_amdgcn_make_buffer_rsrc(ws + (MODE == APPLY ? p.l.xh[p.from ^ 1] : p.l.s[p.to]) + rows_at, 0, rows_bytes, 0x00020000);
    const auto out1 = __builtin_amdgcn_make_buffer_rsrc(ws + p.l.xlo + rows_at, 0, rows_bytes, 0x00020000);

    unrolled<0, NV>([&](auto strip) __attribute__((always_inline)) {
        constexpr int tv = decltype(strip)::value;
        if (ADDED) {
            // behind this strip's loads are those of later ones and the stores of earlier ones
            if (whole)
                wait_loads<younger(tv, NV, T::DEPTH, 2 * PER, STORES)>();
            else
                wait_loads<younger(tv, NV, T::DEPTH, 2 * PER, 0)>();
        }
        uint8_t *slot = smem + ring + (tv % T::DEPTH) * 2 * T::STRIP;
        const int v = wave_v + 16 * tv + l16;
        const bool real = wave_v + 16 * tv < end_v;  // whole 16s
        float square = 0.0f;
#pragma unroll
        for (int tu = 0; tu < NU; ++tu) {
            const int u = wave_u + 16 * tu + 4 * lg;
            uint8_t *here = slot + (l16 * CHUNKS + ((2 * tu + (lg >> 1)) ^ (l16 & T::TURN))) * 16 + (lg & 1) * 8;
            v4f x = acc[tu][tv];
            v4h first;
            if (MODE == GRAM) {
#pragma unroll
                for (int e = 0; e < 4; ++e) first[e] = (_Float16)(u + e == v ? 0.0f : x[e] * (SA / (SX * SX)));
            } else if (MODE == SYMM) {
                // (p r)_uv of p and r whose diagonals are apart: of the rest, p_u r_uv and p_uv r_v with one of them on the diagonal, and both.
                // Only their sum is symmetric (p and r commute, their rests do not).
                const v4h p4 = *reinterpret_cast<const v4h *>(here), r4 = *reinterpret_cast<const v4h *>(here + T::STRIP);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float product = x[e] * (p.cpr / (p.p_scale * p.r_scale));
                    const float fp = fmaf(p.cpr, drv[tv], p.cp), fr = fmaf(p.cpr, dpu[tu][e], p.cr);
                    const float y = fmaf(fp, (float)p4[e] * (1.0f / p.p_scale), fmaf(fr, (float)r4[e] * (1.0f / p.r_scale), product));
                    if (u + e == v && real)
                        reinterpret_cast<float *>(ws + p.l.d[p.to])[v] = p.one + p.cp * dpv[tv] + p.cr * drv[tv] + fmaf(p.cpr * dpv[tv], drv[tv], product);
                    first[e] = (_Float16)(u + e == v ? 0.0f : y * p.to_scale);
                }
            } else {
                const v4h hi = *reinterpret_cast<const v4h *>(here), lo = *reinterpret_cast<const v4h *>(here + T::STRIP);
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = fmaf(dpv[tv], fmaf((float)lo[e], 1.0f / LO, (float)hi[e]), x[e] * p.p_unit);
                if (MODE == APPLY) {
                    v4h rest;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        if (u < end_u) square = fmaf(x[e], x[e], square);
                        first[e] = (_Float16)x[e];
                        rest[e] = (_Float16)((x[e] - (float)first[e]) * LO);
                    }
                    *reinterpret_cast<v4h *>(here + T::STRIP) = rest;
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e) first[e] = __builtin_bit_cast(_Float16, bf16_bits(x[e] * (p.out_scale / SX)));
                }
            }
            *reinterpret_cast<v4h *>(here) = first;
            const uint2 words = __builtin_bit_cast(uint2, first);  // kept for the rows along v
            acc[tu][tv][0] = __uint_as_float(words.x);
            acc[tu][tv][1] = __uint_as_float(words.y);
        }
        if (MODE == APPLY) {
            square += __shfl_xor(square, 16);
            square += __shfl_xor(square, 32);
            if (lg == 0 && real) reinterpret_cast<float *>(ws + p.l.squares)[(int64_t)(2 * bu + wu) * mp + v] = square;
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // (a wave's own strip: no barrier)
        if (straight) {
            uint4 rows[PER], rest[PER];
#pragma unroll
            for (int k = 0; k < PER; ++k) {
                rows[k] = *reinterpret_cast<const uint4 *>(slot + (k * 64 + lane) * 16);
                if (MODE == APPLY) rest[k] = *reinterpret_cast<const uint4 *>(slot + T::STRIP + (k * 64 + lane) * 16);
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            if (ADDED && tv + T::DEPTH < NV) fetch(tv + T::DEPTH);
#pragma unroll
            for (int k = 0; k < PER; ++k) {
                int rv, ru;
                place(k, rv, ru);
                rv += wave_v + 16 * tv;
                ru += wave_u;
                if (MODE == LAST && !whole) {
                    store_row(p.out + matrix * p.out_matrix, p.ld_out, p.N, p.K, rv, ru, rows[k]);
                } else {
                    const uint32_t ld = MODE == LAST ? (uint32_t)p.ld_out : ld_out;
                    const uint32_t at = ru < (MODE == LAST ? p.K : end_u) && rv < (MODE == LAST ? p.N : end_v) ? ((uint32_t)(rv - v0) * ld + ru) * 2 : 0xFFFFFFF0u;
                    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(v4u, rows[k]), out0, at, 0, 0);
                    if (MODE == APPLY) __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(v4u, rest[k]), out1, at, 0, 0);
                }
            }
        } else if (ADDED && tv + T::DEPTH < NV) {
            fetch(tv + T::DEPTH);
        }
    });
    if (!turned) return;

    // ---- the same outputs in rows along v ----
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");  // other waves' strips may lie in this one's part
    uint8_t *slice = smem + wave * T::SLICE;
#pragma unroll
    for (int tu = 0; tu < NU; ++tu)
#pragma unroll
        for (int tv = 0; tv < NV; ++tv)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                *reinterpret_cast<uint16_t *>(slice + (16 * tu + 4 * lg + e) * T::PITCH + (16 * tv + l16) * 2) =
                    (uint16_t)(__float_as_uint(acc[tu][tv][e >> 1]) >> (16 * (e & 1)));
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
    for (int k = 0; k < NU * NV / 2; ++k) {
        const int chunk = k * 64 + lane, r = chunk / (2 * NV), c = (chunk - r * 2 * NV) * 8;
        const int u = wave_u + r, v = wave_v + c;
        const uint4 t = *reinterpret_cast<const uint4 *>(slice + r * T::PITCH + c * 2);
        if (MODE == LAST)
            store_row(p.out + matrix * p.out_matrix, p.ld_out, p.N, p.K, u, v, t);
        else if (u < end_u && v < end_v)
            *reinterpret_cast<uint4 *>(ws + p.l.s[p.to] + ((int64_t)u * mp + v) * 2) = t;
    }
}

// X X^T on the smallest tiles: a few tiles leave most compute units idle, so that the long contraction is cut into pieces, whose sums the last
// one to finish adds up (us: tiles' chains as below; 1.5 for writing and counting, 0.2 for each piece that is read, 0.004 for each one written).  In
// calls, whole and in pieces: 64 x 14336 57 us and 20 in twelve; 300 x 5000 24 and 15 in eight; 512 x 4096 19 and 13 in four; 1024 x 4096 19 and 16 in three.
struct Pieces {
    int splits;
    double us;
};
Pieces gram_pieces(const OrthoLayout &l, int64_t batch)
{
    const int64_t blocks = l.mp / 64, tiles = batch * (blocks * (blocks + 1) / 2), stages = l.np / 64;
    Pieces best{1, 0};
    for (int s = 1; s <= 16 && (s == 1 || 4 * s <= stages); ++s) {
        const int64_t share = (tiles * s + 255) / 256;
        const double work = 0.2 * (double)share, chain = work > 0.23 ? work : 0.23;
        const double us = (double)((stages + s - 1) / s) * chain + 5.0 * (double)((share + 2) / 3) + (s > 1 ? 1.5 + 0.2 * s + 0.004 * (double)(tiles * s) : 0.0);
        if (s == 1 || us < 0.95 * best.us) best = {s, us};
    }
    return best;
}
size_t pieces_bytes(const OrthoLayout &l, int64_t batch)
{
    const int splits = gram_pieces(l, batch).splits;
    const int64_t blocks = l.mp / 64;
    return splits > 1 ? (size_t)(batch * (blocks * (blocks + 1) / 2) * splits) * 64 * 64 * 4 : 0;
}

template <int NU, int NV, int NBUF, int MODE>
hipError_t product(ProductArgs &p, int64_t batch, hipStream_t st)
{
    using T = Tile<NU, NV, NBUF>;
    constexpr bool symmetric = MODE == GRAM || MODE == SYMM;
    p.blocks_v = (int)((p.l.mp + T::TV - 1) / T::TV);
    p.blocks_u = symmetric ? p.blocks_v : (int)((p.l.np + T::TU - 1) / T::TU);
    p.tiles = symmetric ? p.blocks_v * (p.blocks_v + 1) / 2 : p.blocks_u * p.blocks_v;
    p.splits = MODE == GRAM && NU == 2 ? gram_pieces(p.l, batch).splits : 1;
    p.tiles_all = (int)(p.tiles * batch * p.splits);
    p.stages = (int)((MODE == GRAM ? p.l.np : p.l.mp) / 64);
    hipLaunchKernelGGL((ortho_product_kernel<NU, NV, NBUF, MODE>), dim3(p.tiles_all), dim3(256), 0, st, p);
    if (MODE == APPLY) {
        p.pieces = 2 * p.blocks_u;
        p.from ^= 1;
    }
    return hipGetLastError();
}

// Tiles of a product: those with the lowest estimate.  A compute unit that R tiles fall to takes a tile's start and end (`fixed`) and `stage` for each of its
// stages, one tile after the other where one fills it; small tiles share it, `per_cu` of them, and a single one is bound by the chain through its
// stages (`alone`).  Measured in calls (us, P X of m x n unless named): 4096 x 14336 256 x 256 and 192 x 256 tiles 460, 192 x 192 519, 128 x 128 487; 4096 x
// 6144 183 with 192 x 256, 196 with 128 x 128, 211 with 192 x 192, 226 with 256 x 256; 4096 x 4096 129 with 256 x 256, 138 with 128 x 128; 1440 x 4320 28 with
// 128 x 128, 38 with 64 x 64; X X^T there 28 with 64 x 64, 44 with 128 x 128, of 4096 x 6144 98 with 192 x 192, 149 with 128 x 128; A A of 4096 74 with
// 192 x 192, 103 with 128 x 128, of 1024 8.2 with 64 x 64, 17 with 128 x 128.  The constants are fitted to kernels launched by themselves on the same operands over and
// over, which take up to a quarter less; the tiles they choose are the fastest, or within 2 % of them, in calls too.
// What bounds the loop: by itself P X of 4096 x 6144 takes 154 us, its matrix instructions alone 117, with fragment reads 135, its loads alone 114: a compute
// unit gets 60 to 78 bytes a ns out of L2 here, whatever the tile, which is what small tiles are bound by.  A tile of 192 x 192 keeps LDS as busy as the
// matrix unit (1125 of 1152 clocks a stage), one of 256 x 256 three quarters of that.
struct Choice {
    int shape;
    double us;
};
constexpr int ORTHO_SHAPES = 5;
template <int MODE>
Choice choose(const OrthoLayout &l, int64_t batch)
{
    constexpr bool symmetric = MODE == GRAM || MODE == SYMM;
    const double stages = (double)(MODE == GRAM ? l.np : l.mp) / 64;
    struct Shape {
        int nu, nv, per_cu;
        double stage, alone, fixed;  // us
    };
    static const Shape shapes[ORTHO_SHAPES] = {{8, 8, 1, 1.38, 1.38, 10}, {6, 8, 1, 1.15, 1.15, 7}, {6, 6, 1, 0.93, 0.93, 10}, {4, 4, 2, 0.43, 0.6, 7},
                                               {2, 2, 3, 0.2, 0.23, 5}};
    Choice best{-1, 0};
    for (int i = symmetric ? 2 : 0; i < ORTHO_SHAPES; ++i) {
        const Shape &s = shapes[i];
        const int64_t bv = (l.mp + 32 * s.nv - 1) / (32 * s.nv), bu = (l.np + 32 * s.nu - 1) / (32 * s.nu);
        const int64_t tiles = batch * (symmetric ? bv * (bv + 1) / 2 : bu * bv), share = (tiles + 255) / 256;
        const double work = (double)share * s.stage;
        double us = stages * (work > s.alone ? work : s.alone) + (double)((share + s.per_cu - 1) / s.per_cu) * s.fixed;
        if (MODE == GRAM && s.nu == 2) us = gram_pieces(l, batch).us;
        if (best.shape < 0 || us < best.us) best = {i, us};
    }
    return best;
}

template <int MODE>
hipError_t product(ProductArgs &p, int64_t batch, hipStream_t st)
{
    const int shape = choose<MODE>(p.l, batch).shape;
    if constexpr (MODE == APPLY || MODE == LAST) {
        if (shape == 0) return product<8, 8, 2, MODE>(p, batch, st);
        if (shape == 1) return product<6, 8, 2, MODE>(p, batch, st);
    }
    if (shape == 2) return product<6, 6, 2, MODE>(p, batch, st);
    if (shape == 3) return product<4, 4, 2, MODE>(p, batch, st);
    return product<2, 2, 3, MODE>(p, batch, st);
}

// Joined steps, where they are asked for, lose most accuracy where a matrix is small (a single eigenvalue's error is not lost among many; 3 x 5: up to 1.6e-2),
// and gain nothing there: launches are what small matrices take.  Above, where the products with X that they save take longer than the three of m x m ones that
// each adds, and a launch.  Five steps, single and as three and two (us): 4096 x 14336 4045 and 2665; 6144 x 4096 1900 and 1724; 4320 x 1440 364 and 319; 1024 x
// 4096 223 and 209; 600 x 8000 226 and 185; but 2048 x 3000 459 and 473, 1024 x 1536 163 and 180, 512 x 2048 130 and 133.
constexpr int64_t JOINED_FROM = 512;
bool joined_steps_pay(const OrthoLayout &l, int64_t batch)
{
    return l.m >= JOINED_FROM && choose<GRAM>(l, batch).us + choose<APPLY>(l, batch).us > 3 * choose<SYMM>(l, batch).us + 1.3;
}

// to = cp p + cr r + cpr p r + one I
hipError_t symmetric(ProductArgs &p, int64_t batch, hipStream_t st, int a, float a_scale, int b, float b_scale, int to, float to_scale, float cp,
                     float cr, float cpr, float one)
{
    p.p = a;
    p.r = b;
    p.to = to;
    p.p_scale = a_scale;
    p.r_scale = b_scale;
    p.to_scale = to_scale;
    p.cp = cp;
    p.cr = cr;
    p.cpr = cpr;
    p.one = one;
    return product<SYMM>(p, batch, st);
}

}  // namespace

size_t ortho_workspace_bytes(int64_t batch, int64_t N, int64_t K)
{
    const OrthoLayout l = ortho_layout(N, K);
    return (size_t)batch * l.total + pieces_bytes(l, batch);
}

hipError_t launch_orthogonalize(const OrthoArgs &a, hipStream_t st)
{
    const OrthoLayout l = ortho_layout(a.N, a.K);
    const int64_t vectors = a.N * ((a.K + 7) / 8), groups = (vectors + 255) / 256;
    const int sums = (int)(groups < SUM_GROUPS ? groups : SUM_GROUPS);
    const int64_t blocks = l.mp / 64;
    const int counters = gram_pieces(l, a.batch).splits > 1 ? (int)(blocks * (blocks + 1) / 2) : 0;
    const dim3 split((uint32_t)((a.K + 63) / 64), (uint32_t)((a.N + 63) / 64), (uint32_t)a.batch);
    if (a.g_fp32) {
        hipLaunchKernelGGL(ortho_momentum_kernel<float>, dim3(sums, (uint32_t)a.batch), dim3(256), 0, st, a, a.workspace, l, counters);
        hipLaunchKernelGGL(ortho_split_kernel<float>, split, dim3(256), 0, st, a, a.workspace, l, sums);
    } else {
        hipLaunchKernelGGL(ortho_momentum_kernel<uint16_t>, dim3(sums, (uint32_t)a.batch), dim3(256), 0, st, a, a.workspace, l, counters);
        hipLaunchKernelGGL(ortho_split_kernel<uint16_t>, split, dim3(256), 0, st, a, a.workspace, l, sums);
    }
    hipError_t e = hipGetLastError();
    ProductArgs p{};
    p.workspace = a.workspace;
    p.partial = a.workspace + (size_t)a.batch * l.total;
    p.l = l;
    p.out_scale = a.out_scale;
    p.out = static_cast<uint16_t *>(a.out);
    p.N = a.N;
    p.K = a.K;
    p.ld_out = a.ld_out;
    p.out_matrix = a.out_matrix;
    p.pieces = (int)(l.np / 64);
    const bool joined = a.joined && joined_steps_pay(l, a.batch);
    enum { S0, S1, S2, S3 };
    for (int step = 0; step < a.steps && e == hipSuccess;) {
        const int left = a.steps - step, run = !joined || left == 1 ? 1 : left % 2 ? 3 : 2;  // three of an odd number, the first
        p.to = S0;
        if ((e = product<GRAM>(p, a.batch, st)) != hipSuccess) break;                                                     // S0 = A
        if ((e = symmetric(p, a.batch, st, S0, SA, S0, SA, S1, SQ, a.b, 0, a.c, run > 1 ? 0.0f : a.a)) != hipSuccess) break;  // S1 = Q, or P
        int product_of_all = S1;
        if (run > 1) {
            if ((e = symmetric(p, a.batch, st, S0, SA, S1, SQ, S2, SA, a.a, 0, 1, 0)) != hipSuccess) break;               // S2 = B = P A
            if ((e = symmetric(p, a.batch, st, S1, SQ, S2, SA, S0, SA, 0, a.a, 1, 0)) != hipSuccess) break;               // S0 = A' = P B
            if ((e = symmetric(p, a.batch, st, S0, SA, S0, SA, S2, SQ, a.b, 0, a.c, 0)) != hipSuccess) break;             // S2 = Q'
            product_of_all = run > 2 ? S3 : S0;
            if ((e = symmetric(p, a.batch, st, S1, SQ, S2, SQ, product_of_all, SQ, a.a, a.a, 1, a.a * a.a)) != hipSuccess) break;  // T = P' P
        }
        if (run > 2) {
            if ((e = symmetric(p, a.batch, st, S0, SA, S2, SQ, S1, SA, a.a, 0, 1, 0)) != hipSuccess) break;               // S1 = B' = P' A'
            if ((e = symmetric(p, a.batch, st, S2, SQ, S1, SA, S0, SA, 0, a.a, 1, 0)) != hipSuccess) break;               // S0 = A'' = P' B'
            if ((e = symmetric(p, a.batch, st, S0, SA, S0, SA, S2, SQ, a.b, 0, a.c, 0)) != hipSuccess) break;             // S2 = Q''
            if ((e = symmetric(p, a.batch, st, S2, SQ, S3, SQ, S0, ST, 0, a.a, 1, 0)) != hipSuccess) break;               // S0 = P'' T
            product_of_all = S0;
        }
        p.p = product_of_all;
        p.p_unit = 1.0f / (run > 2 ? ST : SQ);
        step += run;
        e = step < a.steps ? product<APPLY>(p, a.batch, st) : product<LAST>(p, a.batch, st);
    }
    return e;
}

}  // namespace mxfp4
