// Orthogonalised updates of weight matrices (Newton-Schulz products) and the optimiser step around them: rg_orthogonalize, rg_muon_step.
//
// With n the narrower side and m the wider one a step is A = X X^T (n x n, symmetric), P = b A + c A^2 (symmetric) and
// X <- a X + P X: n(n+1)m + n(n+1)n + 2 n^2 m operations, of which the symmetric products compute one half and write the other by
// reflection.  Large matrices are bound by the matrix cores, small ones by the launches.
//
// Precision.  A rounding of X itself is noise in the directions of X's small singular values, which every step
// multiplies by 3.4; a rounding of P only tilts the directions that are there.  So the state X is kept in fp32 and a X is added from it, and
// only the operands of the products are 16 bits: fp16, scaled by 2^14, since nothing here is four or more (singular values stay below
// 1.21, A's entries below 1.46, P's below 2.9).  A update of rank 8 with 16-bit products comes out 4e-4 off so (relative, 2-norm), 2e-2 with X in fp16,
// 3e-1 with X in bf16.  For fp32 matrices an operand is the sum of two fp16 numbers, 22 bits, and a product is three: 4e-7 to 6e-6 off, as fp32 products are.
// So it is for matrices of 16 bits whose narrower side is 32 or less: over so few singular values the roundings do not average out
// (up to 9e-3 off with 2 rows, 2e-3 with 32), and their products cost nothing beside the launches.
//
// The division by the norm is exact: X starts as G 2^-e with a norm in [1/2, 1), and the factor f = 2^e / (|G| + eps) that is left
// goes into the first step's coefficients: P = b f^2 A + c f^4 A^2, X <- f (a X + P X).
//
// Every operand is kept with the axis that a product runs along contiguous: X and its transpose both, in blocks padded by zeros
// to whole tiles, so that no product checks a bound.
#include "rg_internal.h"
#include "rg_elements.h"
#include "rg_launch.h"

#include <cmath>

namespace rg {

namespace {

constexpr float NS_A = 3.4445f, NS_B = -4.7750f, NS_C = 2.0315f;
constexpr float SCALE = 16384.f, UNSCALE = 1.f / 16384.f;             // of the fp16 operands
constexpr int SUM_BLOCKS = 256;                                       // partial sums of squares of a matrix, at most

typedef f16 f16x8 __attribute__((ext_vector_type(8)));
typedef f16 f16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

// An operand: the fp16 numbers nearest to its values, and (fp32 matrices) those nearest to what they leave.
struct Operand { f16 *hi, *lo; };

struct Matrix {
    rg_update u;
    int32_t n, m, n_pad, m_pad;          // narrower and wider side, and padded
    bool tall;                           // rows > cols: X is the transpose
    uint32_t sum_blocks, sum_first;      // workgroups of the first pass
    uint32_t tile_first;                 // of the second
    uint32_t half_first, whole_first;    // tiles in front of this matrix' in products whose result is symmetric, and in others
    double *sums;                        // [sum_blocks]
    float *factor;                       // f
    float *x;                            // [n_pad][m_pad]
    Operand xr, xt[2];                   // X's rows [n_pad][m_pad], its columns [m_pad][n_pad] before and after a step
    Operand a, p;                        // [n_pad][n_pad]
};

struct Group {
    Matrix mat[RG_UPDATES_PER_LAUNCH];
    uint32_t count;
    bool muon, nesterov;
    float momentum, lr, keep;            // keep = 1 - lr * weight_decay
    float eps;
};

static_assert(sizeof(Group) <= 4000, "kernel arguments are 4 KB at most");

// The matrix that workgroup (or tile) t belongs to, counted by FIRST.
template <uint32_t Matrix::*FIRST> __device__ __forceinline__ uint32_t matrix_of(const Group &g, uint32_t t)
{
    uint32_t k = 0;
    while (k + 1 < g.count && t >= g.mat[k + 1].*FIRST) ++k;
    return k;
}

template <typename T> __device__ __forceinline__ const T *row_at(const void *p, uint64_t stride, int64_t r) { return reinterpret_cast<const T *>(static_cast<const uint8_t *>(p) + (uint64_t)r * stride); }
template <typename T> __device__ __forceinline__ T *row_at(void *p, uint64_t stride, int64_t r) { return reinterpret_cast<T *>(static_cast<uint8_t *>(p) + (uint64_t)r * stride); }

// ---------------------------------------------------------------- momentum, sum of squares
template <typename T>
__global__ void __launch_bounds__(256) update_sums_kernel(Group g)
{
    const Matrix &m = g.mat[matrix_of<&Matrix::sum_first>(g, blockIdx.x)];
    const uint32_t block = blockIdx.x - m.sum_first;
    uint32_t tx = 256;
    while (tx > 1 && tx / 2 >= m.u.cols) tx /= 2;                       // threads along a row
    const uint32_t ty = 256 / tx;
    double s = 0.0;
    for (uint32_t r = block * ty + threadIdx.x / tx; r < m.u.rows; r += m.sum_blocks * ty) {
        const T *grad = row_at<T>(m.u.grad, m.u.grad_stride, r);
        const float *mom = row_at<float>(m.u.momentum, m.u.momentum_stride, r);
        float *mom_out = row_at<float>(m.u.momentum_out, m.u.momentum_out_stride, r);
        for (uint32_t c = threadIdx.x % tx; c < m.u.cols; c += tx) {
            float v = (float)grad[c];
            if (g.muon) {
                const float next = g.momentum * mom[c] + v;
                mom_out[c] = next;
                v = g.nesterov ? v + g.momentum * next : next;
            }
            s += (double)v * (double)v;
        }
    }
    __shared__ double part[4];
    for (int k = 1; k < 64; k <<= 1) s += __shfl_xor(s, k);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x == 0) m.sums[block] = part[0] + part[1] + part[2] + part[3];
}

// ---------------------------------------------------------------- X in the layouts of the products
__device__ __forceinline__ void put(const Operand &o, uint64_t at, float v, bool split)
{
    const f16 h = (f16)v;
    o.hi[at] = h;
    if (split) o.lo[at] = (f16)(v - (float)h);
}

// A workgroup takes 64 x 64 elements of the padded X.
template <typename T, bool SPLIT>
__global__ void __launch_bounds__(256) update_start_kernel(Group g)
{
    const Matrix &m = g.mat[matrix_of<&Matrix::tile_first>(g, blockIdx.x)];
    const uint32_t tile = blockIdx.x - m.tile_first;
    __shared__ double part[4];
    __shared__ float block[64][65];
    double s = threadIdx.x < m.sum_blocks ? m.sums[threadIdx.x] : 0.0;
    for (int k = 1; k < 64; k <<= 1) s += __shfl_xor(s, k);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = s;
    __syncthreads();
    const double norm = sqrt(part[0] + part[1] + part[2] + part[3]);
    int e = 0;
    if (norm > 0.0 && norm < INFINITY) (void)frexp(norm, &e);
    if (tile == 0 && threadIdx.x == 0) {
        const double f = ldexp(1.0, e) / (norm + (double)g.eps);
        *m.factor = norm == 0.0 && g.eps > 0.f ? 0.f : norm < INFINITY ? (float)f : NAN;
    }
    const int32_t across = m.m_pad / 64;
    const int32_t i0 = (int32_t)(tile / across) * 64, j0 = (int32_t)(tile % across) * 64;
    const int32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    // G is read along its rows: along X's rows, or, where X is G's transpose, along its columns
    for (int32_t k = wave; k < 64; k += 4) {
        const int32_t r = (m.tall ? j0 : i0) + k, c = (m.tall ? i0 : j0) + lane;
        float v = 0.f;
        if (r < (int32_t)m.u.rows && c < (int32_t)m.u.cols) {
            v = (float)row_at<T>(m.u.grad, m.u.grad_stride, r)[c];
            if (g.muon) {
                const float next = row_at<float>(m.u.momentum_out, m.u.momentum_out_stride, r)[c];
                v = g.nesterov ? v + g.momentum * next : next;
            }
            v = ldexpf(v, -e);
        }
        if (m.tall) block[lane][k] = v; else block[k][lane] = v;
    }
    __syncthreads();
    for (int32_t k = wave; k < 64; k += 4) {
        const uint64_t row = (uint64_t)(i0 + k) * m.m_pad + j0 + lane, column = (uint64_t)(j0 + k) * m.n_pad + i0 + lane;
        const float v = block[k][lane];
        m.x[row] = v;
        put(m.xr, row, v * SCALE, SPLIT);
        put(m.xt[0], column, block[lane][k] * SCALE, SPLIT);
    }
}

// ---------------------------------------------------------------- products
// C = L R^T of a tile of TILE x TILE by four waves: both operands run along K contiguously, K a multiple of 64.  Steps of DEPTH along K pass through LDS,
// two of them there: one is multiplied while the other arrives, written into LDS by the loads themselves.  A row of a step is 16-byte chunks,
// stored in an order that depends on the row, so that the lanes of a read (32 rows, one chunk of each) spread over the banks.
template <int TILE, bool SPLIT>
struct Product {
    static constexpr int DEPTH = SPLIT ? 32 : 64;
    static constexpr int CHUNKS = DEPTH / 8;
    static constexpr int PARTS = SPLIT ? 2 : 1;
    static constexpr int PART = TILE * DEPTH;                    // elements of one part of one operand's step
    static constexpr int STAGE = 2 * PARTS * PART;
    static constexpr int LDS_BYTES = 2 * STAGE * 2;
    static constexpr int BLOCKS = TILE / 64;                     // blocks of 32 x 32 of a wave, either way
    static constexpr int LOADS = TILE * CHUNKS / 256;            // of a thread, to a part
    static_assert(TILE * CHUNKS % 256 == 0, "");

    static __device__ __forceinline__ int slot_of(int row, int chunk) { return chunk ^ ((DEPTH == 64 ? row >> 1 : row >> 2) & (CHUNKS - 1)); }

    static __device__ __forceinline__ void load(const f16 *const (&src)[2 * PARTS], uint64_t ld, int32_t k0, f16 *stage)
    {
#pragma unroll
        for (int p = 0; p < 2 * PARTS; ++p)
#pragma unroll
            for (int i = 0; i < LOADS; ++i) {
                const int q = i * 256 + (int)threadIdx.x, row = q / CHUNKS, chunk = slot_of(row, q % CHUNKS);
                const f16 *from = src[p] + (uint64_t)row * ld + k0 + chunk * 8;
                f16 *to = stage + p * PART + (i * 256 + (int)(threadIdx.x & ~63u)) * 8;
                __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)from, (__attribute__((address_space(3))) void *)to, 16, 0, 0);
            }
    }

    static __device__ __forceinline__ f16x8 fragment(const f16 *part, int row, int chunk) { return *reinterpret_cast<const f16x8 *>(part + row * DEPTH + slot_of(row, chunk) * 8); }

    // Every load into LDS of this wave has arrived, and then of every wave.  (A barrier by itself waits for LDS operations, not for
    // loads from global memory; the builtin's bits leave the other counters alone.)
    static __device__ __forceinline__ void arrive()
    {
        __builtin_amdgcn_s_waitcnt(0x0F70);
        __syncthreads();
    }

    // src: the tile's first rows of L (hi, lo) and of R
    static __device__ __forceinline__ void run(const f16 *const (&src)[2 * PARTS], uint64_t ld, int32_t K, f16 *lds, f32x16 (&acc)[BLOCKS][BLOCKS])
    {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        const int l0 = (wave >> 1) * (TILE / 2) + (lane & 31), r0 = (wave & 1) * (TILE / 2) + (lane & 31), half = lane >> 5;
#pragma unroll
        for (int i = 0; i < BLOCKS; ++i)
#pragma unroll
            for (int j = 0; j < BLOCKS; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;
        load(src, ld, 0, lds);
        arrive();
        int now = 0;
        for (int32_t k0 = 0; k0 < K; k0 += DEPTH, now ^= 1) {
            const f16 *stage = lds + now * STAGE;
            f16x8 l[PARTS][BLOCKS][DEPTH / 16], r[PARTS][BLOCKS][DEPTH / 16];
#pragma unroll
            for (int s = 0; s < DEPTH / 16; ++s)
#pragma unroll
                for (int p = 0; p < PARTS; ++p)
#pragma unroll
                    for (int i = 0; i < BLOCKS; ++i) {
                        l[p][i][s] = fragment(stage + p * PART, l0 + i * 32, s * 2 + half);
                        r[p][i][s] = fragment(stage + (PARTS + p) * PART, r0 + i * 32, s * 2 + half);
                    }
            // The next step's loads go out behind these reads (of the other stage, which no wave reads any more since the last barrier).
            if (k0 + DEPTH < K) load(src, ld, k0 + DEPTH, lds + (now ^ 1) * STAGE);
#pragma unroll
            for (int s = 0; s < DEPTH / 16; ++s)
#pragma unroll
                for (int i = 0; i < BLOCKS; ++i)
#pragma unroll
                    for (int j = 0; j < BLOCKS; ++j) {
                        if constexpr (SPLIT) {
                            acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(l[1][i][s], r[0][j][s], acc[i][j], 0, 0, 0);
                            acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(l[0][i][s], r[1][j][s], acc[i][j], 0, 0, 0);
                        }
                        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(l[0][i][s], r[0][j][s], acc[i][j], 0, 0, 0);
                    }
            __builtin_amdgcn_sched_barrier(0);                   // the wait stays behind the products
            arrive();
        }
    }

    // body(row, column of the tile, value) for the elements of this lane: four consecutive rows of a column at a time
    template <typename F> static __device__ __forceinline__ void each(const f32x16 (&acc)[BLOCKS][BLOCKS], F &&body)
    {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
        for (int i = 0; i < BLOCKS; ++i)
#pragma unroll
            for (int j = 0; j < BLOCKS; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    body((wave >> 1) * (TILE / 2) + i * 32 + (e >> 2) * 8 + (lane >> 5) * 4 + (e & 3), (wave & 1) * (TILE / 2) + j * 32 + (lane & 31), acc[i][j][e]);
    }
};

// Tile t of the lower half, row by row: (row, column), column <= row.
__device__ __forceinline__ void half_tile(uint32_t t, int32_t &row, int32_t &column)
{
    uint32_t r = (uint32_t)((sqrtf(8.f * (float)t + 1.f) - 1.f) * 0.5f);
    while ((r + 1) * (r + 2) / 2 <= t) ++r;
    while (r * (r + 1) / 2 > t) --r;
    row = (int32_t)r;
    column = (int32_t)(t - r * (r + 1) / 2);
}

// A = X X^T (POLY false), P = b f^2 A + c f^4 A^2 (POLY true): the tiles of the lower half, and their reflections.
template <int TILE, bool SPLIT, bool POLY>
__global__ void __launch_bounds__(256) update_half_kernel(Group g, bool first)
{
    extern __shared__ __align__(16) uint8_t lds_bytes[];
    using Prod = Product<TILE, SPLIT>;
    const Matrix &m = g.mat[matrix_of<&Matrix::half_first>(g, blockIdx.x)];
    int32_t ti, tj;
    half_tile(blockIdx.x - m.half_first, ti, tj);
    const Operand &from = POLY ? m.a : m.xr, &to = POLY ? m.p : m.a;
    const int32_t K = POLY ? m.n_pad : m.m_pad;
    const uint64_t ld = (uint64_t)K, left = (uint64_t)ti * TILE * ld, right = (uint64_t)tj * TILE * ld;
    const f16 *src[2 * Prod::PARTS];
    src[0] = from.hi + left;
    src[Prod::PARTS] = from.hi + right;
    if constexpr (SPLIT) { src[1] = from.lo + left; src[3] = from.lo + right; }
    f32x16 acc[Prod::BLOCKS][Prod::BLOCKS];
    Prod::run(src, ld, K, reinterpret_cast<f16 *>(lds_bytes), acc);
    float cb = NS_B, cc = NS_C * UNSCALE;
    if (POLY && first) {
        const float f = *m.factor;
        cb *= f * f;
        cc *= f * f * f * f;
    }
    Prod::each(acc, [&](int r, int c, float v) {
        const int64_t i = ti * TILE + r, j = tj * TILE + c;
        const uint64_t at = (uint64_t)i * m.n_pad + j;
        if (POLY) {
            float a = (float)m.a.hi[at];
            if (SPLIT) a += (float)m.a.lo[at];
            v = cb * a + cc * v;
        } else {
            v *= UNSCALE;
        }
        put(to, at, v, SPLIT);
        if (ti != tj) put(to, (uint64_t)j * m.n_pad + i, v, SPLIT);
    });
}

// X <- f (a X + P X); behind the last step the result goes out instead.
template <typename T, int TILE, bool SPLIT, bool LAST>
__global__ void __launch_bounds__(256) update_apply_kernel(Group g, uint32_t step)
{
    extern __shared__ __align__(16) uint8_t lds_bytes[];
    using Prod = Product<TILE, SPLIT>;
    const Matrix &m = g.mat[matrix_of<&Matrix::whole_first>(g, blockIdx.x)];
    const uint32_t t = blockIdx.x - m.whole_first, across = (uint32_t)m.m_pad / TILE;
    const int32_t ti = (int32_t)(t / across), tj = (int32_t)(t % across);
    const Operand &columns = m.xt[step & 1], &next = m.xt[(step & 1) ^ 1];
    const uint64_t ld = (uint64_t)m.n_pad, left = (uint64_t)ti * TILE * ld, right = (uint64_t)tj * TILE * ld;
    const f16 *src[2 * Prod::PARTS];
    src[0] = m.p.hi + left;
    src[Prod::PARTS] = columns.hi + right;
    if constexpr (SPLIT) { src[1] = m.p.lo + left; src[3] = columns.lo + right; }
    f32x16 acc[Prod::BLOCKS][Prod::BLOCKS];
    Prod::run(src, ld, m.n_pad, reinterpret_cast<f16 *>(lds_bytes), acc);
    const float f = step == 0 ? *m.factor : 1.f;
    const float grow = g.muon ? g.lr * sqrtf(fmaxf(1.f, (float)m.u.rows / (float)m.u.cols)) : 0.f;
    Prod::each(acc, [&](int r, int c, float v) {
        const int32_t i = ti * TILE + r, j = tj * TILE + c;
        const uint64_t at = (uint64_t)i * m.m_pad + j;
        v = f * (NS_A * m.x[at] + v * (UNSCALE * UNSCALE));
        if constexpr (LAST) {
            if (i >= m.n || j >= m.m) return;
            const int32_t row = m.tall ? j : i, col = m.tall ? i : j;
            if (g.muon) v = g.keep * (float)row_at<T>(m.u.weight, m.u.weight_stride, row)[col] - grow * v;
            row_at<T>(m.u.out, m.u.out_stride, row)[col] = (T)v;
        } else {
            m.x[at] = v;
            put(m.xr, at, v * SCALE, SPLIT);
            put(next, (uint64_t)j * m.n_pad + i, v * SCALE, SPLIT);
        }
    });
}

// ---------------------------------------------------------------- launches
// LDS beyond 64 KB has to be asked for, once per kernel and device.
template <typename K> rg_status allow_lds(K kernel, int bytes)
{
    if (bytes <= 64 * 1024) return RG_OK;
    RG_HIP(hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, bytes));
    return RG_OK;
}

template <typename T, int TILE, bool SPLIT>
rg_status launch_group(const Group &g, uint32_t steps, uint32_t sum_grid, uint32_t tiles, uint32_t half, uint32_t whole, hipStream_t st)
{
    constexpr int LDS = Product<TILE, SPLIT>::LDS_BYTES;
    hipLaunchKernelGGL(update_sums_kernel<T>, dim3(sum_grid), dim3(256), 0, st, g);
    RG_HIP(hipGetLastError());
    hipLaunchKernelGGL((update_start_kernel<T, SPLIT>), dim3(tiles), dim3(256), 0, st, g);
    RG_HIP(hipGetLastError());
    RG_TRY(allow_lds(update_half_kernel<TILE, SPLIT, false>, LDS));
    RG_TRY(allow_lds(update_half_kernel<TILE, SPLIT, true>, LDS));
    RG_TRY(allow_lds(update_apply_kernel<T, TILE, SPLIT, false>, LDS));
    RG_TRY(allow_lds(update_apply_kernel<T, TILE, SPLIT, true>, LDS));
    for (uint32_t s = 0; s < steps; ++s) {
        hipLaunchKernelGGL((update_half_kernel<TILE, SPLIT, false>), dim3(half), dim3(256), LDS, st, g, s == 0);
        RG_HIP(hipGetLastError());
        hipLaunchKernelGGL((update_half_kernel<TILE, SPLIT, true>), dim3(half), dim3(256), LDS, st, g, s == 0);
        RG_HIP(hipGetLastError());
        if (s + 1 < steps) hipLaunchKernelGGL((update_apply_kernel<T, TILE, SPLIT, false>), dim3(whole), dim3(256), LDS, st, g, s);
        else hipLaunchKernelGGL((update_apply_kernel<T, TILE, SPLIT, true>), dim3(whole), dim3(256), LDS, st, g, s);
        RG_HIP(hipGetLastError());
    }
    return RG_OK;
}

// Hands out the workspace; with no workspace it only counts.
struct Carver {
    uint8_t *base;
    uint64_t used = 0;
    template <typename P> void take(P *&p, uint64_t n)
    {
        p = base ? reinterpret_cast<P *>(base + used) : nullptr;
        used += (n * sizeof(P) + 255) & ~255ull;
    }
    void take(Operand &o, uint64_t n, bool split)
    {
        take(o.hi, n);
        o.lo = nullptr;
        if (split) take(o.lo, n);
    }
};

void lay_out(Matrix &m, const rg_update &u, int tile, bool split, Carver &c)
{
    m.u = u;
    m.tall = u.rows > u.cols;
    m.n = (int32_t)(m.tall ? u.cols : u.rows);
    m.m = (int32_t)(m.tall ? u.rows : u.cols);
    m.n_pad = (m.n + tile - 1) / tile * tile;
    m.m_pad = (m.m + tile - 1) / tile * tile;
    const uint64_t nm = (uint64_t)m.n_pad * m.m_pad, nn = (uint64_t)m.n_pad * m.n_pad;
    c.take(m.sums, SUM_BLOCKS);
    c.take(m.factor, 1);
    c.take(m.x, nm);
    c.take(m.xr, nm, split);
    c.take(m.xt[0], nm, split);
    c.take(m.xt[1], nm, split);
    c.take(m.a, nn, split);
    c.take(m.p, nn, split);
}

// Groups of matrices of a size class, in order, each with the whole workspace to itself.
struct Options { bool muon, nesterov; float momentum, lr, weight_decay, eps; uint32_t steps; };

template <typename F> rg_status each_group(const rg_update *u, uint32_t n, uint32_t type, F &&body)
{
    for (const UpdateClass c : {UPDATE_NARROW, UPDATE_SMALL, UPDATE_LARGE}) {
        const rg_update *picked[RG_UPDATES_PER_LAUNCH];
        uint32_t count = 0;
        for (uint32_t k = 0; k < n; ++k) {
            if (u[k].rows == 0 || u[k].cols == 0 || update_class(u[k].rows, u[k].cols, type == RG_F32) != c) continue;
            picked[count++] = &u[k];
            if (count == RG_UPDATES_PER_LAUNCH) { RG_TRY(body(c, picked, count)); count = 0; }
        }
        if (count) RG_TRY(body(c, picked, count));
    }
    return RG_OK;
}

template <typename T>
rg_status run_group(UpdateClass kind, const rg_update *const *u, uint32_t count, const Options &o, uint8_t *workspace, hipStream_t st)
{
    Group g{};
    g.count = count;
    g.muon = o.muon; g.nesterov = o.nesterov;
    g.momentum = o.momentum; g.lr = o.lr; g.keep = (float)(1.0 - (double)o.lr * (double)o.weight_decay);
    g.eps = o.eps;
    Carver c{workspace};
    constexpr bool WIDE = sizeof(T) == 4;
    const int tile = tile_of(kind);
    uint32_t sums = 0, tiles = 0, half = 0, whole = 0;
    for (uint32_t k = 0; k < count; ++k) {
        Matrix &m = g.mat[k];
        lay_out(m, *u[k], tile, WIDE || kind == UPDATE_NARROW, c);
        m.sum_blocks = (uint32_t)std::max<uint64_t>(1, std::min<uint64_t>(SUM_BLOCKS, (uint64_t)m.n * m.m / 4096));
        m.sum_first = sums; m.tile_first = tiles; m.half_first = half; m.whole_first = whole;
        const uint32_t tn = (uint32_t)(m.n_pad / tile), tm = (uint32_t)(m.m_pad / tile);
        sums += m.sum_blocks;
        tiles += (uint32_t)(m.n_pad / 64) * (uint32_t)(m.m_pad / 64);
        half += tn * (tn + 1) / 2;
        whole += tn * tm;
    }
    if (kind == UPDATE_LARGE) return launch_group<T, UPDATE_TILE, WIDE>(g, o.steps, sums, tiles, half, whole, st);
    if (kind == UPDATE_SMALL) return launch_group<T, UPDATE_TILE_SMALL, WIDE>(g, o.steps, sums, tiles, half, whole, st);
    return launch_group<T, UPDATE_TILE_SMALL, true>(g, o.steps, sums, tiles, half, whole, st);
}

rg_status check_updates(const rg_update *u, uint32_t n, uint32_t type)
{
    if (!element_bytes(type)) { set_error("type %u is none of RG_F32, RG_BF16, RG_F16", type); return RG_EINVAL; }
    if (n && !u) { set_error("null argument"); return RG_EINVAL; }
    for (uint32_t k = 0; k < n; ++k)
        if (u[k].rows > RG_MAX_SIDE || u[k].cols > RG_MAX_SIDE) { set_error("matrix %u: %u x %u is beyond RG_MAX_SIDE", k, u[k].rows, u[k].cols); return RG_ERANGE; }
    return RG_OK;
}

rg_status check_array(uint32_t k, const char *what, const void *p, uint64_t stride, const rg_update &u, uint32_t bytes, bool output)
{
    if (!p) { set_error("matrix %u: %s is null", k, what); return RG_EINVAL; }
    if ((reinterpret_cast<uintptr_t>(p) | stride) % bytes) { set_error("matrix %u: %s: address and stride have to be multiples of %u bytes", k, what, bytes); return RG_EINVAL; }
    if (output && u.rows > 1 && stride < (uint64_t)u.cols * bytes) { set_error("matrix %u: %s: a stride of %llu bytes is less than a row", k, what, (unsigned long long)stride); return RG_EINVAL; }
    if (stride > 1ull << 40) { set_error("matrix %u: %s: a stride of %llu bytes is beyond the limit (2^40)", k, what, (unsigned long long)stride); return RG_ERANGE; }
    return RG_OK;
}

uint64_t workspace_of(const rg_update *u, uint32_t n, uint32_t type)
{
    uint64_t most = 0;
    (void)each_group(u, n, type, [&](UpdateClass kind, const rg_update *const *picked, uint32_t count) {
        Carver c{nullptr};
        for (uint32_t k = 0; k < count; ++k) {
            Matrix m;
            lay_out(m, *picked[k], tile_of(kind), type == RG_F32 || kind == UPDATE_NARROW, c);
        }
        most = std::max(most, c.used);
        return RG_OK;
    });
    return most;
}

rg_status run_updates(const rg_update *u, uint32_t n, uint32_t type, const Options &o, void *workspace, uint64_t workspace_bytes, void *stream)
{
    RG_TRY(check_updates(u, n, type));
    if (o.steps < 1 || o.steps > RG_MAX_STEPS) { set_error("%u steps are not 1 to RG_MAX_STEPS", o.steps); return RG_EINVAL; }
    if (!(o.eps >= 0.f) || std::isinf(o.eps)) { set_error("eps has to be a number >= 0"); return RG_EINVAL; }
    if (!std::isfinite(o.lr) || !std::isfinite(o.weight_decay) || !std::isfinite(o.momentum)) { set_error("lr, weight_decay and momentum have to be finite"); return RG_EINVAL; }
    const uint32_t bytes = element_bytes(type);
    for (uint32_t k = 0; k < n; ++k) {
        if (u[k].rows == 0 || u[k].cols == 0) continue;
        RG_TRY(check_array(k, "grad", u[k].grad, u[k].grad_stride, u[k], bytes, false));
        RG_TRY(check_array(k, "out", u[k].out, u[k].out_stride, u[k], bytes, true));
        if (!o.muon) continue;
        RG_TRY(check_array(k, "weight", u[k].weight, u[k].weight_stride, u[k], bytes, false));
        RG_TRY(check_array(k, "momentum", u[k].momentum, u[k].momentum_stride, u[k], 4, false));
        RG_TRY(check_array(k, "momentum_out", u[k].momentum_out, u[k].momentum_out_stride, u[k], 4, true));
    }
    const uint64_t want = workspace_of(u, n, type);
    if (want == 0) return RG_OK;
    if (!workspace || reinterpret_cast<uintptr_t>(workspace) % 256) { set_error("the workspace is null or not aligned to 256 bytes"); return RG_EINVAL; }
    if (workspace_bytes < want) { set_error("the workspace holds %llu bytes of %llu", (unsigned long long)workspace_bytes, (unsigned long long)want); return RG_ERANGE; }
    const hipStream_t st = as_stream(stream);
    uint8_t *ws = static_cast<uint8_t *>(workspace);
    return each_group(u, n, type, [&](UpdateClass kind, const rg_update *const *picked, uint32_t count) {
        return type == RG_F32 ? run_group<float>(kind, picked, count, o, ws, st) : type == RG_BF16 ? run_group<bf16>(kind, picked, count, o, ws, st) : run_group<f16>(kind, picked, count, o, ws, st);
    });
}

}  // namespace
}  // namespace rg

using namespace rg;

extern "C" rg_status rg_update_workspace(const rg_update *u, uint32_t n, uint32_t type, uint64_t *bytes)
{
    if (!bytes) { set_error("null argument"); return RG_EINVAL; }
    RG_TRY(check_updates(u, n, type));
    *bytes = workspace_of(u, n, type);
    return RG_OK;
}

extern "C" rg_status rg_orthogonalize(const rg_update *u, uint32_t n, uint32_t type, uint32_t steps, float eps, void *workspace, uint64_t workspace_bytes, void *stream)
{
    return run_updates(u, n, type, Options{false, false, 0.f, 0.f, 0.f, eps, steps}, workspace, workspace_bytes, stream);
}

extern "C" rg_status rg_muon_step(const rg_update *u, uint32_t n, uint32_t type, float lr, float weight_decay, float momentum, int nesterov, uint32_t steps, float eps,
                                  void *workspace, uint64_t workspace_bytes, void *stream)
{
    return run_updates(u, n, type, Options{true, nesterov != 0, momentum, lr, weight_decay, eps, steps}, workspace, workspace_bytes, stream);
}
