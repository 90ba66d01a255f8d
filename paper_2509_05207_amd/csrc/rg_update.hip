// Orthogonalised updates of weight matrices (Newton-Schulz products) and the optimiser step around them: rg_orthogonalize, rg_muon_step.
//
// With n the narrower side and m the wider one a step is A = X X^T (n x n, symmetric), P = b A + c A^2 (symmetric) and
// X <- a X + P X: n(n+1)m + n(n+1)n + 2 n^2 m operations, of which the symmetric products compute one half and write the other by
// reflection.  Large matrices are bound by the matrix cores, small ones by the launches.
//
// Precision.  A rounding of X itself is noise in the directions of X's small singular values, which every step
// multiplies by 3.4; a rounding of P only tilts the directions that are there.  So the state X is kept in fp32 and a X is added from it.  The operands of
// the products are fp16 numbers, scaled by 2^14, since nothing here is four or more (singular values stay below 1.21, A's entries below 1.46, P's below 2.9), and
// always the sum of two, 22 bits, with no digits below 2^-38 of the matrix' norm; a product is three, hi hi + hi lo + lo hi.  Results are 1e-7 to 3e-6 off so (relative, 2-norm), as much as by
// fp32 products, whatever the type; its own rounding comes last, once.  (fp32 matrices of few rows, of which that is not so, have products in 64 bits: see narrow matrices.)  One part, 11 bits, is not enough for matrices of 16 bits either: roundings of singular values that are alike
// do not average out (43 rows of a unit matrix 8e-3 off, 48 x 4,096 orthonormal rows 4e-3, 400 x 500 of noise 1.6e-3, where rounding to bf16 costs 1.7e-3 and to fp16 2e-4).
//
// The division by the norm is exact: X starts as G 2^-e with a norm in [1/2, 1), and the factor f = 2^e / (|G| + eps) that is left
// goes into the first step's coefficients: P = b f^2 A + c f^4 A^2, X <- f (a X + P X).
//
// Every operand is kept with the axis that a product runs along contiguous: X and its transpose both, in blocks padded by zeros
// to whole tiles, so that no product checks a bound.
#include "rg_internal.h"
#include "rg_elements.h"
#include "rg_launch.h"

#include <atomic>
#include <cmath>
#include <type_traits>

namespace rg {

namespace {

constexpr float NS_A = 3.4445f, NS_B = -4.7750f, NS_C = 2.0315f;
constexpr float SCALE = 16384.f, UNSCALE = 1.f / 16384.f;             // of the fp16 operands
constexpr int SUM_BLOCKS = 1024;                                      // partial sums of squares of a matrix, at most

typedef f16 f16x8 __attribute__((ext_vector_type(8)));
typedef f16 f16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// An operand's rows: the fp16 numbers nearest to its values, every 32 of them followed by the 32 nearest to what they leave, so that both parts
// of a piece lie in one line of 128 bytes.
__host__ __device__ __forceinline__ uint32_t row_length(int32_t n) { return 2u * (uint32_t)n; }
__device__ __forceinline__ uint64_t place(int32_t row, int32_t column, int32_t n_columns)
{
    return (uint64_t)row * row_length(n_columns) + (uint32_t)column + ((uint32_t)column & ~31u);
}
constexpr int LO = 32;                   // from a number to what it leaves

struct Matrix {
    rg_update u;
    int32_t n, m, n_pad, m_pad;          // narrower and wider side, and padded
    bool tall;                           // rows > cols: X is the transpose
    uint32_t sum_blocks;                 // workgroups of the first pass; of a narrow matrix, parts of its columns
    double *sums;                        // [sum_blocks]; of a narrow matrix, of tiles of A
    float *factor;                       // f
    float *x;                            // [n_pad][m_pad]
    f16 *xr, *xt[2];                     // operands: X's rows [n_pad][m_pad], its columns [m_pad][n_pad] before and after a step
    f16 *a, *p;                          // [n_pad][n_pad]
};

// Workgroups of a launch in front of each matrix'; beyond the last matrix none comes.
struct Starts { uint32_t first[RG_UPDATES_PER_LAUNCH]; };

struct Group {
    Starts sums, starts, half, whole;    // of the launches: sums of squares; X laid out; symmetric products; others
    bool muon, nesterov;
    float momentum, lr, keep;            // keep = 1 - lr * weight_decay
    float eps;
    Matrix mat[RG_UPDATES_PER_LAUNCH];
};

static_assert(sizeof(Group) <= 4000, "kernel arguments are 4 KB at most");

// The matrix that workgroup t belongs to, and the workgroup's number within it.
__device__ __forceinline__ uint32_t matrix_of(const Starts &s, uint32_t t, uint32_t &within)
{
    uint32_t k = 0, first = 0;
#pragma unroll
    for (uint32_t j = 1; j < RG_UPDATES_PER_LAUNCH; ++j)
        if (t >= s.first[j]) { k = j; first = s.first[j]; }
    within = t - first;
    return k;
}

template <typename T> __device__ __forceinline__ const T *row_at(const void *p, uint64_t stride, int64_t r) { return reinterpret_cast<const T *>(static_cast<const uint8_t *>(p) + (uint64_t)r * stride); }
template <typename T> __device__ __forceinline__ T *row_at(void *p, uint64_t stride, int64_t r) { return reinterpret_cast<T *>(static_cast<uint8_t *>(p) + (uint64_t)r * stride); }

// ---------------------------------------------------------------- momentum, sum of squares
constexpr int PACK = 8;

// Elements [c, c + PACK) of a row of cols, what lies beyond it zero.
template <typename T> __device__ __forceinline__ void load_part(const T *row, uint32_t c, uint32_t cols, float (&v)[PACK])
{
    if (c + PACK <= cols) {
        load_pack(row + c, v);
    } else {
#pragma unroll
        for (int e = 0; e < PACK; ++e) v[e] = c + e < cols ? (float)row[c + e] : 0.f;
    }
}

// The update that a step orthogonalises, out of the gradient and (muon) the new momentum.
__device__ __forceinline__ float update_of(const Group &g, float grad, float next) { return g.nesterov ? grad + g.momentum * next : next; }

// The new momentum, and partial sums of the update's squares, in 64 bits.  Bound by HBM.  (Six matrices of 1,024 x 4,096 bf16, us: 43; 252 MB, 5.9 TB/s.)
template <typename T>
__global__ void __launch_bounds__(256) update_sums_kernel(Group g)
{
    uint32_t block;
    const Matrix &m = g.mat[matrix_of(g.sums, blockIdx.x, block)];
    const uint32_t cols = m.u.cols, packs = (cols + PACK - 1) / PACK, all = m.u.rows * packs;
    double s = 0.0;
    for (uint32_t p = block * 256 + threadIdx.x; p < all; p += m.sum_blocks * 256) {
        const uint32_t r = p / packs, c = (p - r * packs) * PACK;
        float v[PACK];
        load_part(row_at<T>(m.u.grad, m.u.grad_stride, r), c, cols, v);
        if (g.muon) {
            float next[PACK];
            load_part(row_at<float>(m.u.momentum, m.u.momentum_stride, r), c, cols, next);
            float *out = row_at<float>(m.u.momentum_out, m.u.momentum_out_stride, r) + c;
#pragma unroll
            for (int e = 0; e < PACK; ++e) {
                next[e] = g.momentum * next[e] + v[e];
                v[e] = update_of(g, v[e], next[e]);
            }
            if (c + PACK <= cols) {
                store_pack(out, next);
            } else {
#pragma unroll
                for (int e = 0; e < PACK; ++e)
                    if (c + e < cols) out[e] = next[e];
            }
        }
#pragma unroll
        for (int e = 0; e < PACK; ++e) s += (double)v[e] * (double)v[e];
    }
    __shared__ double part[4];
    for (int k = 1; k < 64; k <<= 1) s += __shfl_xor(s, k);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x == 0) m.sums[block] = part[0] + part[1] + part[2] + part[3];
}

// ---------------------------------------------------------------- X in the layouts of the products
// V consecutive numbers of an operand (V divides 32).
template <int V> __device__ __forceinline__ void put(f16 *to, const float (&v)[V])
{
    typedef f16 P __attribute__((ext_vector_type(V)));
    P h;
#pragma unroll
    for (int e = 0; e < V; ++e) h[e] = (f16)v[e];
    *reinterpret_cast<P *>(to) = h;
#pragma unroll
    for (int e = 0; e < V; ++e) h[e] = (f16)(v[e] - (float)h[e]);
    *reinterpret_cast<P *>(to + LO) = h;
}

// f of a matrix of this norm, which starts as G 2^-e2.
__device__ __forceinline__ float factor_of(double norm, float eps, int &e2)
{
    e2 = 0;
    if (norm > 0.0 && norm < INFINITY) (void)frexp(norm, &e2);
    if (!(norm < INFINITY)) return NAN;
    return norm == 0.0 && eps > 0.f ? 0.f : (float)(ldexp(1.0, e2) / (norm + (double)eps));
}

// A workgroup takes 64 x 64 elements of the padded X, which go through LDS to be written by columns too.  Bound by HBM.  (The same six, us: 83; 453 MB, 5.5 TB/s.)
template <typename T>
__global__ void __launch_bounds__(256) update_start_kernel(Group g)
{
    uint32_t tile;
    const Matrix &m = g.mat[matrix_of(g.starts, blockIdx.x, tile)];
    __shared__ double part[4];
    __shared__ float block[64][65];
    // G is read along its rows: along X's rows, or, where X is G's transpose, along its columns.  What is read does not wait for the norm.
    const int32_t across = m.m_pad / 64;
    const int32_t i0 = (int32_t)(tile / across) * 64, j0 = (int32_t)(tile % across) * 64;
    const int32_t k = (int32_t)threadIdx.x >> 3, c = ((int32_t)threadIdx.x & 7) * PACK;
    float v[2][PACK];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int32_t row = (m.tall ? j0 : i0) + k + 32 * h, col = (m.tall ? i0 : j0) + c;
        if (row < (int32_t)m.u.rows) {
            load_part(row_at<T>(m.u.grad, m.u.grad_stride, row), col, m.u.cols, v[h]);
            if (g.muon) {
                float next[PACK];
                load_part(row_at<float>(m.u.momentum_out, m.u.momentum_out_stride, row), col, m.u.cols, next);
#pragma unroll
                for (int e = 0; e < PACK; ++e) v[h][e] = update_of(g, v[h][e], next[e]);
            }
        } else {
#pragma unroll
            for (int e = 0; e < PACK; ++e) v[h][e] = 0.f;
        }
    }
    double s = 0.0;
    for (uint32_t p = threadIdx.x; p < m.sum_blocks; p += 256) s += m.sums[p];
    for (int q = 1; q < 64; q <<= 1) s += __shfl_xor(s, q);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = s;
    __syncthreads();
    int e2 = 0;
    const float f = factor_of(sqrt(part[0] + part[1] + part[2] + part[3]), g.eps, e2);
    if (tile == 0 && threadIdx.x == 0) *m.factor = f;
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int e = 0; e < PACK; ++e) {
            const float x = ldexpf(v[h][e], -e2);
            if (m.tall) block[c + e][k + 32 * h] = x; else block[k + 32 * h][c + e] = x;
        }
    __syncthreads();
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int32_t line = k + 32 * h;
        float x[PACK];
#pragma unroll
        for (int e = 0; e < PACK; ++e) x[e] = block[line][c + e];
        const uint64_t row = (uint64_t)(i0 + line) * m.m_pad + j0 + c;
        *reinterpret_cast<f32x4 *>(m.x + row) = f32x4{x[0], x[1], x[2], x[3]};
        *reinterpret_cast<f32x4 *>(m.x + row + 4) = f32x4{x[4], x[5], x[6], x[7]};
#pragma unroll
        for (int e = 0; e < PACK; ++e) x[e] *= SCALE;
        put(m.xr + place(i0 + line, j0 + c, m.m_pad), x);
#pragma unroll
        for (int e = 0; e < PACK; ++e) x[e] = block[c + e][line] * SCALE;
        put(m.xt[0] + place(j0 + line, i0 + c, m.n_pad), x);
    }
}

// ---------------------------------------------------------------- products
// C = L R^T of a tile of TILE x TILE by WM x WN waves of BI x BJ blocks of 16 x 16; both operands run along K contiguously, K a multiple of 64.  Steps of
// DEPTH along K pass through LDS, STAGES of them there: one is multiplied while the others arrive, written into LDS by the loads
// themselves.  A row of a step is 16-byte chunks, stored in an order that depends on the row, so that the 16 lanes that LDS serves at a time (16 rows, one
// chunk of each) fall on all banks once.
//
// A step is what LDS takes in, what the waves read from it and the matrix operations, which overlap in part: all waves stand at about the same point of a
// step (4,096 x 4,096, X X^T by tiles of 192, us: 191; without matrix operations 108, without reads from LDS 146, without loads 141, matrix operations alone 125, loads
// alone 109; the matrix units are busy for 60 % of it).  Larger tiles read less for the same products (the same matrix, tiles of 64, 96, 128, 192, us: X X^T 333, 239, 270, 191, P X 510, 445, 403, 412, and 386 by
// pairs of 128, of which one finishes while the other multiplies); smaller ones fill the chip with less work (2,048 x 2,048, X X^T 49, 43, 53, 85, P X 80, 69, 62, 100).  Waves of 96 x 96 and 128 x 128,
// one to a vector unit, read half as much and are slower: nothing else runs while such a wave waits (operands of one part, X X^T by tiles of 192: 80, so 130).
//
// Where there are no more tiles than compute units a wave alone on its vector unit waits for LDS most of a step.  KG > 1: KG waves share a block, each with
// its own slices of a step; their sums meet in LDS at the end, and each finishes one block of the wave's BI x BJ (or one of them the only block).  There the cross terms
// of operands in two parts have sums of their own, lo hi + hi lo, so that a result and its reflection are the same bits whatever the tile.
template <int WM, int WN, int BI, int BJ, int DEPTH_, int STAGES_, int KG = 1>
struct Product {
    static constexpr int DEPTH = DEPTH_, STAGES = STAGES_;       // DEPTH: numbers of a row in a step, of both parts together
    static constexpr int THREADS = WM * WN * KG * 64, TILE = WM * BI * 16;
    static_assert(TILE == WN * BJ * 16, "the lower half of a symmetric product is made of square tiles");
    static constexpr int CHUNKS = DEPTH / 8;
    static constexpr int STAGE = 2 * TILE * DEPTH;               // numbers: L's rows, R's rows
    static constexpr int LDS_BYTES = STAGES * STAGE * 2;
    static constexpr int SIDE_LOADS = TILE * CHUNKS / THREADS;   // of a thread, to a step
    static_assert(DEPTH % 64 == 0 && TILE * CHUNKS % THREADS == 0 && LDS_BYTES <= 160 * 1024, "");
    static constexpr int SLICES = DEPTH / 32 / KG;               // of a wave; what one matrix operation takes along K each, hi and lo parts by turns
    static_assert(DEPTH == SLICES * KG * 32 && SLICES % 2 == 0 && (KG == 1 || ((KG == BI * BJ || BI * BJ == 1) && WM * WN * KG * BI * BJ * 1024 <= LDS_BYTES)), "");
    static constexpr bool APART = KG > 1;                        // sums of the cross terms
    typedef f32x4 Acc[BI][BJ];

    static __device__ __forceinline__ int slot_of(int row, int chunk) { return chunk ^ (DEPTH == 64 ? (row >> 1) & 7 : row & 15); }

    // Rows from first on of the operand, of which it has n_rows (what a tile has beyond is read from the last row and not used).
    struct Side { const f16 *rows; int32_t first, n_rows; };

    // Where a thread's loads of a step come from: 32-bit offsets (an operand of RG_MAX_SIDE rows is 1 GiB at most).
    struct Source {
        const uint8_t *base[2];
        uint32_t offset[2][SIDE_LOADS];
        uint32_t along[KG > 1 ? SIDE_LOADS : 1], most;             // KG > 1, where a step can leave the row: the bytes along it apart, and the last chunk's
        __device__ __forceinline__ void load_one(int32_t k0, f16 *stage, int side, int i) const
        {
            const auto *from = (const __attribute__((address_space(1))) uint8_t *)(base[side] + (KG > 1 ? 0 : 2 * (int64_t)k0));
            f16 *to = stage + side * TILE * DEPTH + (i * THREADS + (int)(threadIdx.x & ~63u)) * 8;
            const uint32_t at = KG > 1 ? offset[side][i] + min(along[KG > 1 ? i : 0] + 2u * (uint32_t)k0, most) : offset[side][i];
            __builtin_amdgcn_global_load_lds(from + at, (__attribute__((address_space(3))) void *)to, 16, 0, 0);
        }
        __device__ __forceinline__ void load(int32_t k0, f16 *stage) const
        {
#pragma unroll
            for (int side = 0; side < 2; ++side)
#pragma unroll
                for (int i = 0; i < SIDE_LOADS; ++i) load_one(k0, stage, side, i);
        }
    };

    // Waits until all but the newest N of this wave's loads have arrived, and then for every wave to be there.  __syncthreads would wait for all of the
    // loads: this is the barrier alone, and what was read from LDS before has been used before.  The fences keep the compiler to the order and cost no instruction.
    template <int N> static __device__ __forceinline__ void arrive()
    {
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_waitcnt((N & 15) | (7 << 4) | ((N >> 4) << 14));             // vmcnt N, lgkmcnt 0
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_sched_barrier(0);
    }

    // K: numbers along a row of the operands, of both parts together; a multiple of 128
    static __device__ __forceinline__ void run(const Side &L, const Side &R, int32_t K, f16 *lds, Acc &acc)
    {
        // The wave's number is the same in all its lanes, and the compiler has to know: matrix operations take no heed of which lanes are active, so that a
        // slice may only be passed over by a branch of the whole wave.
        const int all = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
        const int lane = threadIdx.x & 63, group = all / (WM * WN), wave = all % (WM * WN);
        Source src;
        src.base[0] = reinterpret_cast<const uint8_t *>(L.rows);
        src.base[1] = reinterpret_cast<const uint8_t *>(R.rows);
        src.most = (uint32_t)K * 2u - 16u;
#pragma unroll
        for (int i = 0; i < SIDE_LOADS; ++i) {
            const int q = i * THREADS + (int)threadIdx.x, row = q / CHUNKS;
            const uint32_t at = (uint32_t)slot_of(row, q % CHUNKS) * 16u;
            if constexpr (KG > 1) src.along[i] = at;
            src.offset[0][i] = (uint32_t)min(L.first + row, L.n_rows - 1) * (uint32_t)K * 2u + (KG > 1 ? 0 : at);
            src.offset[1][i] = (uint32_t)min(R.first + row, R.n_rows - 1) * (uint32_t)K * 2u + (KG > 1 ? 0 : at);
        }
#pragma unroll
        for (int i = 0; i < BI; ++i)
#pragma unroll
            for (int j = 0; j < BJ; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
        Acc lo_hi, hi_lo;
        if constexpr (APART)
#pragma unroll
            for (int i = 0; i < BI; ++i)
#pragma unroll
                for (int j = 0; j < BJ; ++j) lo_hi[i][j] = hi_lo[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
        const int row_l = (wave / WN) * BI * 16 + (lane & 15), row_r = TILE + (wave % WN) * BJ * 16 + (lane & 15);
        f16x8 l[SLICES][BI], r[SLICES][BJ];
        const auto read_one = [&](const f16 *stage, int s, int row, f16x8 &x) {
            const int slot = slot_of(lane & 15, (group * SLICES + s) * 4 + (lane >> 4)) * 8;      // the rows of a block begin at multiples of 16
            x = *reinterpret_cast<const f16x8 *>(stage + row * DEPTH + slot);
        };
        const auto read = [&](const f16 *stage, int s, f16x8 (&x)[BI], f16x8 (&y)[BJ]) {
#pragma unroll
            for (int i = 0; i < BI; ++i) read_one(stage, s, row_l + i * 16, x[i]);
#pragma unroll
            for (int j = 0; j < BJ; ++j) read_one(stage, s, row_r + j * 16, y[j]);
        };
        const auto add_row = [&](Acc &to, int i, const f16x8 (&x)[BI], const f16x8 (&y)[BJ]) {
#pragma unroll
            for (int j = 0; j < BJ; ++j) to[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(x[i], y[j], to[i][j], 0, 0, 0);
        };
        // All stages are filled at first, and a stage again as soon as every wave has read the last of it, which is in the middle of a step: the barrier
        // there also says that the next step has arrived, whose first slice is read while the present one's last is multiplied.  Behind the last step the
        // last one is loaded again, so that the number of loads under way stays the same, and read, so that there is no branch.
        const int32_t last = (K - 1) / DEPTH * DEPTH;
        if (KG > 1 && K <= STAGES * DEPTH) {                       // all of it fits: one wait
            for (int32_t k0 = 0; k0 < K; k0 += DEPTH) src.load(k0, lds + k0 / DEPTH * STAGE);
            arrive<0>();
            for (int32_t k0 = 0; k0 < K; k0 += DEPTH)
#pragma unroll
                for (int s = 0; s < SLICES; ++s) {
                    if (k0 + (group * SLICES + s) * 32 >= K) continue;                      // a slice is inside or outside as a whole
                    read(lds + k0 / DEPTH * STAGE, s, l[s], r[s]);
#pragma unroll
                    for (int i = 0; i < BI; ++i)
                        if (s % 2 == 1) {
                            add_row(APART ? lo_hi : acc, i, l[s], r[s - 1]);
                            add_row(APART ? hi_lo : acc, i, l[s - 1], r[s]);
                        } else {
                            add_row(acc, i, l[s], r[s]);
                        }
                }
            arrive<0>();                                           // LDS is read, and may be written
            finish(acc, lo_hi, hi_lo, lds, lane, group, wave);
            return;
        }
#pragma unroll
        for (int q = 0; q < STAGES; ++q) src.load(min(q * DEPTH, last), lds + q * STAGE);
        arrive<(STAGES - 1) * 2 * SIDE_LOADS>();
        f16x8 next_l[BI], next_r[BJ];
        read(lds, 0, next_l, next_r);
        int now = 0;
        for (int32_t k0 = 0; k0 < K; k0 += DEPTH) {
            f16 *stage = lds + now * STAGE;
            now = now == STAGES - 1 ? 0 : now + 1;
#pragma unroll
            for (int s = 0; s < SLICES; ++s) {
                // What was read is there.  What comes next goes out a few reads and loads at a time, between the products of one row of blocks and the next: a wave that
                // issued them all at once would wait for the units that take them, and its matrix operations with it (4,096 x 4,096, operands of one part, X X^T, us: 99 so, 85 in turns).
                // (The wait is explicit because the compiler, with loads into LDS under way, would wait for the next reads too.)
                __builtin_amdgcn_sched_barrier(0);
                __builtin_amdgcn_s_waitcnt(15 | (7 << 4) | (3 << 14));
                __builtin_amdgcn_sched_barrier(0);
                if (s == 0) {
#pragma unroll
                    for (int i = 0; i < BI; ++i) l[0][i] = next_l[i];
#pragma unroll
                    for (int j = 0; j < BJ; ++j) r[0][j] = next_r[j];
                }
                const bool step_ends = s + 1 == SLICES;
                if (step_ends) arrive<(STAGES - 2) * 2 * SIDE_LOADS>();
                const bool inside = KG == 1 || k0 + (group * SLICES + s) * 32 < K;          // a slice is inside or outside as a whole
                const int t = step_ends ? 0 : s + 1;
                const f16 *from = step_ends ? lds + now * STAGE : stage;
                f16x8 (&to_l)[BI] = step_ends ? next_l : l[t], (&to_r)[BJ] = step_ends ? next_r : r[t];
#pragma unroll
                for (int i = 0; i < BI; ++i) {
                    constexpr int READS = (BI + BJ + BI - 1) / BI, LOADS = (2 * SIDE_LOADS + BI - 1) / BI;
#pragma unroll
                    for (int q = i * READS; q < (i + 1) * READS; ++q) {
                        if (q < BJ) read_one(from, t, row_r + q * 16, to_r[q]);
                        else if (q < BI + BJ) read_one(from, t, row_l + (q - BJ) * 16, to_l[q - BJ]);
                    }
                    if (step_ends)
#pragma unroll
                        for (int q = i * LOADS; q < (i + 1) * LOADS; ++q)
                            if (q < 2 * SIDE_LOADS) src.load_one(min(k0 + STAGES * DEPTH, last), stage, q / SIDE_LOADS, q % SIDE_LOADS);
                    __builtin_amdgcn_sched_barrier(0);
                    if (inside) {
                        if (s % 2 == 1) {
                            add_row(APART ? lo_hi : acc, i, l[s], r[s - 1]);
                            add_row(APART ? hi_lo : acc, i, l[s - 1], r[s]);
                        } else {
                            add_row(acc, i, l[s], r[s]);
                        }
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        }
        arrive<0>();                                               // a workgroup's LDS is not left with loads under way
        finish(acc, lo_hi, hi_lo, lds, lane, group, wave);
    }

    // The sums of the waves that share blocks: each is left with one block, whole.
    static __device__ __forceinline__ void finish(Acc &acc, const Acc &lo_hi, const Acc &hi_lo, f16 *lds, int lane, int group, int wave)
    {
        if constexpr (KG > 1) {
            constexpr int BLOCKS = BI * BJ;
            f32x4 *sums = reinterpret_cast<f32x4 *>(lds) + lane;   // [group][wave][block][lane]
#pragma unroll
            for (int b = 0; b < BLOCKS; ++b) {
                f32x4 v = acc[b / BJ][b % BJ];
                if constexpr (APART) v += lo_hi[b / BJ][b % BJ] + hi_lo[b / BJ][b % BJ];
                sums[((group * WM * WN + wave) * BLOCKS + b) * 64] = v;
            }
            __syncthreads();
            if (group >= BLOCKS) return;
            acc[0][0] = sums[(wave * BLOCKS + group) * 64];
#pragma unroll
            for (int q = 1; q < KG; ++q) acc[0][0] += sums[((q * WM * WN + wave) * BLOCKS + group) * 64];
        }
    }

    // body(row, column of the tile, values, what first(row, column) gave): four consecutive rows of a column at a time.  All of first's reads
    // are under way before the first of body's writes, which the compiler could not know to be apart from them.
    template <typename G, typename F> static __device__ __forceinline__ void each(const Acc &acc, G &&first, F &&body)
    {
        const int lane = threadIdx.x & 63, group = (threadIdx.x >> 6) / (WM * WN), wave = (threadIdx.x >> 6) % (WM * WN);
        const int row = (wave / WN) * BI * 16 + (lane >> 4) * 4, column = (wave % WN) * BJ * 16 + (lane & 15);
        if constexpr (KG > 1) {
            if (group >= BI * BJ) return;
            float v[4] = {acc[0][0][0], acc[0][0][1], acc[0][0][2], acc[0][0][3]};
            const int r = row + group / BJ * 16, c = column + group % BJ * 16;
            body(r, c, v, first(r, c));
        } else {
            decltype(first(0, 0)) had[BI][BJ];
#pragma unroll
            for (int i = 0; i < BI; ++i)
#pragma unroll
                for (int j = 0; j < BJ; ++j) had[i][j] = first(row + i * 16, column + j * 16);
#pragma unroll
            for (int i = 0; i < BI; ++i)
#pragma unroll
                for (int j = 0; j < BJ; ++j) {
                    float v[4] = {acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3]};
                    body(row + i * 16, column + j * 16, v, had[i][j]);
                }
        }
    }
};

// Four lanes that hold four rows of a column each, columns side by side, come to hold four columns of a row each: the lane's own row is
// its place among the four.  The same call takes them back.
__device__ __forceinline__ void quad_transpose(float (&v)[4])
{
    const bool odd = threadIdx.x & 1, upper = threadIdx.x & 2;
#pragma unroll
    for (int k = 0; k < 4; k += 2) {
        const float got = dpp_move<0xB1>(odd ? v[k] : v[k + 1]);
        if (odd) v[k] = got; else v[k + 1] = got;
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const float got = dpp_move<0x4E>(upper ? v[k] : v[k + 2]);
        if (upper) v[k] = got; else v[k + 2] = got;
    }
}

// Workgroup g runs on XCD g mod 8, and every XCD has an L2 of its own: tiles that share operands, which follow one another, go to one XCD.
__device__ __forceinline__ uint32_t tile_of_workgroup()
{
    constexpr uint32_t XCDS = 8;
    const uint32_t x = blockIdx.x % XCDS, each = gridDim.x / XCDS, rest = gridDim.x % XCDS;
    return x * each + min(x, rest) + blockIdx.x / XCDS;
}

// Tile t of the lower half, row by row: (row, column), column <= row.
__device__ __forceinline__ void half_tile(uint32_t t, int32_t &row, int32_t &column)
{
    uint32_t r = (uint32_t)((sqrtf(8.f * (float)t + 1.f) - 1.f) * 0.5f);
    while ((r + 1) * (r + 2) / 2 <= t) ++r;
    while (r * (r + 1) / 2 > t) --r;
    row = (int32_t)r;
    column = (int32_t)(t - r * (r + 1) / 2);
}

// A = X X^T (POLY false), P = b f^2 A + c f^4 A^2 (POLY true): the tiles of the lower half, and their reflections.  (4,096 x 4,096 bf16, us: 194 and 208, 1,060 and 990 TFLOP/s of three
// products; six of 1,024 x 4,096 129 and 46, 600 and 420.)
template <typename Prod, bool POLY>
__global__ void __launch_bounds__(Prod::THREADS) update_half_kernel(Group g, bool first)
{
    extern __shared__ __align__(16) uint8_t lds_bytes[];
    uint32_t t;
    const Matrix &m = g.mat[matrix_of(g.half, tile_of_workgroup(), t)];
    int32_t ti, tj;
    half_tile(t, ti, tj);
    const f16 *from = POLY ? m.a : m.xr;
    f16 *to = POLY ? m.p : m.a;
    typename Prod::Acc acc;
    Prod::run({from, ti * Prod::TILE, m.n_pad}, {from, tj * Prod::TILE, m.n_pad}, (int32_t)row_length(POLY ? m.n_pad : m.m_pad), reinterpret_cast<f16 *>(lds_bytes), acc);
    float cb = NS_B, cc = NS_C * UNSCALE;
    if (POLY && first) {
        const float f = *m.factor;
        cb *= f * f;
        cc *= f * f * f * f;
    }
    // Whole quads of lanes are inside or outside: sides are padded to multiples of 64.
    const auto inside = [&](int32_t i, int32_t j) { return i < m.n_pad && j - (int32_t)(threadIdx.x & 3) < m.n_pad; };
    struct Four { f16x4 hi, lo; };
    const auto first_of = [&](int r, int c) {                     // A from its reflection, which has the four side by side
        const int32_t i = ti * Prod::TILE + r, j = tj * Prod::TILE + c;
        Four a = {};
        if (POLY && inside(i, j)) {
            const f16 *from_a = m.a + place(j, i, m.n_pad);
            a.hi = *reinterpret_cast<const f16x4 *>(from_a);
            a.lo = *reinterpret_cast<const f16x4 *>(from_a + LO);
        }
        return a;
    };
    Prod::each(acc, first_of, [&](int r, int c, float (&v)[4], const Four &a) {
        const int32_t i = ti * Prod::TILE + r, j = tj * Prod::TILE + c;
        if (!inside(i, j)) return;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = POLY ? cb * ((float)a.hi[e] + (float)a.lo[e]) + cc * v[e] : v[e] * UNSCALE;
        if (ti != tj) put(to + place(j, i, m.n_pad), v);
        quad_transpose(v);
        put(to + place(i + (int32_t)(threadIdx.x & 3), j & ~3, m.n_pad), v);
    });
}

// X <- f (a X + P X); behind the last step the result goes out instead.  What a tile's results read and write (16 bytes an element) overlaps with another tile's
// product where two share a compute unit.  (4,096 x 4,096 bf16, us: 394, 1,050 TFLOP/s of three products; six of 1,024 x 4,096 230, 670 TFLOP/s beside 2.2 TB/s.)  Reads of X ahead of the
// product gained nothing (1999 x 517 fp32, us: 17.6 so, 18.4 ahead).
template <typename T, typename Prod, bool LAST, bool MUON>
__global__ void __launch_bounds__(Prod::THREADS) update_apply_kernel(Group g, uint32_t step)
{
    extern __shared__ __align__(16) uint8_t lds_bytes[];
    uint32_t t;
    const Matrix &m = g.mat[matrix_of(g.whole, tile_of_workgroup(), t)];
    // Eight columns of tiles at a time, row by row: what an XCD works on at once is about square, and reads the fewest rows of P and columns of X.
    constexpr uint32_t ABREAST = 8;
    const uint32_t down = ((uint32_t)m.n_pad + Prod::TILE - 1) / Prod::TILE, across = ((uint32_t)m.m_pad + Prod::TILE - 1) / Prod::TILE;
    const uint32_t band = t / (down * ABREAST), in_band = t - band * down * ABREAST, width = min(ABREAST, across - band * ABREAST);
    const int32_t ti = (int32_t)(in_band / width), tj = (int32_t)(band * ABREAST + in_band % width);
    typename Prod::Acc acc;
    Prod::run({m.p, ti * Prod::TILE, m.n_pad}, {m.xt[step & 1], tj * Prod::TILE, m.m_pad}, (int32_t)row_length(m.n_pad), reinterpret_cast<f16 *>(lds_bytes), acc);
    f16 *next = m.xt[(step & 1) ^ 1];
    const float f = step == 0 ? *m.factor : 1.f;
    const float grow = MUON ? g.lr * sqrtf(fmaxf(1.f, (float)m.u.rows / (float)m.u.cols)) : 0.f;
    const int32_t mine = threadIdx.x & 3;                          // this lane's place in its quad, all of which is inside or outside
    const auto inside = [&](int32_t i, int32_t j) { return i < m.n_pad && j - mine < m.m_pad; };
    // Where four results go that lie side by side: along X's rows, or, in the last step, along its columns where X is the transpose.
    struct Place { int32_t row, col, n; };
    const auto goes = [&](int32_t i0, int32_t j) {
        const int32_t row = m.tall ? j : i0 + mine, col = m.tall ? i0 : j & ~3;
        return Place{row, col, row < (int32_t)m.u.rows ? min(4, (int32_t)m.u.cols - col) : 0};
    };
    struct Before { f32x4 x; float w[MUON ? 4 : 1]; };
    const auto first_of = [&](int r, int c) {
        const int32_t i0 = ti * Prod::TILE + r, j = tj * Prod::TILE + c;
        Before b = {};
        if (!inside(i0, j)) return b;
        b.x = *reinterpret_cast<const f32x4 *>(m.x + (uint64_t)(i0 + mine) * m.m_pad + (j & ~3));
        if constexpr (MUON) {
            const Place to = goes(i0, j);
            const T *w = row_at<T>(m.u.weight, m.u.weight_stride, to.row) + to.col;
            if (to.n == 4) {
                load_pack(w, b.w);
            } else {
#pragma unroll
                for (int e = 0; e < 3; ++e) b.w[e] = e < to.n ? (float)w[e] : 0.f;
            }
        }
        return b;
    };
    Prod::each(acc, first_of, [&](int r, int c, float (&v)[4], const Before &b) {
        const int32_t i0 = ti * Prod::TILE + r, j = tj * Prod::TILE + c;
        if (!inside(i0, j)) return;
        quad_transpose(v);                                         // this lane's row of X, four columns
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = f * (NS_A * b.x[e] + v[e] * (UNSCALE * UNSCALE));
        if constexpr (LAST) {
            if (m.tall) quad_transpose(v);
            const Place to = goes(i0, j);
            T *out = row_at<T>(m.u.out, m.u.out_stride, to.row) + to.col;
            if constexpr (MUON)
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = g.keep * b.w[e] - grow * v[e];
            if (to.n == 4) {
                store_pack(out, v);
            } else {
#pragma unroll
                for (int e = 0; e < 3; ++e)
                    if (e < to.n) out[e] = (T)v[e];
            }
        } else {
            *reinterpret_cast<f32x4 *>(m.x + (uint64_t)(i0 + mine) * m.m_pad + (j & ~3)) = f32x4{v[0], v[1], v[2], v[3]};
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] *= SCALE;
            put(m.xr + place(i0 + mine, j & ~3, m.m_pad), v);
            quad_transpose(v);
            put(next + place(j, i0, m.n_pad), v);
        }
    });
}

// ---------------------------------------------------------------- small matrices
// Matrices of up to 64 x TINY_WIDE (but for fp32 ones of few rows), one workgroup each, all of it in one launch (47 x 256 bf16, us: 25 so, 78 by 17 launches).  Each of 16 waves keeps strips of 16
// columns of X in registers, laid out as matrix operations leave their results: a lane has a column, and of each block of 16 rows the
// four from 4 (lane / 16) on.  P X needs X with eight rows of a column to a lane, and which eight is free as long as P is read to match: a lane's fours
// of two blocks, so that X never leaves the registers for it.  For X X^T its rows go through LDS, as A and P do, in two parts always (products cost little here).
// Bound by the latency of LDS and of four barriers a step.
constexpr int TINY_THREADS = 1024, TINY_WAVES = 16;
constexpr int TINY_STRIPS = TINY_WIDE / 16 / TINY_WAVES;           // of a wave
constexpr int TINY_LDS = 64 * TINY_WIDE * 4 + 64 * 64 * 4;         // X, and A or P

// A row's 16-byte chunks in LDS, in an order that depends on the row: 16 rows of one chunk lie on all banks.
__device__ __forceinline__ f16 *tiny_at(f16 *base, int row, uint32_t length, uint32_t number)
{
    return base + (uint32_t)row * length + ((number / 8) ^ (uint32_t)(row & 15)) * 8 + number % 8;
}

__device__ __forceinline__ void tiny_put(f16 *base, int row, uint32_t length, uint32_t number, const float (&v)[4])
{
    f16x4 h, l;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        h[e] = (f16)v[e];
        l[e] = (f16)(v[e] - (float)h[e]);
    }
    *reinterpret_cast<f16x4 *>(tiny_at(base, row, length, number)) = h;
    *reinterpret_cast<f16x4 *>(tiny_at(base, row, length, number + LO)) = l;
}

// The product of 16 rows of L and 16 of R (both in LDS, K numbers of both parts a row).
__device__ __forceinline__ f32x4 tiny_product(f16 *l, int row_l, f16 *r, int row_r, uint32_t K)
{
    const int lane = threadIdx.x & 63;
    row_l += lane & 15;
    row_r += lane & 15;
    f32x4 hh = {0.f, 0.f, 0.f, 0.f}, lh = hh, hl = hh;              // three chains: an operation waits for the one before it in its chain
    for (uint32_t k = 0; k < K; k += 64) {
        const uint32_t at = k + (uint32_t)(lane >> 4) * 8;
        const f16x8 lhi = *reinterpret_cast<const f16x8 *>(tiny_at(l, row_l, K, at)), llo = *reinterpret_cast<const f16x8 *>(tiny_at(l, row_l, K, at + LO));
        const f16x8 rhi = *reinterpret_cast<const f16x8 *>(tiny_at(r, row_r, K, at)), rlo = *reinterpret_cast<const f16x8 *>(tiny_at(r, row_r, K, at + LO));
        hh = __builtin_amdgcn_mfma_f32_16x16x32_f16(lhi, rhi, hh, 0, 0, 0);
        lh = __builtin_amdgcn_mfma_f32_16x16x32_f16(llo, rhi, lh, 0, 0, 0);
        hl = __builtin_amdgcn_mfma_f32_16x16x32_f16(lhi, rlo, hl, 0, 0, 0);
    }
    return hh + (lh + hl);
}

template <typename T, bool MUON>
__global__ void __launch_bounds__(TINY_THREADS) update_tiny_kernel(Group g, uint32_t steps)
{
    extern __shared__ __align__(16) uint8_t lds_bytes[];
    __shared__ double part[TINY_WAVES];
    const Matrix &m = g.mat[blockIdx.x];
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), lane = threadIdx.x & 63;
    f16 *rows = reinterpret_cast<f16 *>(lds_bytes), *square = rows + 64 * TINY_WIDE * 2;
    const uint32_t length = row_length(m.m_pad);
    // Where element e of block b of strip s is in X.
    const auto row_of = [&](int b, int e) { return b * 16 + (lane >> 4) * 4 + e; };
    const auto column_of = [&](int s) { return (wave + s * TINY_WAVES) * 16 + (lane & 15); };
    // body(strip, block, element, row and column of G) for what is inside; all reads of a kind are under way before the first write, which the compiler could
    // not know to be apart from them.
    const auto each = [&](auto &&body) {
#pragma unroll
        for (int s = 0; s < TINY_STRIPS; ++s)
#pragma unroll
            for (int b = 0; b < 4; ++b)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int32_t i = row_of(b, e), j = column_of(s);
                    if (i < m.n && j < m.m) body(s, b, e, m.tall ? j : i, m.tall ? i : j);
                }
    };
    float x[TINY_STRIPS][4][4] = {};
    each([&](int s, int b, int e, int32_t r, int32_t c) { x[s][b][e] = (float)row_at<T>(m.u.grad, m.u.grad_stride, r)[c]; });
    if (MUON) {
        float next[TINY_STRIPS][4][4] = {};
        each([&](int s, int b, int e, int32_t r, int32_t c) { next[s][b][e] = row_at<float>(m.u.momentum, m.u.momentum_stride, r)[c]; });
        each([&](int s, int b, int e, int32_t r, int32_t c) {
            const float v = g.momentum * next[s][b][e] + x[s][b][e];
            row_at<float>(m.u.momentum_out, m.u.momentum_out_stride, r)[c] = v;
            x[s][b][e] = update_of(g, x[s][b][e], v);
        });
    }
    double sum = 0.0;
#pragma unroll
    for (int s = 0; s < TINY_STRIPS; ++s)
#pragma unroll
        for (int b = 0; b < 4; ++b)
#pragma unroll
            for (int e = 0; e < 4; ++e) sum += (double)x[s][b][e] * (double)x[s][b][e];
    for (int k = 1; k < 64; k <<= 1) sum += __shfl_xor(sum, k);
    if (lane == 0) part[wave] = sum;
    __syncthreads();
    sum = 0.0;
    for (int k = 0; k < TINY_WAVES; ++k) sum += part[k];
    int e2 = 0;
    float f = factor_of(sqrt(sum), g.eps, e2);
#pragma unroll
    for (int s = 0; s < TINY_STRIPS; ++s)
#pragma unroll
        for (int b = 0; b < 4; ++b)
#pragma unroll
            for (int e = 0; e < 4; ++e) x[s][b][e] = ldexpf(x[s][b][e], -e2) * SCALE;          // as the operands are
    // What lies beyond X's rows stays zero, and is not computed: the vector unit's instructions are what a step takes time for, four waves' on each.
    const int blocks = (m.n + 15) / 16, bi = (wave / 4) * 16, bj = (wave % 4) * 16;
    const bool has_block = max(wave / 4, wave % 4) < blocks;
    const uint32_t mirror = (uint32_t)(bi + (lane >> 4) * 4), mirror_at = mirror + (mirror & ~31u);
    float v[4] = {0.f, 0.f, 0.f, 0.f};
    tiny_put(square, bj + (lane & 15), 128, mirror_at, v);
    for (uint32_t step = 0; step < steps; ++step) {
        // X's rows into LDS: strips of columns that m_pad has
#pragma unroll
        for (int s = 0; s < TINY_STRIPS; ++s)
            if ((wave + s * TINY_WAVES) * 16 < m.m_pad)
#pragma unroll
                for (int b = 0; b < 4; ++b) {
                    float w[4] = {x[s][b][0], x[s][b][1], x[s][b][2], x[s][b][3]};
                    quad_transpose(w);
                    const uint32_t column = (uint32_t)column_of(s) & ~3u;
                    tiny_put(rows, row_of(b, lane & 3), length, column + (column & ~31u), w);
                }
        __syncthreads();
        // A: a block of 16 x 16 a wave.  It is symmetric, and is written by columns.
        f32x4 p = {0.f, 0.f, 0.f, 0.f};
        if (has_block) {
            p = tiny_product(rows, bi, rows, bj, length);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = p[e] * UNSCALE;
            tiny_put(square, bj + (lane & 15), 128, mirror_at, v);
        }
        __syncthreads();
        if (has_block) p = tiny_product(square, bi, square, bj, 128);
        __syncthreads();                                           // A is read
        if (has_block) {
            const float cb = NS_B * f * f, cc = NS_C * UNSCALE * f * f * f * f;
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = cb * v[e] + cc * p[e];
            tiny_put(square, bj + (lane & 15), 128, mirror_at, v);
        }
        __syncthreads();
#pragma unroll
        for (int s = 0; s < TINY_STRIPS; ++s) {
            if ((wave + s * TINY_WAVES) * 16 >= m.m) continue;
            f16x8 xh[2], xl[2];                                    // slices of 32 rows: a lane's fours of two blocks
#pragma unroll
            for (int q = 0; q < 2; ++q)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float w = x[s][q * 2 + e / 4][e % 4];
                    xh[q][e] = (f16)w;
                    xl[q][e] = (f16)(w - (float)xh[q][e]);
                }
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                if (b >= blocks) continue;
                f32x4 big = {0.f, 0.f, 0.f, 0.f}, small = big;
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    if (q * 2 >= blocks) continue;
                    f16x8 ph, pl;
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        const uint32_t at = (uint32_t)q * 64 + (uint32_t)half * 16 + (uint32_t)(lane >> 4) * 4;
                        const f16x4 h = *reinterpret_cast<const f16x4 *>(tiny_at(square, b * 16 + (lane & 15), 128, at));
                        const f16x4 l = *reinterpret_cast<const f16x4 *>(tiny_at(square, b * 16 + (lane & 15), 128, at + LO));
#pragma unroll
                        for (int e = 0; e < 4; ++e) { ph[half * 4 + e] = h[e]; pl[half * 4 + e] = l[e]; }
                    }
                    big = __builtin_amdgcn_mfma_f32_16x16x32_f16(ph, xh[q], big, 0, 0, 0);
                    small = __builtin_amdgcn_mfma_f32_16x16x32_f16(pl, xh[q], small, 0, 0, 0);
                    small = __builtin_amdgcn_mfma_f32_16x16x32_f16(ph, xl[q], small, 0, 0, 0);
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) x[s][b][e] = f * (NS_A * x[s][b][e] + (big[e] + small[e]) * UNSCALE);
            }
        }
        f = 1.f;
    }
#pragma unroll
    for (int s = 0; s < TINY_STRIPS; ++s)
#pragma unroll
        for (int b = 0; b < 4; ++b)
#pragma unroll
            for (int e = 0; e < 4; ++e) x[s][b][e] *= UNSCALE;
    const float grow = MUON ? g.lr * sqrtf(fmaxf(1.f, (float)m.u.rows / (float)m.u.cols)) : 0.f;
    if (MUON) {
        float w[TINY_STRIPS][4][4];
        each([&](int s, int b, int e, int32_t r, int32_t c) { w[s][b][e] = (float)row_at<T>(m.u.weight, m.u.weight_stride, r)[c]; });
        each([&](int s, int b, int e, int32_t r, int32_t c) { row_at<T>(m.u.out, m.u.out_stride, r)[c] = (T)(g.keep * w[s][b][e] - grow * x[s][b][e]); });
    } else {
        each([&](int s, int b, int e, int32_t r, int32_t c) { row_at<T>(m.u.out, m.u.out_stride, r)[c] = (T)x[s][b][e]; });
    }
}

// ---------------------------------------------------------------- narrow matrices
// Of few rows A and P have so few entries that their roundings do not average out, as they do over the singular values of larger matrices: with operands of 22 bits and sums of 32, fp32 results
// were 1e-6 to 5e-6 off, two to three times as much as by fp32 products (see narrow in rg_launch.h; to 16 bits a result is rounded 50 times as far and more).  But there all of it is cheap but X itself, and every X is a
// polynomial of A in front of the first one: with B = U U^T, r = 1 / (|U| + eps), A = r^2 B,
//     Q = a + b A + c A^2,   M <- Q M,   A <- Q^2 A,   and at last X = r M U.
// These few n x n products are made in 64 bits, and X is rounded once: results are off by that rounding alone, 3e-8.  Everything is symmetric and commutes, so that
// only the lower half of a product is computed, and both operands are read along their rows.  A direction that U lacks has an A of 1e-16 instead of none, of either sign, which grows 12 times a step: up to
// NARROW_STEPS steps are taken at once, in which that stays nothing, and then X is kept, in fp32, and B made of it again.
//
// One launch sums B up, by parts of X's columns; in another every workgroup adds the parts up in their order, makes M, and has its own columns of X.  (All workgroups make the same M, which takes as long as one that the
// others would wait for, and a launch less.)  What is up to TINY_WIDE has one part, and one workgroup and one launch for all of it.  Bound by the 64-bit matrix operations, of about 115 cycles each on
// a vector unit, and the latency of five barriers a step (16 x 256, us: 16, of which 1.6 a step; 32 x 256 24, 2.5 a step;
// 48 x 4,096 48, 16 x 16,384 28; with operands of 22 bits 17, 20, 116 and 304).
typedef double f64x4 __attribute__((ext_vector_type(4)));
constexpr double EXACT_A = 3.4445, EXACT_B = -4.7750, EXACT_C = 2.0315;
constexpr int NARROW_THREADS = 1024, NARROW_WAVES = 16;
constexpr uint32_t NARROW_STEPS = 6;
constexpr int NARROW_PASS = 256;         // columns of U in LDS at a time

struct Narrow {
    int n, m, blocks, length, tiles;     // blocks of 16 rows; of a row in LDS; tiles of the lower half
    __device__ __forceinline__ explicit Narrow(const Matrix &a) : n(a.n), m(a.m), blocks((a.n + 15) / 16), length(16 * (blocks | 1)), tiles(blocks * (blocks + 1) / 2) {}
};
// Rows of 16 or 48 numbers: two rows of 16 numbers of 64 bits, or four of 32, lie on all banks once.
constexpr int NARROW_GRAM_LDS = NARROW_PASS * 48 * 4, NARROW_LDS = std::max(NARROW_GRAM_LDS, 3 * 48 * 48 * 8);
static_assert(UPDATE_NARROW_SIDE == 48, "three blocks of rows at most");

// Where element e of a lane lies in a tile of 16 x 16 that a 64-bit matrix operation leaves.
__device__ __forceinline__ int row64(int e) { return 4 * e + (((int)threadIdx.x & 63) >> 4); }

// U at (row of X, column of X).
__device__ __forceinline__ float narrow_at(const Group &g, const Matrix &m, bool first, int i, int c)
{
    if (!first) return m.x[(uint64_t)i * m.m_pad + c];
    const int r = m.tall ? c : i, k = m.tall ? i : c;
    const float v = row_at<float>(m.u.grad, m.u.grad_stride, r)[k];
    return g.muon ? update_of(g, v, row_at<float>(m.u.momentum_out, m.u.momentum_out_stride, r)[k]) : v;
}

// The part's share of B, and (muon) the new momentum of its columns.
__device__ __forceinline__ void narrow_gram(const Group &g, const Matrix &m, bool first, uint32_t part, uint8_t *lds_bytes)
{
    const Narrow s(m);
    float *columns = reinterpret_cast<float *>(lds_bytes);         // [NARROW_PASS][length]: a column of U after another
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), lane = threadIdx.x & 63;
    const int slices = NARROW_WAVES / s.tiles, slice = wave / s.tiles, tile = wave % s.tiles, quads = s.blocks * 4;      // a tile has several waves, each with its own columns
    int32_t ti, tj;
    half_tile((uint32_t)tile, ti, tj);
    f64x4 acc = {0.0, 0.0, 0.0, 0.0};
    const int each = (int)narrow_part((uint64_t)s.m), from = (int)part * each, to = min(s.m, from + each);
    for (int c0 = from; c0 < to; c0 += NARROW_PASS) {
        const int count = min(NARROW_PASS, to - c0);
        // Four rows of a column a thread; neighbours along G's rows.
        for (int u = threadIdx.x; u < NARROW_PASS * quads; u += NARROW_THREADS) {
            const int quad = m.tall ? u % quads : u / NARROW_PASS, c = m.tall ? u / quads : u % NARROW_PASS;
            f32x4 v = {0.f, 0.f, 0.f, 0.f};
            if (c < count) {
                if (first && g.muon) {
                    float old[4] = {}, grad[4] = {};
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int i = quad * 4 + e, r = m.tall ? c0 + c : i, k = m.tall ? i : c0 + c;
                        if (i >= s.n) continue;
                        grad[e] = row_at<float>(m.u.grad, m.u.grad_stride, r)[k];
                        old[e] = row_at<float>(m.u.momentum, m.u.momentum_stride, r)[k];
                    }
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int i = quad * 4 + e, r = m.tall ? c0 + c : i, k = m.tall ? i : c0 + c;
                        if (i >= s.n) continue;
                        const float next = g.momentum * old[e] + grad[e];
                        row_at<float>(m.u.momentum_out, m.u.momentum_out_stride, r)[k] = next;
                        v[e] = update_of(g, grad[e], next);
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (quad * 4 + e < s.n) v[e] = narrow_at(g, m, first, quad * 4 + e, c0 + c);
                }
            }
            *reinterpret_cast<f32x4 *>(columns + c * s.length + quad * 4) = v;
        }
        __syncthreads();
        if (slice < slices)
            for (int k = slice * 4; k < count; k += slices * 4) {
                const float *at = columns + (k + (lane >> 4)) * s.length + (lane & 15);
                acc = __builtin_amdgcn_mfma_f64_16x16x4f64((double)at[ti * 16], (double)at[tj * 16], acc, 0, 0, 0);
            }
        __syncthreads();
    }
    double *sums = reinterpret_cast<double *>(lds_bytes);
    if (slice < slices)
#pragma unroll
        for (int e = 0; e < 4; ++e) sums[(slice * s.tiles + tile) * 256 + e * 64 + lane] = acc[e];
    __syncthreads();
    const int all = s.tiles * 256;
    for (int q = threadIdx.x; q < all; q += NARROW_THREADS) {
        double v = sums[q];
        for (int k = 1; k < slices; ++k) v += sums[k * all + q];
        m.sums[(uint64_t)part * all + q] = v;
    }
    __syncthreads();
}

__global__ void __launch_bounds__(NARROW_THREADS) narrow_gram_kernel(Group g, bool first)
{
    extern __shared__ __align__(16) uint8_t lds_bytes[];
    uint32_t part;
    const Matrix &m = g.mat[matrix_of(g.starts, blockIdx.x, part)];
    narrow_gram(g, m, first, part, lds_bytes);
}

// Tile (ti, tj) of the product of two symmetric matrices in LDS.  All operands are read ahead of the operations, which are in two chains: each waits for the one before it in its chain.
template <int BLOCKS> __device__ __forceinline__ f64x4 narrow_product(const double *x, const double *y, int ti, int tj)
{
    constexpr int LENGTH = 16 * (BLOCKS | 1);
    const int lane = threadIdx.x & 63, at = (lane >> 4) * LENGTH + (lane & 15);
    double l[BLOCKS * 4], r[BLOCKS * 4];
#pragma unroll
    for (int k = 0; k < BLOCKS * 4; ++k) {
        l[k] = x[at + k * 4 * LENGTH + ti * 16];
        r[k] = y[at + k * 4 * LENGTH + tj * 16];
    }
    f64x4 acc[2] = {{0.0, 0.0, 0.0, 0.0}, {0.0, 0.0, 0.0, 0.0}};
#pragma unroll
    for (int k = 0; k < BLOCKS * 4; ++k) acc[k & 1] = __builtin_amdgcn_mfma_f64_16x16x4f64(l[k], r[k], acc[k & 1], 0, 0, 0);
    return acc[0] + acc[1];
}
__device__ __forceinline__ f64x4 narrow_product(const double *x, const double *y, int ti, int tj, const Narrow &s)
{
    switch (s.blocks) {
    case 1: return narrow_product<1>(x, y, ti, tj);
    case 2: return narrow_product<2>(x, y, ti, tj);
    default: return narrow_product<3>(x, y, ti, tj);
    }
}

// A tile and its reflection.
__device__ __forceinline__ void narrow_put(double *to, int ti, int tj, const Narrow &s, const f64x4 &v)
{
    const int j = tj * 16 + ((int)threadIdx.x & 15);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int i = ti * 16 + row64(e);
        to[i * s.length + j] = v[e];
        if (ti != tj) to[j * s.length + i] = v[e];
    }
}

// ALONE: the matrix' only workgroup, which makes B too.
template <bool MUON, bool ALONE>
__global__ void __launch_bounds__(NARROW_THREADS) narrow_apply_kernel(Group g, uint32_t steps, bool first, bool last)
{
    extern __shared__ __align__(16) uint8_t lds_bytes[];
    uint32_t group;
    const Matrix &m = g.mat[matrix_of(g.whole, blockIdx.x, group)];
    if (ALONE) narrow_gram(g, m, first, 0, lds_bytes);
    const Narrow s(m);
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), lane = threadIdx.x & 63, all = s.tiles * 256;
    const int size = s.blocks * 16 * s.length;
    double *a = reinterpret_cast<double *>(lds_bytes), *q = a + size, *p = q + size;                     // B and then A, Q, M
    for (int x = threadIdx.x; x < all; x += NARROW_THREADS) {
        double v = 0.0;
        for (uint32_t k = 0; k < m.sum_blocks; ++k) v += m.sums[(uint64_t)k * all + x];
        int32_t ti, tj;
        half_tile((uint32_t)x / 256, ti, tj);
        const int i = ti * 16 + row64((x >> 6) & 3), j = tj * 16 + (x & 15);
        a[i * s.length + j] = v;
        if (ti != tj) a[j * s.length + i] = v;
    }
    __syncthreads();
    double r = 1.0;
    if (first) {
        double squares = lane < s.n ? a[lane * s.length + lane] : 0.0;
        for (int k = 1; k < 64; k <<= 1) squares += __shfl_xor(squares, k);
        r = squares < INFINITY ? 1.0 / (sqrt(squares) + (double)g.eps) : NAN;                            // nothing over nothing is a NaN by B
    }
    double scale = r * r;                                          // of the first step, whose A is this times B
    for (uint32_t step = 0; step < steps; ++step) {
        const bool more = step + 1 < steps;
        if (wave < s.tiles) {
            int32_t ti, tj;
            half_tile((uint32_t)wave, ti, tj);
            f64x4 v = narrow_product(a, a, ti, tj, s);
            const int j = tj * 16 + (lane & 15);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int i = ti * 16 + row64(e);
                v[e] = (i == j ? EXACT_A : 0.0) + scale * (EXACT_B * a[i * s.length + j] + scale * EXACT_C * v[e]);
            }
            narrow_put(q, ti, tj, s, v);
            if (step == 0) narrow_put(p, ti, tj, s, v);
        }
        __syncthreads();
        // Q A and Q M, in the places of A and M: a wave a tile, 12 of them at most
        const int from = more ? 0 : s.tiles, units = s.tiles * (step == 0 ? 1 : 2);
        const int unit = from + wave;
        int32_t ti = 0, tj = 0;
        f64x4 v = {0.0, 0.0, 0.0, 0.0};
        if (unit < units) {
            half_tile((uint32_t)(unit % s.tiles), ti, tj);
            v = narrow_product(q, unit < s.tiles ? a : p, ti, tj, s);
        }
        __syncthreads();
        if (unit < units) narrow_put(unit < s.tiles ? a : p, ti, tj, s, v);
        __syncthreads();
        if (!more) break;
        if (wave < s.tiles) {
            half_tile((uint32_t)wave, ti, tj);
            v = narrow_product(q, a, ti, tj, s);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] *= scale;
        }
        __syncthreads();
        if (wave < s.tiles) narrow_put(a, ti, tj, s, v);
        __syncthreads();
        scale = 1.0;
    }
    // X = r M U, 16 columns of it a wave at a time: it reads all of them before it writes the first, which may be in their place.
    const float grow = MUON ? g.lr * sqrtf(fmaxf(1.f, (float)m.u.rows / (float)m.u.cols)) : 0.f;
    const int each = ALONE ? s.m : (int)narrow_share((uint64_t)s.m), to = min(s.m, ((int)group + 1) * each);
    for (int c0 = (int)group * each + wave * 16; c0 < to; c0 += NARROW_WAVES * 16) {
        const int c = c0 + (lane & 15);
        float u[12];
#pragma unroll
        for (int k = 0; k < 12; ++k) {
            const int i = k * 4 + (lane >> 4);
            u[k] = i < s.n && c < to ? narrow_at(g, m, first, i, c) : 0.f;
        }
        for (int t = 0; t < s.blocks; ++t) {
            f64x4 v = {0.0, 0.0, 0.0, 0.0};
#pragma unroll
            for (int k = 0; k < 12; ++k)
                if (k < s.blocks * 4) v = __builtin_amdgcn_mfma_f64_16x16x4f64(p[(k * 4 + (lane >> 4)) * s.length + t * 16 + (lane & 15)], (double)u[k], v, 0, 0, 0);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int i = t * 16 + row64(e), row = m.tall ? c : i, col = m.tall ? i : c;
                if (i >= s.n || c >= to) continue;
                const float x = (float)(r * v[e]);
                if (!last) m.x[(uint64_t)i * m.m_pad + c] = x;
                else if constexpr (MUON) row_at<float>(m.u.out, m.u.out_stride, row)[col] = g.keep * row_at<float>(m.u.weight, m.u.weight_stride, row)[col] - grow * x;
                else row_at<float>(m.u.out, m.u.out_stride, row)[col] = x;
            }
        }
    }
}

// ---------------------------------------------------------------- launches
// LDS beyond 64 KB has to be asked for, once per kernel and device.
template <typename K> rg_status allow_lds(K kernel, int bytes, std::atomic<uint64_t> &known)
{
    if (bytes <= 64 * 1024) return RG_OK;
    int dev = 0;
    RG_HIP(hipGetDevice(&dev));
    const uint64_t bit = dev >= 0 && dev < 64 ? 1ull << dev : 0;
    if (known.load(std::memory_order_relaxed) & bit) return RG_OK;
    RG_HIP(hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, bytes));
    known.fetch_or(bit, std::memory_order_relaxed);
    return RG_OK;
}

template <typename Prod, bool POLY> rg_status launch_half(const Group &g, uint32_t grid, uint32_t step, hipStream_t st)
{
    static std::atomic<uint64_t> known{0};
    RG_TRY(allow_lds(update_half_kernel<Prod, POLY>, Prod::LDS_BYTES, known));
    hipLaunchKernelGGL((update_half_kernel<Prod, POLY>), dim3(grid), dim3(Prod::THREADS), Prod::LDS_BYTES, st, g, step == 0);
    RG_HIP(hipGetLastError());
    return RG_OK;
}

template <typename T, typename Prod, bool LAST, bool MUON> rg_status launch_apply(const Group &g, uint32_t grid, uint32_t step, hipStream_t st)
{
    static std::atomic<uint64_t> known{0};
    RG_TRY(allow_lds(update_apply_kernel<T, Prod, LAST, MUON>, Prod::LDS_BYTES, known));
    hipLaunchKernelGGL((update_apply_kernel<T, Prod, LAST, MUON>), dim3(grid), dim3(Prod::THREADS), Prod::LDS_BYTES, st, g, step);
    RG_HIP(hipGetLastError());
    return RG_OK;
}

// The tiles.
using Tile32Shared = Product<2, 2, 1, 1, 128, 4, 2>;
using Tile64Shared = Product<2, 4, 2, 1, 128, 4, 2>;
using Tile64 = Product<2, 2, 2, 2, 64, 3>;
using Tile96 = Product<2, 2, 3, 3, 64, 3>;
using Tile128 = Product<2, 4, 4, 2, 64, 3>;
using Tile128Pair = Product<2, 4, 4, 2, 64, 2>;
using Tile192 = Product<2, 4, 6, 3, 64, 3>;

template <typename F> rg_status with_tile(int tile, F &&body)
{
    switch (tile) {
    case 32: return body(Tile32Shared{});
    case UPDATE_TILE_SHARED: return body(Tile64Shared{});
    case 64: return body(Tile64{});
    case 96: return body(Tile96{});
    case 128: return body(Tile128{});
    case UPDATE_TILE_PAIR: return body(Tile128Pair{});
    case 192: return body(Tile192{});
    }
    set_error("no product of tiles of %d", tile);
    return RG_EHIP;
}

struct Shape { uint32_t sums, starts, half, whole; int half_tile, whole_tile; };

template <typename T>
rg_status launch_group(const Group &g, uint32_t steps, const Shape &s, hipStream_t st)
{
    hipLaunchKernelGGL(update_sums_kernel<T>, dim3(s.sums), dim3(256), 0, st, g);
    RG_HIP(hipGetLastError());
    hipLaunchKernelGGL(update_start_kernel<T>, dim3(s.starts), dim3(256), 0, st, g);
    RG_HIP(hipGetLastError());
    for (uint32_t k = 0; k < steps; ++k) {
        RG_TRY(with_tile(s.half_tile, [&](auto p) {
            RG_TRY((launch_half<decltype(p), false>(g, s.half, k, st)));
            return launch_half<decltype(p), true>(g, s.half, k, st);
        }));
        RG_TRY(with_tile(s.whole_tile, [&](auto p) {
            if (k + 1 < steps) return launch_apply<float, decltype(p), false, false>(g, s.whole, k, st);        // T plays no part in it
            return g.muon ? launch_apply<T, decltype(p), true, true>(g, s.whole, k, st) : launch_apply<T, decltype(p), true, false>(g, s.whole, k, st);
        }));
    }
    return RG_OK;
}

template <typename T, bool MUON> rg_status launch_tiny(const Group &g, uint32_t count, uint32_t steps, hipStream_t st)
{
    static std::atomic<uint64_t> known{0};
    RG_TRY(allow_lds(update_tiny_kernel<T, MUON>, TINY_LDS, known));
    hipLaunchKernelGGL((update_tiny_kernel<T, MUON>), dim3(count), dim3(TINY_THREADS), TINY_LDS, st, g, steps);
    RG_HIP(hipGetLastError());
    return RG_OK;
}

template <bool MUON, bool ALONE> rg_status launch_narrow(const Group &g, uint32_t steps, const Shape &s, hipStream_t st)
{
    static_assert(NARROW_GRAM_LDS <= 64 * 1024 && NARROW_LDS <= 64 * 1024, "more has to be asked for");
    for (uint32_t k = 0; k < steps; k += NARROW_STEPS) {
        if (!ALONE) {
            hipLaunchKernelGGL(narrow_gram_kernel, dim3(s.starts), dim3(NARROW_THREADS), NARROW_GRAM_LDS, st, g, k == 0);
            RG_HIP(hipGetLastError());
        }
        hipLaunchKernelGGL((narrow_apply_kernel<MUON, ALONE>), dim3(s.whole), dim3(NARROW_THREADS), NARROW_LDS, st, g, std::min(NARROW_STEPS, steps - k), k == 0, k + NARROW_STEPS >= steps);
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
};

void lay_out(Matrix &m, const rg_update &u, const UpdateKind &kind, Carver &c)
{
    m.u = u;
    m.tall = u.rows > u.cols;
    m.n = (int32_t)(m.tall ? u.cols : u.rows);
    m.m = (int32_t)(m.tall ? u.rows : u.cols);
    m.n_pad = (m.n + UPDATE_PAD - 1) / UPDATE_PAD * UPDATE_PAD;
    m.m_pad = (m.m + UPDATE_PAD - 1) / UPDATE_PAD * UPDATE_PAD;
    const uint64_t nm = (uint64_t)m.n_pad * m.m_pad, nn = (uint64_t)m.n_pad * m.n_pad;
    if (kind.narrow) {
        m.sum_blocks = narrow_parts((uint64_t)m.m);
        const uint64_t blocks = (uint64_t)(m.n + 15) / 16;
        c.take(m.sums, m.sum_blocks * (blocks * (blocks + 1) / 2) * 256);
        c.take(m.x, nm);                                           // where there are more than NARROW_STEPS steps
        return;
    }
    c.take(m.sums, SUM_BLOCKS);
    c.take(m.factor, 1);
    if (kind.tiny) return;                                         // all the rest in registers and LDS
    c.take(m.x, nm);
    for (f16 **p : {&m.xr, &m.xt[0], &m.xt[1]}) c.take(*p, nm * 2);
    for (f16 **p : {&m.a, &m.p}) c.take(*p, nn * 2);
}

UpdateKind kind_of_matrix(const rg_update &u, uint32_t type, int n_cu)
{
    UpdateKind k = update_kind(u.rows, u.cols, true, n_cu);
    k.narrow = type == RG_F32 && narrow(u.rows, u.cols);
    return k;
}

// Groups of matrices of a size class, in order, each with the whole workspace to itself.
struct Options { bool muon, nesterov; float momentum, lr, weight_decay, eps; uint32_t steps; };

template <typename F> rg_status each_group(const rg_update *u, uint32_t n, uint32_t type, F &&body)
{
    int n_cu = 0;
    RG_TRY(compute_units(&n_cu));
    const auto empty = [&](uint32_t k) { return u[k].rows == 0 || u[k].cols == 0; };
    const auto kind_of = [&](uint32_t k) { return kind_of_matrix(u[k], type, n_cu); };
    for (uint32_t first = 0; first < n; ++first) {
        if (empty(first)) continue;
        const UpdateKind kind = kind_of(first);
        bool seen = false;
        for (uint32_t k = 0; k < first && !seen; ++k) seen = !empty(k) && kind_of(k) == kind;
        if (seen) continue;
        const rg_update *picked[RG_UPDATES_PER_LAUNCH];
        uint32_t count = 0;
        for (uint32_t k = first; k < n; ++k) {
            if (empty(k) || !(kind_of(k) == kind)) continue;
            picked[count++] = &u[k];
            if (count == RG_UPDATES_PER_LAUNCH) { RG_TRY(body(kind, n_cu, picked, count)); count = 0; }
        }
        if (count) RG_TRY(body(kind, n_cu, picked, count));
    }
    return RG_OK;
}

template <typename T>
rg_status run_group(const UpdateKind &kind, int n_cu, const rg_update *const *u, uint32_t count, const Options &o, uint8_t *workspace, hipStream_t st)
{
    Group g{};
    g.muon = o.muon; g.nesterov = o.nesterov;
    g.momentum = o.momentum; g.lr = o.lr; g.keep = (float)(1.0 - (double)o.lr * (double)o.weight_decay);
    g.eps = o.eps;
    Carver c{workspace};
    for (uint32_t k = 0; k < count; ++k) lay_out(g.mat[k], *u[k], kind, c);
    Shape s{};
    for (Starts *p : {&g.sums, &g.starts, &g.half, &g.whole})
        for (uint32_t &x : p->first) x = UINT32_MAX;
    if constexpr (std::is_same_v<T, float>)
        if (kind.narrow) {
            for (uint32_t k = 0; k < count; ++k) {
                g.starts.first[k] = s.starts; g.whole.first[k] = s.whole;
                s.starts += g.mat[k].sum_blocks;
                s.whole += kind.tiny ? 1u : narrow_shares((uint64_t)g.mat[k].m);
            }
            if (kind.tiny) return g.muon ? launch_narrow<true, true>(g, o.steps, s, st) : launch_narrow<false, true>(g, o.steps, s, st);
            return g.muon ? launch_narrow<true, false>(g, o.steps, s, st) : launch_narrow<false, false>(g, o.steps, s, st);
        }
    if (kind.tiny) return g.muon ? launch_tiny<T, true>(g, count, o.steps, st) : launch_tiny<T, false>(g, count, o.steps, st);
    const auto tiles = [&](int tile, bool half) {
        uint64_t all = 0;
        for (uint32_t k = 0; k < count; ++k) all += half ? half_tiles(g.mat[k].n_pad, tile_side(tile)) : whole_tiles(g.mat[k].n_pad, g.mat[k].m_pad, tile_side(tile));
        return all;
    };
    const auto pick = [&](int asked, bool half) {
        const auto count_of = [&](int tile) { return tiles(tile, half); };
        return asked == UPDATE_TILE_SHARED ? shared_tile(count_of, n_cu) : asked ? asked : update_tile(count_of, n_cu, kind.split);
    };
    s.half_tile = pick(kind.half_tile, true);
    s.whole_tile = pick(kind.whole_tile, false);
    for (uint32_t k = 0; k < count; ++k) {
        Matrix &m = g.mat[k];
        m.sum_blocks = (uint32_t)std::max<uint64_t>(1, std::min<uint64_t>(SUM_BLOCKS, (uint64_t)m.n * m.m / 4096));
        g.sums.first[k] = s.sums; g.starts.first[k] = s.starts; g.half.first[k] = s.half; g.whole.first[k] = s.whole;
        s.sums += m.sum_blocks;
        s.starts += (uint32_t)whole_tiles(m.n_pad, m.m_pad, 64);
        s.half += (uint32_t)half_tiles(m.n_pad, tile_side(s.half_tile));
        s.whole += (uint32_t)whole_tiles(m.n_pad, m.m_pad, tile_side(s.whole_tile));
    }
    return launch_group<T>(g, o.steps, s, st);
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

// A result in the place of an input has its rows where the input has them.
rg_status check_place(uint32_t k, const char *what, const void *out, uint64_t out_stride, const void *in, uint64_t in_stride, const rg_update &u)
{
    if (out != in || out_stride == in_stride || u.rows <= 1) return RG_OK;
    set_error("matrix %u: %s: in place, but with another stride", k, what);
    return RG_EINVAL;
}

rg_status workspace_of(const rg_update *u, uint32_t n, uint32_t type, uint64_t *bytes)
{
    uint64_t most = 0;
    RG_TRY(each_group(u, n, type, [&](const UpdateKind &kind, int, const rg_update *const *picked, uint32_t count) {
        Carver c{nullptr};
        for (uint32_t k = 0; k < count; ++k) {
            Matrix m;
            lay_out(m, *picked[k], kind, c);
        }
        most = std::max(most, c.used);
        return RG_OK;
    }));
    *bytes = most;
    return RG_OK;
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
        RG_TRY(check_place(k, "out", u[k].out, u[k].out_stride, u[k].grad, u[k].grad_stride, u[k]));
        if (!o.muon) continue;
        RG_TRY(check_array(k, "weight", u[k].weight, u[k].weight_stride, u[k], bytes, false));
        RG_TRY(check_array(k, "momentum", u[k].momentum, u[k].momentum_stride, u[k], 4, false));
        RG_TRY(check_array(k, "momentum_out", u[k].momentum_out, u[k].momentum_out_stride, u[k], 4, true));
        RG_TRY(check_place(k, "out", u[k].out, u[k].out_stride, u[k].weight, u[k].weight_stride, u[k]));
        RG_TRY(check_place(k, "momentum_out", u[k].momentum_out, u[k].momentum_out_stride, u[k].momentum, u[k].momentum_stride, u[k]));
    }
    uint64_t want = 0;
    RG_TRY(workspace_of(u, n, type, &want));
    if (want && (!workspace || reinterpret_cast<uintptr_t>(workspace) % 256)) { set_error("the workspace is null or not aligned to 256 bytes"); return RG_EINVAL; }
    if (workspace_bytes < want) { set_error("the workspace holds %llu bytes of %llu", (unsigned long long)workspace_bytes, (unsigned long long)want); return RG_ERANGE; }
    const hipStream_t st = as_stream(stream);
    uint8_t *ws = static_cast<uint8_t *>(workspace);
    return each_group(u, n, type, [&](const UpdateKind &kind, int n_cu, const rg_update *const *picked, uint32_t count) {
        return type == RG_F32 ? run_group<float>(kind, n_cu, picked, count, o, ws, st) : type == RG_BF16 ? run_group<bf16>(kind, n_cu, picked, count, o, ws, st) : run_group<f16>(kind, n_cu, picked, count, o, ws, st);
    });
}

}  // namespace
}  // namespace rg

using namespace rg;

extern "C" rg_status rg_update_workspace(const rg_update *u, uint32_t n, uint32_t type, uint64_t *bytes)
{
    if (!bytes) { set_error("null argument"); return RG_EINVAL; }
    RG_TRY(check_updates(u, n, type));
    return workspace_of(u, n, type, bytes);
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
