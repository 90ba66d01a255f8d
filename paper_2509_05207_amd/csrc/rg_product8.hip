// Products on rows held in 8 bits: rg_rows8_product, in 8-bit integers with a scale for each row of either side, and its backward pass,
// which takes nothing of the forward pass but the held rows.
#include "rg_internal.h"
#include "rg_elements.h"
#include "rg_launch.h"

#include <atomic>

namespace rg {

namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef bf16 bf16x8 __attribute__((ext_vector_type(8)));

template <typename T> __device__ __forceinline__ T *row_at(void *p, uint64_t stride, int64_t r) { return reinterpret_cast<T *>(static_cast<uint8_t *>(p) + (uint64_t)r * stride); }
template <typename T> __device__ __forceinline__ const T *row_at(const void *p, uint64_t stride, int64_t r) { return reinterpret_cast<const T *>(static_cast<const uint8_t *>(p) + (uint64_t)r * stride); }

// Four results side by side, of which n are inside.
template <typename O> __device__ __forceinline__ void store_four(O *p, const f32x4 &v, int32_t n)
{
    if (n >= 4) {
        const float w[4] = {v[0], v[1], v[2], v[3]};
        store_pack<O, 4>(p, w);
    } else {
#pragma unroll
        for (int e = 0; e < 3; ++e)
            if (e < n) p[e] = (O)v[e];
    }
}

// ---------------------------------------------------------------- y = x w^T + bias
struct ProductArgs {
    const uint8_t *x, *w;
    uint64_t x_stride, w_stride;
    const void *bias;
    uint32_t bias_type;
    uint8_t *y;
    uint64_t y_stride;
    int32_t n_rows, n_outs, n_cols, held_bytes;
    int32_t *partial;                // [splits][n_rows][n_outs to a multiple of 4], or NULL: a sum is done by one workgroup
    int32_t each;                    // steps of 128 codes of a split
    uint32_t tiles;
};

// A chunk of 16 bytes with codes in it may have the scale's four behind them: where that is so, the scales' own bytes have gone into a sum, and are taken off again.
__device__ __forceinline__ bool scale_in_sum(int32_t n_cols) { const int32_t r = n_cols & 15; return r >= 1 && r <= 12; }

__device__ __forceinline__ float bias_at(const ProductArgs &a, int32_t m)
{
    if (!a.bias) return 0.f;
    return a.bias_type == RG_F32 ? static_cast<const float *>(a.bias)[m] : a.bias_type == RG_BF16 ? (float)static_cast<const bf16 *>(a.bias)[m] : (float)static_cast<const f16 *>(a.bias)[m];
}

// A product that is rounded before it goes into a sum or a difference.
__device__ __forceinline__ float rounded(float a, float b)
{
#pragma clang fp contract(off)
    return a * b;
}

__device__ __forceinline__ int32_t sum_of_codes(int32_t sum, uint32_t sx, uint32_t sw, bool scales_in)
{
    return scales_in ? sum - __builtin_amdgcn_sdot4((int)sx, (int)sw, 0, false) : sum;
}

// What a sum of codes stands for: sum s_x s_w + bias, in 64 bits.
__device__ __forceinline__ float wide_value(int32_t sum, uint32_t sx, uint32_t sw, float bias)
{
    return (float)((double)sum * ((double)__builtin_bit_cast(float, sx) * (double)__builtin_bit_cast(float, sw)) + (double)bias);
}

// A result of 16 bits before its rounding to them.  (Where that is fp16 the compiler makes one instruction of some of these and their rounding, which rounds once, so that bits would depend on a result's place.)
template <typename T> __device__ __forceinline__ float in_32_bits(float a, float b, float c)
{
    float v = fmaf(a, b, c);
    if constexpr (__is_same(T, f16)) asm("" : "+v"(v));
    return v;
}

// A product in two parts and the bias, added up.
__device__ __forceinline__ float with_bias(float t, float rest, float bias)
{
    const float whole = t + bias, of_bias = whole - t;
    return whole + (rest + ((t - (whole - of_bias)) + (bias - of_bias)));
}

// The same in 32.  T of 16 bits: the sum and the scales' product are rounded, and so is the result before it is rounded to T.  T of 32 bits: the sum has up to 31 bits, the scales' product 48,
// and both have a part that 32 bits leave over, as have their product and the sum with the bias; with these the result is off by its own rounding and less than ten times 2^-48 of what the product and the
// bias are by themselves.
template <typename T> __device__ __forceinline__ float product_value(int32_t sum, float sx, float sw, float bias)
{
    const float p = rounded(sx, sw), hi = (float)sum;
    if constexpr (sizeof(T) == 2) return in_32_bits<T>(hi, p, bias);
    const float lo = (float)(sum - (int32_t)hi), t = rounded(hi, p);
    return with_bias(t, fmaf(hi, fmaf(sx, sw, -p), fmaf(lo, p, fmaf(hi, p, -t))), bias);
}
// Scales and biases of which no part of the above leaves the range.
__device__ __forceinline__ bool moderate(float scale) { return fabsf(scale) >= 0x1p-38f && fabsf(scale) <= 0x1p48f; }
__device__ __forceinline__ bool moderate_bias(float b) { return fabsf(b) < 0x1p120f; }
// Others: the same steps on the scales' mantissas, whose powers of two come in before the bias does; what is near the end of the range is added up 2^8 below it.  Powers of two are exact, so that results of moderate
// scales are the same to the bit either way, and do not depend on what is done beside them.
template <typename T> __device__ __forceinline__ float product_value_apart(int32_t sum, float sx, float sw, float bias)
{
    const float mx = __builtin_amdgcn_frexp_mantf(sx), mw = __builtin_amdgcn_frexp_mantf(sw), p = rounded(mx, mw), hi = (float)sum;
    const int power = __builtin_amdgcn_frexp_expf(sx) + __builtin_amdgcn_frexp_expf(sw);
    if constexpr (sizeof(T) == 2) {
        const int of_p = min(max(power, -100), 100);
        return in_32_bits<T>(ldexpf(hi, min(power - of_p, 90)), ldexpf(p, of_p), bias);          // (beyond 2^90 it passes the range anyway, but is a number still)
    }
    const float lo = (float)(sum - (int32_t)hi), t = rounded(hi, p);
    const int down = fabsf(ldexpf(t, power)) >= 0x1p120f || fabsf(bias) >= 0x1p120f ? 8 : 0;
    const float at = ldexpf(t, power - down), b = ldexpf(bias, -down), v = with_bias(at, ldexpf(fmaf(hi, fmaf(mx, mw, -p), fmaf(lo, p, fmaf(hi, p, -t))), power - down), b);
    // (An infinity has no rest, and one of the bias stands against numbers of any size.)
    const uint32_t number = (uint32_t)(fabsf(t) < __builtin_inff()) & (uint32_t)!(fabsf(bias) < __builtin_inff());
    const float beyond = number ? bias : at + b;
    return fabsf(at + b) < __builtin_inff() ? ldexpf(v, down) : beyond;
}
// A row of zeros has the least scale that there is.  Of a sum of zero the first way makes the bias whatever the scales, so rows of that scale go it too, where their codes, or all their sums, are zero.
__device__ __forceinline__ bool least_scale(float scale) { return scale == 0x1p-126f; }

__device__ const i32x4 ZERO_CHUNK = {0, 0, 0, 0};

// Few results: 16 rows by 16 outputs to a workgroup, whose waves share out the steps of 64 codes, straight from memory into registers, and add their sums up in LDS.  Bound by w's way
// from memory, and where that is short by a launch and what follows one another in it (bf16, 4 and 16 waves, us: 1 x 4,096 to 4,096 6.3 and 5.0, 100 x 512 to 256 3.6 and 4.9).  Up to 64 rows a
// workgroup, w read once for all of them: 15.8 for 64 x 4,096 to 4,096, where tiles of split codes, which the rule takes, and their join have 12.6; 11.7 for 14.6 with 8,192 to 1,000, and later for 300 rows than tiles.
template <typename T, int WAVES>
__global__ void __launch_bounds__(WAVES * 64) product_few_kernel(ProductArgs a)
{
    constexpr int AT_ONCE = 4;                                     // steps whose loads are under way together
    __shared__ i32x4 sums[WAVES][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int32_t down = (a.n_rows + 15) / 16;
    const int32_t n0 = (int32_t)(blockIdx.x % (uint32_t)down) * 16, m0 = (int32_t)(blockIdx.x / (uint32_t)down) * 16;
    const uint8_t *w = a.w + (uint64_t)min(m0 + (lane & 15), a.n_outs - 1) * a.w_stride, *x = a.x + (uint64_t)min(n0 + (lane & 15), a.n_rows - 1) * a.x_stride;
    const int32_t chunks = (a.n_cols + 15) / 16, steps = (chunks + 3) / 4;
    i32x4 acc = {0, 0, 0, 0};
    for (int32_t t0 = wave; t0 < steps; t0 += WAVES * AT_ONCE) {
        i32x4 u[AT_ONCE], v[AT_ONCE];
#pragma unroll
        for (int q = 0; q < AT_ONCE; ++q) {
            // Chunks beyond the row: its last one's codes of w, and zeros in place of x'.
            const int32_t c = (t0 + q * WAVES) * 4 + (lane >> 4);
            u[q] = *reinterpret_cast<const i32x4 *>(w + min(c, chunks - 1) * 16);
            v[q] = *reinterpret_cast<const i32x4 *>(c < chunks ? x + c * 16 : reinterpret_cast<const uint8_t *>(&ZERO_CHUNK));
        }
#pragma unroll
        for (int q = 0; q < AT_ONCE; ++q) acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(u[q], v[q], acc, 0, 0, 0);
    }
    sums[wave][lane] = acc;
    __syncthreads();
    if (wave) return;
#pragma unroll
    for (int k = 1; k < WAVES; ++k) acc += sums[k][lane];
    const int32_t n = n0 + (lane & 15), m = m0 + (lane >> 4) * 4;
    if (n >= a.n_rows || m >= a.n_outs) return;
    const uint32_t sx = *reinterpret_cast<const uint32_t *>(x + a.held_bytes - 4);
    T *y = row_at<T>(a.y, a.y_stride, n) + m;
    float v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int32_t at = min(m + e, a.n_outs - 1);
        const uint32_t sw = *row_at<uint32_t>(a.w + a.held_bytes - 4, a.w_stride, at);
        v[e] = wide_value(sum_of_codes(acc[e], sx, sw, scale_in_sum(a.n_cols)), sx, sw, bias_at(a, at));
    }
    if (m + 4 <= a.n_outs) {
        store_pack<T, 4>(y, v);
    } else {
#pragma unroll
        for (int e = 0; e < 3; ++e)
            if (m + e < a.n_outs) y[e] = (T)v[e];
    }
}

// Tiles of TM rows by TN outputs, by WM x WN waves of BM x BN blocks of 16 x 16.  Steps of 128 codes pass through LDS, two to four of them there: one is multiplied while the others
// arrive, written into LDS by the loads themselves.  A row of a step is eight chunks of 16 bytes, stored in an order that depends on the row, so that the 16 lanes that
// LDS serves at a time (16 rows, one chunk of each) fall on all banks once.
// Workgroup g runs on XCD g mod 8, and every XCD has an L2 of its own: tiles that share operands, which follow one another, go to one XCD.
// Large products are bound by the matrix operations and by what waves read of LDS: 8,192 x 8,192 to 8,192 in bf16 520 us by tiles of 256 (2,110 TOPS; the matrix units are busy for 56 %), 484 on a cool card, 546 behind other
// work.  Where that is a fraction of a tile's start and end, by these: 10,007 x 1,001 to 517 in fp32 19.4 by tiles of 128, a fifth of which are a fifth column for the last 5 outputs.  Workgroups that stay and take one tile after the other have no registers left for it (560).
__device__ __forceinline__ uint32_t tile_of_workgroup()
{
    constexpr uint32_t XCDS = 8;
    const uint32_t x = blockIdx.x % XCDS, each = gridDim.x / XCDS, rest = gridDim.x % XCDS;
    return x * each + min(x, rest) + blockIdx.x / XCDS;
}

template <int WM_, int WN_, int BM_, int BN_, int STAGES_, int PACK_>
struct Tiles {
    static constexpr int WM = WM_, WN = WN_, BM = BM_, BN = BN_, STAGES = STAGES_, PACK = PACK_;
    static constexpr int THREADS = WM * WN * 64, TM = WM * BM * 16, TN = WN * BN * 16, DEPTH = 128;
    static constexpr int ROWS = TM + TN, STAGE = ROWS * DEPTH, LOADS = ROWS * 8 / THREADS;
    static constexpr int LDS_BYTES = STAGES * STAGE + ROWS * 4;          // behind the stages the scales
    static_assert(ROWS * 8 % THREADS == 0 && TM * 8 % THREADS == 0 && LDS_BYTES <= 160 * 1024, "");
    typedef i32x4 Acc[BM][BN];
    typedef const __attribute__((address_space(1))) uint8_t *Global;

    static __device__ __forceinline__ int slot_of(int row, int chunk) { return chunk ^ ((row >> 1) & 7); }

    // Waits until no more than the newest AWAY of this wave's loads are under way, and then for every wave to be there.  The fences keep the compiler to the order and cost no instruction.
    template <int AWAY> static __device__ __forceinline__ void arrive()
    {
        static_assert(AWAY < 64, "");
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_waitcnt((AWAY & 15) | (AWAY >> 4 << 14) | (7 << 4));           // vmcnt AWAY, lgkmcnt 0
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_sched_barrier(0);
    }

    // Rows of w lie in a stage in an order by which a lane, which comes to hold four outputs of each block, holds PACK that follow one another, and the four lanes of a row 4 PACK: 64 bytes.
    static __device__ __forceinline__ int output_of(int row)
    {
        const int in = row % (4 * PACK), r = in % 16;
        return row - in + r / 4 * PACK + in / 16 * 4 + r % 4;
    }
    static __device__ __forceinline__ int of_output(int m)         // the row of a stage
    {
        const int in = m % (4 * PACK), r = in % PACK;
        return TM + m - in + r / 4 * 16 + in / PACK * 4 + r % 4;
    }

    // Eight columns of tiles at a time, row by row: what an XCD works on at once is about square.
    struct Place { int32_t n0, m0; };
    static __device__ __forceinline__ Place place_of(const ProductArgs &a, uint32_t t)
    {
        constexpr uint32_t ABREAST = 8;
        const uint32_t down = ((uint32_t)a.n_rows + TM - 1) / TM, across = ((uint32_t)a.n_outs + TN - 1) / TN;
        const uint32_t band = t / (down * ABREAST), in_band = t - band * down * ABREAST, width = min(ABREAST, across - band * ABREAST);
        return {(int32_t)(in_band / width) * TM, (int32_t)(band * ABREAST + in_band % width) * TN};
    }

    struct Source {
        Global base[2];                                            // of the tile's first row of x, of w
        uint32_t offset[LOADS];
        int32_t chunks, row_last, first, last;                     // of a row; the step that has the last of them; the workgroup's steps
        __device__ __forceinline__ Source(const ProductArgs &a, const Place &p, int32_t split) : chunks((a.n_cols + 15) / 16), row_last((chunks - 1) / 8), first(split * a.each), last(min(first + a.each - 1, row_last))
        {
            base[0] = (Global)(a.x + (uint64_t)p.n0 * a.x_stride);
            base[1] = (Global)(a.w + (uint64_t)p.m0 * a.w_stride);
#pragma unroll
            for (int i = 0; i < LOADS; ++i) {
                const int q = i * THREADS + (int)threadIdx.x, row = q / 8;
                offset[i] = row_offset(a, p, row) + (uint32_t)slot_of(row, q % 8) * 16u;
            }
        }
        static __device__ __forceinline__ uint32_t row_offset(const ProductArgs &a, const Place &p, int row)
        {
            return row < TM ? (uint32_t)min(row, a.n_rows - 1 - p.n0) * (uint32_t)a.x_stride : (uint32_t)min(output_of(row - TM), a.n_outs - 1 - p.m0) * (uint32_t)a.w_stride;
        }
        __device__ __forceinline__ void load(int32_t step, uint8_t *stage) const
        {
            constexpr int OF_X = TM * 8 / THREADS;
            step = min(step, last);                                // behind the last step that step again
            const bool ragged = step == row_last && (chunks & 7);
#pragma unroll
            for (int i = 0; i < LOADS; ++i) {
                Global from = base[i < OF_X ? 0 : 1] + (int64_t)step * DEPTH + offset[i];
                if (ragged) {                                      // chunks beyond the row are zeros
                    const int q = i * THREADS + (int)threadIdx.x;
                    if (step * 8 + slot_of(q / 8, q % 8) >= chunks) from = (Global)reinterpret_cast<const uint8_t *>(&ZERO_CHUNK);
                }
                __builtin_amdgcn_global_load_lds(from, (__attribute__((address_space(3))) void *)(stage + (i * THREADS + (int)(threadIdx.x & ~63u)) * 16), 16, 0, 0);
            }
        }
    };
};

// Bias of V outputs from each of m, m + 4 V, ..., read in one go.
template <int N, int V, typename B> __device__ __forceinline__ void load_bias(const B *bias, int32_t m, int32_t n_outs, float (&b)[N])
{
#pragma unroll
    for (int e = 0; e < N; ++e) b[e] = (float)bias[min(m + e / V * V * 4 + e % V, n_outs - 1)];
}

// The tile's results.
template <typename T, typename Tile, bool APART> __device__ __forceinline__ void store_tile(const ProductArgs &a, const typename Tile::Place &p, const typename Tile::Acc &acc, const float *scales,
                                                                                           const float (&b)[Tile::BN * 4])
{
    constexpr int V = Tile::PACK;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, first = (wave % Tile::WN) * Tile::BN * 16 + (lane >> 4) * V;
    const float *sx = scales + (wave / Tile::WN) * Tile::BM * 16 + (lane & 15);
    const int32_t n0 = p.n0 + (wave / Tile::WN) * Tile::BM * 16 + (lane & 15);
    const bool scales_in = scale_in_sum(a.n_cols);
#pragma unroll
    for (int k = 0; k < Tile::BN * 4; k += V) {                    // V outputs that lie side by side
        const int32_t m = p.m0 + first + k * 4;
        float sw[V];
#pragma unroll
        for (int e = 0; e < V; ++e) sw[e] = scales[Tile::of_output(first + k * 4 + e)];
        if (m >= a.n_outs) continue;
#pragma unroll
        for (int i = 0; i < Tile::BM; ++i) {
            if (n0 + i * 16 >= a.n_rows) continue;
            float v[V];
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float x = sx[i * 16];
                const int32_t sum = sum_of_codes(acc[i][(k + e) / 4][(k + e) % 4], __builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, sw[e]), scales_in);
                v[e] = APART ? product_value_apart<T>(sum, x, sw[e], b[k + e]) : product_value<T>(sum, x, sw[e], b[k + e]);
            }
            T *y = row_at<T>(a.y, a.y_stride, n0 + i * 16) + m;
            if (m + V <= a.n_outs) {
                store_pack<T, V>(y, v);
            } else {
#pragma unroll
                for (int e = 0; e < V; ++e)
                    if (m + e < a.n_outs) y[e] = (T)v[e];
            }
        }
    }
}

template <typename T, typename Tile> __device__ __forceinline__ void finish_tile(const ProductArgs &a, const typename Tile::Place &p, const typename Tile::Acc &acc, const float *scales)
{
    constexpr int V = Tile::PACK;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, first = (wave % Tile::WN) * Tile::BN * 16 + (lane >> 4) * V;
    float b[Tile::BN * 4] = {};
    if (a.bias) {
        if (a.bias_type == RG_F32) load_bias<Tile::BN * 4, V>(static_cast<const float *>(a.bias), p.m0 + first, a.n_outs, b);
        else if (a.bias_type == RG_BF16) load_bias<Tile::BN * 4, V>(static_cast<const bf16 *>(a.bias), p.m0 + first, a.n_outs, b);
        else load_bias<Tile::BN * 4, V>(static_cast<const f16 *>(a.bias), p.m0 + first, a.n_outs, b);
    }
    const float *sx = scales + (wave / Tile::WN) * Tile::BM * 16 + (lane & 15);
    const auto sw = [&](int k) { return scales[Tile::of_output(first + k / V * V * 4 + k % V)]; };
    const auto sums = [&](int i, int k, float x, float w) { return sum_of_codes(acc[i][k / 4][k % 4], __builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, w), scale_in_sum(a.n_cols)); };
    uint32_t far = 0, least = 0;                                   // (bits, so that the compiler makes no branches of them)
#pragma unroll
    for (int i = 0; i < Tile::BM; ++i) {
        least |= (uint32_t)least_scale(sx[i * 16]);
        far |= (uint32_t)!moderate(sx[i * 16]) & (uint32_t)!least_scale(sx[i * 16]);
    }
#pragma unroll
    for (int k = 0; k < Tile::BN * 4; ++k) {
        least |= (uint32_t)least_scale(sw(k));
        far |= ((uint32_t)!moderate(sw(k)) & (uint32_t)!least_scale(sw(k))) | (uint32_t)!moderate_bias(b[k]);
    }
    if (__ballot(least)) {                                         // (by rows and outputs, of which most have none: all at once they spill)
#pragma unroll
        for (int i = 0; i < Tile::BM; ++i) {
            const float x = sx[i * 16];
            if (!__ballot(least_scale(x))) continue;
            int32_t left = 0;
#pragma unroll
            for (int k = 0; k < Tile::BN * 4; ++k) left |= sums(i, k, x, sw(k));
            far |= (uint32_t)least_scale(x) & (uint32_t)(left != 0);
        }
#pragma unroll
        for (int k = 0; k < Tile::BN * 4; ++k) {
            const float w = sw(k);
            if (!__ballot(least_scale(w))) continue;
            int32_t left = 0;
#pragma unroll
            for (int i = 0; i < Tile::BM; ++i) left |= sums(i, k, sx[i * 16], w);
            far |= (uint32_t)least_scale(w) & (uint32_t)(left != 0);
        }
    }
    if (__ballot(far)) store_tile<T, Tile, true>(a, p, acc, scales, b);
    else store_tile<T, Tile, false>(a, p, acc, scales, b);
}

// A split's sums as they are, rows of a multiple of 4 apart.
__host__ __device__ constexpr int64_t sums_pitch(int64_t n_outs) { return (n_outs + 3) / 4 * 4; }
template <typename Tile> __device__ __forceinline__ void store_sums(const ProductArgs &a, const typename Tile::Place &p, int32_t split, const typename Tile::Acc &acc)
{
    constexpr int V = Tile::PACK;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int32_t n0 = p.n0 + (wave / Tile::WN) * Tile::BM * 16 + (lane & 15), m0 = p.m0 + (wave % Tile::WN) * Tile::BN * 16 + (lane >> 4) * V;
#pragma unroll
    for (int i = 0; i < Tile::BM; ++i) {
        if (n0 + i * 16 >= a.n_rows) continue;
        int32_t *to = a.partial + ((int64_t)split * a.n_rows + n0 + i * 16) * sums_pitch(a.n_outs);
#pragma unroll
        for (int j = 0; j < Tile::BN; ++j) {
            const int32_t m = m0 + j * 4 / V * V * 4 + j * 4 % V;
            if (m < a.n_outs) *reinterpret_cast<i32x4 *>(to + m) = acc[i][j];
        }
    }
}

template <typename T, typename Tile>
__global__ void __launch_bounds__(Tile::THREADS, 2) product_tiles_kernel(ProductArgs a)
{
    extern __shared__ __align__(16) uint8_t lds[];
    constexpr int BM = Tile::BM, BN = Tile::BN;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const uint32_t number = tile_of_workgroup();
    const int32_t split = (int32_t)(number / a.tiles);
    const typename Tile::Place place = Tile::place_of(a, number % a.tiles);
    const typename Tile::Source src(a, place, split);
    constexpr int STAGES = Tile::STAGES;
#pragma unroll
    for (int s = 0; s < STAGES; ++s) src.load(src.first + s, lds + s * Tile::STAGE);
    float *scales = reinterpret_cast<float *>(lds + STAGES * Tile::STAGE);
    for (int row = threadIdx.x; row < Tile::ROWS; row += Tile::THREADS) {
        const auto *from = (const __attribute__((address_space(1))) float *)(src.base[row < Tile::TM ? 0 : 1] + Tile::Source::row_offset(a, place, row) + (a.held_bytes - 4));
        scales[row] = *from;
    }
    typename Tile::Acc acc;
#pragma unroll
    for (int i = 0; i < BM; ++i)
#pragma unroll
        for (int j = 0; j < BN; ++j) acc[i][j] = i32x4{0, 0, 0, 0};
    const int row_x = (wave / Tile::WN) * BM * 16 + (lane & 15), row_w = Tile::TM + (wave % Tile::WN) * BN * 16 + (lane & 15);
    const auto read = [&](const uint8_t *stage, int s, i32x4 (&x)[BM], i32x4 (&w)[BN]) {
        const int slot = Tile::slot_of(lane & 15, s * 4 + (lane >> 4)) * 16;              // the rows of a block begin at multiples of 16
#pragma unroll
        for (int i = 0; i < BM; ++i) x[i] = *reinterpret_cast<const i32x4 *>(stage + (row_x + i * 16) * Tile::DEPTH + slot);
#pragma unroll
        for (int j = 0; j < BN; ++j) w[j] = *reinterpret_cast<const i32x4 *>(stage + (row_w + j * 16) * Tile::DEPTH + slot);
    };
    const auto multiply = [&](const i32x4 (&x)[BM], const i32x4 (&w)[BN]) {
#pragma unroll
        for (int i = 0; i < BM; ++i)
#pragma unroll
            for (int j = 0; j < BN; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[j], x[i], acc[i][j], 0, 0, 0);
    };
    Tile::template arrive<0>();
    i32x4 x0[BM], w0[BN], x1[BM], w1[BN];
    read(lds, 0, x0, w0);
    uint8_t *stage = lds;
    for (int32_t t = 0; t <= src.last - src.first; ++t) {
        uint8_t *next = stage == lds + (STAGES - 1) * Tile::STAGE ? lds : stage + Tile::STAGE;
        read(stage, 1, x1, w1);
        multiply(x0, w0);
        Tile::template arrive<(STAGES - 2) * Tile::LOADS>();      // the stage is read, and the next one there
        src.load(src.first + t + STAGES, stage);
        read(next, 0, x0, w0);
        multiply(x1, w1);
        stage = next;
    }
    Tile::template arrive<0>();                                    // a workgroup's LDS is not left with loads under way
    if (a.partial) store_sums<Tile>(a, place, split, acc);
    else finish_tile<T, Tile>(a, place, acc, scales);
}

// The splits' sums, added up, and what they stand for: four results of a row to a thread.  Bound by the sums' way through the caches; 4.0 us of the 17.0 that 300 x 8,192 to 1,000 takes in three splits.
template <typename T>
__global__ void __launch_bounds__(256) product_join_kernel(ProductArgs a, int32_t splits)
{
    const int32_t across = (a.n_outs + 3) / 4;
    const int64_t q = (int64_t)blockIdx.x * 256 + threadIdx.x, n = q / across;
    if (n >= a.n_rows) return;
    const int32_t m = (int32_t)(q - n * across) * 4, count = min(4, a.n_outs - m);
    const int64_t pitch = sums_pitch(a.n_outs);
    const int32_t *from = a.partial + n * pitch + m;
    i32x4 sum{0, 0, 0, 0};                                         // (behind the last output whatever the tile made of that output's codes)
    for (int32_t s = 0; s < splits; ++s) sum += *reinterpret_cast<const i32x4 *>(from + s * a.n_rows * pitch);
    const uint32_t sx = *row_at<uint32_t>(a.x + a.held_bytes - 4, a.x_stride, n);
    float v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int32_t at = m + min(e, count - 1);
        const uint32_t sw = *row_at<uint32_t>(a.w + a.held_bytes - 4, a.w_stride, at);
        v[e] = wide_value(sum_of_codes(sum[e], sx, sw, scale_in_sum(a.n_cols)), sx, sw, bias_at(a, at));
    }
    store_four(row_at<T>(a.y, a.y_stride, n) + m, f32x4{v[0], v[1], v[2], v[3]}, count);
}

// Many rows of few codes: what bounds them is the rows' and the results' way from and to HBM and, beside it, w's way out of LDS, and tiles spend most of their time at their start and end.  Here w lies in LDS, once
// for all rows that a workgroup does (where it has more than that holds, each workgroup has a share of the outputs), and a wave by itself takes 16 rows at a time into registers, the next
// ones under way meanwhile: no barrier behind the first.  w lies as the matrix operations take it: of a block of 16 outputs chunk by chunk, 16 rows side by side.  150,000 x 512 to 256 in bf16: 45 us,
// 3.4 TB/s, where HBM would take 30 and the reads of LDS, all of w for 16 rows, 23; the matrix units are busy for 24 % of it.
struct ThinArgs {
    ProductArgs p;
    int32_t outs;                    // of a workgroup, a multiple of 32
    int32_t shares;                  // of the outputs
};

// The row of w that lies at place r (0 to 31) of two blocks, so that a lane holds V outputs side by side.
template <int V> __device__ __forceinline__ int thin_output(int r) { return V == 8 ? r % 16 / 4 * 8 + r / 16 * 4 + r % 4 : r; }

template <typename T, int KS>
__global__ void __launch_bounds__(THIN_THREADS) product_thin_kernel(ThinArgs t)
{
    constexpr int V = 16 / sizeof(T), WAVES = THIN_THREADS / 64;
    extern __shared__ __align__(16) uint8_t lds[];
    const ProductArgs &a = t.p;
    typedef const __attribute__((address_space(1))) uint8_t *Global;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int32_t chunks = (a.n_cols + 15) / 16, m0 = (int32_t)(blockIdx.x % (uint32_t)t.shares) * t.outs, mine = min(t.outs, a.n_outs - m0);
    const int32_t blocks = (mine + 31) / 32 * 2;
    // Blocks of 16 rows; behind the last block's rows its last row, which nothing is made of.
    const int32_t turns = (int32_t)(gridDim.x / (uint32_t)t.shares) * WAVES;
    int32_t rb = (int32_t)(blockIdx.x / (uint32_t)t.shares) * WAVES + wave;
    i32x4 x[KS], next[KS];
    float sx, next_sx;
    const auto load = [&](int32_t b, i32x4 (&to)[KS], float &s) {
        const uint8_t *row = a.x + (uint64_t)min((int64_t)b * 16 + (lane & 15), (int64_t)a.n_rows - 1) * a.x_stride;
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            const int32_t c = k * 4 + (lane >> 4);
            Global from = c < chunks ? (Global)(row + c * 16) : (Global)reinterpret_cast<const uint8_t *>(&ZERO_CHUNK);
            to[k] = *(const __attribute__((address_space(1))) i32x4 *)from;
        }
        s = *(const __attribute__((address_space(1))) float *)(Global)(row + a.held_bytes - 4);
    };
    load(rb, x, sx);
    float *scales = reinterpret_cast<float *>(lds + (uint32_t)(t.outs / 16 * chunks) * 256), *bias = scales + t.outs;
    int *all_fine = reinterpret_cast<int *>(bias + t.outs);
    if (threadIdx.x == 0) *all_fine = 1;
    for (int32_t block = wave; block < blocks; block += WAVES) {
        const int32_t m = block / 2 * 32 + thin_output<V>(block % 2 * 16 + (lane & 15));
        Global row = (Global)(a.w + (uint64_t)(m0 + min(m, mine - 1)) * a.w_stride);
        uint8_t *to = lds + (uint32_t)(block * chunks) * 256;
        int32_t c = 0;
        for (; c + 4 <= chunks; c += 4) __builtin_amdgcn_global_load_lds(row + (c + (lane >> 4)) * 16, (__attribute__((address_space(3))) void *)(to + c * 256), 16, 0, 0);
        if (c + (lane >> 4) < chunks) *reinterpret_cast<i32x4 *>(to + c * 256 + lane * 16) = *(const __attribute__((address_space(1))) i32x4 *)(row + (c + (lane >> 4)) * 16);
    }
    const bool scales_in = scale_in_sum(a.n_cols);
    // Whether a row of the least scale has other codes than zeros, by its words in this lane's chunks; behind the last ones in a row lies its scale.
    constexpr uint32_t LEAST_BITS = 0x00800000u;
    const auto words_of = [&](const i32x4 &v, int32_t c) { return v[0] | v[1] | v[2] | (scales_in && c == chunks - 1 ? v[3] ^ (int)LEAST_BITS : v[3]); };
    for (int32_t m = threadIdx.x; m < blocks * 16; m += THIN_THREADS) {
        const int32_t at = m0 + min(m, mine - 1);
        scales[m] = *row_at<float>(a.w + a.held_bytes - 4, a.w_stride, at);
        bias[m] = bias_at(a, at);
    }
    __syncthreads();                                               // and what was loaded is there
    bool w_fine = true;
    for (int32_t r = threadIdx.x; r < blocks * 16; r += THIN_THREADS) {
        const int32_t m = r / 32 * 32 + thin_output<V>(r % 32);
        bool fine = moderate(scales[m]);
        if (least_scale(scales[m])) {
            int words = 0;
            for (int32_t c = 0; c < chunks; ++c) words |= words_of(*reinterpret_cast<const i32x4 *>(lds + (uint32_t)(r / 16 * chunks + c) * 256 + r % 16 * 16), c);
            fine = words == 0;
        }
        w_fine = w_fine && fine && moderate_bias(bias[m]);
    }
    if (!w_fine) *all_fine = 0;
    __syncthreads();
    w_fine = *all_fine;
    const int32_t n_blocks = (a.n_rows + 15) / 16;
    while (rb < n_blocks) {
        if (rb + turns < n_blocks) load(rb + turns, next, next_sx);
        bool x_fine = moderate(sx);
        if (__ballot(least_scale(sx))) {
            int words = 0;
#pragma unroll
            for (int k = 0; k < KS; ++k) words |= words_of(x[k], k * 4 + (lane >> 4));
            x_fine = x_fine || (least_scale(sx) && words == 0);
        }
        const bool fine = !__ballot(!(w_fine && x_fine));
        const int32_t n = rb * 16 + (lane & 15);
        T *y = row_at<T>(a.y, a.y_stride, n) + m0;
        for (int32_t pair = 0; pair < blocks; pair += 2) {
            i32x4 acc[2] = {};
            const uint8_t *w = lds + (uint32_t)(pair * chunks) * 256 + (lane & 15) * 16;
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                const int32_t c = min(k * 4 + (lane >> 4), chunks - 1) * 256;
#pragma unroll
                for (int j = 0; j < 2; ++j) acc[j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(*reinterpret_cast<const i32x4 *>(w + j * chunks * 256 + c), x[k], acc[j], 0, 0, 0);
            }
#pragma unroll
            for (int k = 0; k < 8; k += V) {
                const int32_t m = pair * 16 + k * 4 + (lane >> 4) * V;
                if (n >= a.n_rows || m >= mine) continue;
                float v[V], sw[V];
                int32_t sum[V];
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    sw[e] = scales[m + e];
                    sum[e] = sum_of_codes(acc[(k + e) / 4][(k + e) % 4], __builtin_bit_cast(uint32_t, sx), __builtin_bit_cast(uint32_t, sw[e]), scales_in);
                }
                if (fine) {
#pragma unroll
                    for (int e = 0; e < V; ++e) v[e] = product_value<T>(sum[e], sx, sw[e], bias[m + e]);
                } else {
#pragma unroll
                    for (int e = 0; e < V; ++e) v[e] = product_value_apart<T>(sum[e], sx, sw[e], bias[m + e]);
                }
                if (m + V <= mine) {
                    store_pack<T, V>(y + m, v);
                } else {
#pragma unroll
                    for (int e = 0; e < V; ++e)
                        if (m + e < mine) y[m + e] = (T)v[e];
                }
            }
        }
        rb += turns;
        sx = next_sx;
#pragma unroll
        for (int k = 0; k < KS; ++k) x[k] = next[k];
    }
}

// ---------------------------------------------------------------- the backward pass
// C[i][j] = sum over k of A(i, k) s[k] code[k][j]: dx (i: rows, k: outputs, held rows w) and dweight (i: outputs, k: rows, held rows x).  A's elements times the scale, in fp32,
// go in as sums of three bf16 numbers, which hold all 24 bits, for 16-bit A as well: with two, 16 bits, one result of 200 was another bf16 number than the exact one's (150,000 x 256 to 512; of
// fp32 sums one of 4,600), and fp32 gradients of 16-bit rows had no more than those 16 bits.
constexpr int PARTS = GRAD_PARTS;
struct GradArgs {
    const uint8_t *dy, *held;
    uint64_t dy_stride, held_stride;
    uint8_t *out;
    uint64_t out_stride;
    uint32_t out_type;
    const float *scales;             // of the held rows (dx)
    float *sums;                     // [splits][n_i] of dy's columns (dweight's), or NULL
    float *partial;                  // [splits][n_i][n_j], or NULL: a sum is done by one workgroup
    const uint8_t *gather;           // held rows whose scales are put side by side on the way, or NULL
    uint64_t gather_stride;
    float *gathered;
    int32_t n_gather;
    int32_t n_i, n_j, n_k, held_bytes;
    int32_t k_each;                  // of a split
    uint32_t tiles;
    bool rows_apart;                 // dy's rows: what lies behind a row's end, but for the last rows', may be read
};

// A number as a sum of bf16 numbers: cut off, not rounded, but for the last, so that no part is beyond the range.  What an infinity or a NaN leaves is nothing.
__device__ __forceinline__ void parts_of(float v, bf16 (&p)[PARTS])
{
    const bool number = (__builtin_bit_cast(uint32_t, v) & 0x7F800000u) != 0x7F800000u;
#pragma unroll
    for (int q = 0; q < PARTS; ++q) {
        const uint32_t bits = __builtin_bit_cast(uint32_t, v) & 0xFFFF0000u;
        p[q] = q == PARTS - 1 || !number ? (bf16)v : __builtin_bit_cast(bf16, (uint16_t)(bits >> 16));
        v = number ? v - __builtin_bit_cast(float, bits) : 0.f;
    }
}
// Eight of them at once, of numbers; the largest of their magnitudes (passing over NaN, of which something is left over and is NaN).
__device__ __forceinline__ float parts_of_numbers(const float (&from)[8], bf16x8 (&p)[PARTS])
{
    float v[8], most = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = from[e];
#pragma unroll
    for (int e = 0; e < 8; e += 2) most = fmaxf(fmaxf(most, fabsf(v[e])), fabsf(v[e + 1]));
#pragma unroll
    for (int q = 0; q < PARTS; ++q) {
        if (q == PARTS - 1) {
#pragma unroll
            for (int e = 0; e < 8; ++e) p[q][e] = (bf16)v[e];
        } else {
            u32x4 heads;
#pragma unroll
            for (int e = 0; e < 8; e += 2) {
                heads[e / 2] = __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, v[e + 1]), __builtin_bit_cast(uint32_t, v[e]), 0x07060302u);
                v[e] -= __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, v[e]) & 0xFFFF0000u);
                v[e + 1] -= __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, v[e + 1]) & 0xFFFF0000u);
            }
            p[q] = __builtin_bit_cast(bf16x8, heads);
        }
    }
    return most;
}
// Whether a lane of the wave has an infinity, of which the above makes a NaN.
__device__ __forceinline__ bool beyond_numbers(float most) { return __builtin_expect(__ballot(most == __builtin_inff()) != 0, 0); }
// Eight products dy[e] * scale(e) of any kind.  Of numbers whose product is beyond the range every part is the largest bf16 number: a code other than zero makes an infinity of them, a code of zero leaves nothing, where an
// infinity would make a NaN of it.
template <typename S> __device__ __forceinline__ void parts_of_any(const float (&dy)[8], const S &scale, bf16x8 (&p)[PARTS])
{
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float v = rounded(dy[e], scale(e));
        const bool beyond = fabsf(v) == __builtin_inff() && fabsf(dy[e]) < __builtin_inff() && fabsf(scale(e)) < __builtin_inff();
        bf16 one[PARTS];
        parts_of(v, one);
#pragma unroll
        for (int q = 0; q < PARTS; ++q) p[q][e] = beyond ? (bf16)copysignf(0x1.FEp+127f, v) : one[q];
    }
}

typedef int i32x2 __attribute__((ext_vector_type(2)));
// Eight codes of a column, of rows whose eight bytes 16 lanes point at.
__device__ __forceinline__ i32x2 column_of_codes(const uint8_t *from) { return __builtin_amdgcn_ds_read_tr8_b64_v2i32((__attribute__((address_space(3))) i32x2 *)from); }
__device__ __forceinline__ bf16x8 codes_as_bf16(const i32x2 &c)
{
    u32x4 out;
#pragma unroll
    for (int e = 0; e < 8; e += 2) {                               // whole numbers of seven bits: bf16 is the upper half of fp32
        const float lo = (float)(int8_t)(c[e / 4] >> (e % 4 * 8)), hi = (float)(int8_t)(c[e / 4] >> (e % 4 * 8 + 8));
        out[e / 2] = __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, hi), __builtin_bit_cast(uint32_t, lo), 0x07060302u);
    }
    return __builtin_bit_cast(bf16x8, out);
}

// Tiles of TI x TJ by WI x WJ waves of BI x BJ blocks of 16 x 16, in steps of 32 along k.  ALONG: dy's rows run along k (dx); otherwise along i (dweight).  A step's elements of dy are read into registers
// two steps ahead, and one step ahead are multiplied with their scales, parted, and written into LDS; the codes go there as they are.  Of operands that lie along the wrong axis LDS itself makes columns (reads
// that transpose blocks of 16 x 8 bytes or 16 x 4 numbers).  What the lanes read at a time falls on all banks once: the order of the 16-byte chunks of a row, or of the 32-byte pieces of
// one of dy's, depends on the row.  What they write of the codes, 16 bytes at steps of 32, has half of the banks at a time (0.3 to 0.4 cycles of conflicts to an instruction of LDS).
// Bound by the vector units: matrix operations keep them for 40 to 64 % of the time, and what parts dy hardly overlaps with them.  In tiles of 256 (least of 10 passes under the profiler, us):
// dweight and the sums of 199,000 x 602 to 256 in fp32 224 (820 TFLOP/s of bf16, a fifth of them for columns behind the last) and 17 for the join; 150,000 x 512 to 256 in bf16 117 and 17, dx 153; 8,192 x 4,096 to 4,096
// 713 and 631 (1,160 and 1,310).
template <typename T, bool ALONG_, bool SUMS_, int WI_, int WJ_, int BI_, int BJ_>
struct GradTile {
    static constexpr int WI = WI_, WJ = WJ_, BI = BI_, BJ = BJ_;
    static constexpr bool ALONG = ALONG_, SUMS = SUMS_;              // SUMS: of dy's columns as well (dbias)
    static constexpr int THREADS = WI * WJ * 64, TI = WI * BI * 16, TJ = WJ * BJ * 16, DEPTH = 32;
    static constexpr int LEFT = PARTS * TI * DEPTH * 2, RIGHT = DEPTH * TJ * 2, STAGE = LEFT + RIGHT, LDS_BYTES = 2 * STAGE + (SUMS ? THREADS * 32 : 0);      // behind the stages the threads' sums of dy's columns
    static constexpr int PACKS = TI * DEPTH / 8 / THREADS, CHUNKS = (DEPTH * TJ / 16 + THREADS - 1) / THREADS;
    static_assert(PACKS * THREADS * 8 == TI * DEPTH && LDS_BYTES <= 160 * 1024 && TI >= 64 && TJ >= 64, "");
    typedef typename PackOf<T, 8>::type Raw;

    // Bytes into a part of the left operand, of the pack of eight elements that begins at (i, k), one of which runs.
    static __device__ __forceinline__ uint32_t left_at(int i, int k)
    {
        if (ALONG) return (uint32_t)(i * 64 + ((k / 8) ^ (-(i >> 2) & 3)) * 16);
        return across_at<TI>(k, i);
    }
    template <int N> static __device__ __forceinline__ uint32_t across_at(int k, int c)
    {
        const int turn = N >= 128 ? (k & 3) | ((k >> 1) & 4) : ((k >> 1) & 1) | ((k >> 2) & 2);       // of 64 numbers two rows lie on all banks together
        return (uint32_t)(k * N * 2 + ((c / 16) ^ turn) * 32 + (c % 16) * 2);
    }
    // Bytes into the right one, of (k, j): rows of all columns of the tile.
    static __device__ __forceinline__ uint32_t right_at(int k, int j) { return across_at<TJ>(k, j); }

    // What a thread reads of a step.
    struct Step {
        Raw dy[PACKS];
        float scale[ALONG ? 8 : PACKS];
        i32x4 codes[CHUNKS];
    };
    // Where it comes from: addresses of the next step's, as long as all of that is inside; else they are made anew, element by element.
    struct Source {
        const GradArgs &a;
        const uint8_t *dy[PACKS], *scale[ALONG ? 1 : PACKS], *codes[CHUNKS];
        int32_t i0, j0, k0, k_end, k_whole;                        // of the next step; up to where a step's elements may be read whole
        __device__ __forceinline__ Source(const GradArgs &args, int32_t i, int32_t j, int32_t k, int32_t end) : a(args), i0(i), j0(j), k0(k), k_end(end), k_whole(end)
        {
            // Beyond the last column of i nothing is made of what is read, which are the next rows' elements.
            if (!ALONG && i0 + TI > a.n_i) k_whole = a.rows_apart ? min(k_end, a.n_k - 8) : 0;
#pragma unroll
            for (int p = 0; p < PACKS; ++p) {
                const int q = p * THREADS + (int)threadIdx.x;
                if constexpr (ALONG) {                             // (of a row beyond the last nothing is made: the last one's elements do)
                    dy[p] = reinterpret_cast<const uint8_t *>(row_at<T>(a.dy, a.dy_stride, min(i0 + q / 4, a.n_i - 1)) + k0 + q % 4 * 8);
                } else {
                    const int32_t row = min(k0 + q / (TI / 8), k_end - 1);
                    const int32_t first = i0 + q % (TI / 8) * 8;
                    dy[p] = reinterpret_cast<const uint8_t *>(row_at<T>(a.dy, a.dy_stride, row) + (first < a.n_i ? first : 0));
                    scale[p] = a.held + (uint64_t)row * a.held_stride + (a.held_bytes - 4);
                }
            }
            if constexpr (ALONG) scale[0] = reinterpret_cast<const uint8_t *>(a.scales + k0 + (int32_t)(threadIdx.x % 4) * 8);
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c) codes[c] = codes_at(k0, c);
        }
        __device__ __forceinline__ const uint8_t *codes_at(int32_t k, int c) const
        {
            const int q = min(c * THREADS + (int)threadIdx.x, DEPTH * TJ / 16 - 1);
            return a.held + (uint64_t)min(k + q / (TJ / 16), k_end - 1) * a.held_stride + min(j0 + q % (TJ / 16) * 16, a.held_bytes - 16);
        }
        __device__ __forceinline__ void load(Step &s)
        {
            if (k0 + DEPTH <= k_whole) {
#pragma unroll
                for (int p = 0; p < PACKS; ++p) {
                    s.dy[p] = load_raw<T, 8>(reinterpret_cast<const T *>(dy[p]));
                    dy[p] += ALONG ? (uint64_t)DEPTH * sizeof(T) : DEPTH * a.dy_stride;
                }
                if constexpr (ALONG) {
#pragma unroll
                    for (int e = 0; e < 8; e += 4) {
                        const f32x4 v = reinterpret_cast<const f32x4 *>(scale[0])[e / 4];
#pragma unroll
                        for (int x = 0; x < 4; ++x) s.scale[e + x] = v[x];
                    }
                    scale[0] += DEPTH * sizeof(float);
                } else {
#pragma unroll
                    for (int p = 0; p < PACKS; ++p) {
                        s.scale[p] = *reinterpret_cast<const float *>(scale[p]);
                        scale[p] += DEPTH * a.held_stride;
                    }
                }
#pragma unroll
                for (int c = 0; c < CHUNKS; ++c) {
                    s.codes[c] = *reinterpret_cast<const i32x4 *>(codes[c]);
                    codes[c] += DEPTH * a.held_stride;
                }
            } else if (k0 < k_end) {
                load_part(s);
            }
            k0 += DEPTH;
        }
        __device__ __forceinline__ void load_part(Step &s) const
        {
#pragma unroll
            for (int p = 0; p < PACKS; ++p) {
                const int q = p * THREADS + (int)threadIdx.x;
                const int32_t i = i0 + (ALONG ? q / 4 : q % (TI / 8) * 8), k = k0 + (ALONG ? q % 4 * 8 : q / (TI / 8));
                const int32_t row = ALONG ? i : k, first = ALONG ? k : i, rows = ALONG ? a.n_i : k_end, cols = ALONG ? k_end : a.n_i;
                const T *from = row_at<T>(a.dy, a.dy_stride, min(row, rows - 1)) + first;
                if (row < rows && first + 8 <= cols) {
                    s.dy[p] = load_raw<T, 8>(from);
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) s.dy[p][e] = row < rows && first + e < cols ? from[e] : (T)0.f;
                }
                if constexpr (!ALONG) s.scale[p] = *row_at<float>(a.held + a.held_bytes - 4, a.held_stride, min(k, k_end - 1));
            }
            if constexpr (ALONG) {
                const int32_t k = k0 + (int32_t)(threadIdx.x % 4) * 8;
#pragma unroll
                for (int e = 0; e < 8; ++e) s.scale[e] = a.scales[min(k + e, a.n_k - 1)];
            }
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c) s.codes[c] = *reinterpret_cast<const i32x4 *>(codes_at(k0, c));
        }
    };
    static __device__ __forceinline__ void put_parts(int p, const bf16x8 (&parts)[PARTS], uint8_t *stage)
    {
        const int q = p * THREADS + (int)threadIdx.x;
#pragma unroll
        for (int x = 0; x < PARTS; ++x)
            *reinterpret_cast<bf16x8 *>(stage + x * (TI * DEPTH * 2) + left_at(ALONG ? q / 4 : q % (TI / 8) * 8, ALONG ? q % 4 * 8 : q / (TI / 8))) = parts[x];
    }
    // A step into LDS, as if all were numbers; what they were is in `most`.  sums: of dy's columns.
    static __device__ __forceinline__ float put(const Step &s, uint8_t *stage, float (&sums)[8])
    {
        float most = 0.f;
#pragma unroll
        for (int p = 0; p < PACKS; ++p) {
            float v[8];
            bf16x8 parts[PARTS];
            unpack<T, 8>(s.dy[p], v);
            if constexpr (SUMS) {
#pragma unroll
                for (int e = 0; e < 8; ++e) sums[e] += v[e];
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = rounded(v[e], s.scale[ALONG ? e : p]);
            most = fmaxf(most, parts_of_numbers(v, parts));
            put_parts(p, parts, stage);
        }
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            const int q = c * THREADS + (int)threadIdx.x;
            if (DEPTH * TJ / 16 % THREADS && q >= DEPTH * TJ / 16) continue;
            bf16x8 *to = reinterpret_cast<bf16x8 *>(stage + LEFT + right_at(q / (TJ / 16), q % (TJ / 16) * 16));
            to[0] = codes_as_bf16(i32x2{s.codes[c][0], s.codes[c][1]});
            to[1] = codes_as_bf16(i32x2{s.codes[c][2], s.codes[c][3]});
        }
        return most;
    }
    // And once more where they were not.
    static __device__ __forceinline__ void put_any(const Step &s, uint8_t *stage)
    {
#pragma unroll
        for (int p = 0; p < PACKS; ++p) {
            float v[8];
            bf16x8 parts[PARTS];
            unpack<T, 8>(s.dy[p], v);
            parts_of_any(v, [&](int e) { return s.scale[ALONG ? e : p]; }, parts);
            put_parts(p, parts, stage);
        }
    }

    // The operand of a matrix operation: 16 rows of i (columns of j), a lane has eight along k.
    static __device__ __forceinline__ bf16x8 left(const uint8_t *part, int i, int lane)
    {
        if constexpr (ALONG) return *reinterpret_cast<const bf16x8 *>(part + left_at(i + (lane & 15), (lane >> 4) * 8));
        else return column<TI>(part, i, lane);
    }
    static __device__ __forceinline__ bf16x8 right(const uint8_t *part, int j, int lane) { return column<TJ>(part, j, lane); }
    template <int N> static __device__ __forceinline__ bf16x8 column(const uint8_t *part, int c, int lane)
    {
        typedef short s16x4 __attribute__((ext_vector_type(4)));
        const int k = (lane >> 4) * 8 + ((lane >> 2) & 3), at = c + (lane & 3) * 4;
        const s16x4 u = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)(part + across_at<N>(k, at)));
        const s16x4 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)(part + across_at<N>(k + 4, at)));
        return __builtin_bit_cast(bf16x8, __builtin_shufflevector(u, v, 0, 1, 2, 3, 4, 5, 6, 7));
    }

    // Waits until what this wave wrote into LDS is there, and then for every wave.  (Loads stay under way, which __syncthreads would wait for.)
    static __device__ __forceinline__ void arrive()
    {
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_waitcnt(15 | (7 << 4) | (3 << 14));     // lgkmcnt 0
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_sched_barrier(0);
    }
};

template <typename T, typename Tile>
__global__ void __launch_bounds__(Tile::THREADS, 2) grad_kernel(GradArgs a)
{
    extern __shared__ __align__(16) uint8_t lds[];
    constexpr int BI = Tile::BI, BJ = Tile::BJ, DEPTH = Tile::DEPTH;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const uint32_t mine = blockIdx.x * Tile::THREADS + threadIdx.x;
    if (!Tile::ALONG && a.gather && mine < (uint32_t)a.n_gather) a.gathered[mine] = *row_at<float>(a.gather + a.held_bytes - 4, a.gather_stride, mine);
    // Tiles of one row of j follow one another, splits of k of a tile lie apart: what an XCD works on at once shares dy.
    const uint32_t across = ((uint32_t)a.n_j + Tile::TJ - 1) / Tile::TJ, t = tile_of_workgroup();
    const uint32_t tile = t % a.tiles, split = t / a.tiles;
    const int32_t i0 = (int32_t)(tile / across) * Tile::TI, j0 = (int32_t)(tile % across) * Tile::TJ;
    const int64_t k_first = (int64_t)split * a.k_each;
    const int32_t k_end = (int32_t)min((int64_t)a.n_k, k_first + a.k_each);
    const int wi = (wave / Tile::WJ) * BI * 16, wj = (wave % Tile::WJ) * BJ * 16;
    // Of the two waves of a vector unit one prepares the next step before it multiplies, the other behind it: the one's conversions go beside the other's matrix operations.
    const bool early = wave < 4;
    f32x4 acc[BI][BJ] = {};
    // Sums of dy's columns in two levels, so that no more than 16 elements are added up in a row: what a thread has of eight steps goes onto what it has in LDS.  (The largest tile has no registers left.)
    float sums[8] = {};
    f32x4 *const mine_of_sums = reinterpret_cast<f32x4 *>(lds + 2 * Tile::STAGE) + threadIdx.x * 2;
    const auto keep_sums = [&] {
#pragma unroll
        for (int h = 0; h < 2; ++h) mine_of_sums[h] += f32x4{sums[h * 4], sums[h * 4 + 1], sums[h * 4 + 2], sums[h * 4 + 3]};
#pragma unroll
        for (int e = 0; e < 8; ++e) sums[e] = 0.f;
    };
    if constexpr (Tile::SUMS) mine_of_sums[0] = mine_of_sums[1] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (k_first < k_end) {
        typename Tile::Step step;
        typename Tile::Source src(a, i0, j0, (int32_t)k_first, k_end);
        const int32_t last = (k_end - 1 - (int32_t)k_first) / DEPTH;
        const auto prepare = [&](uint8_t *stage) __attribute__((always_inline)) {
            if (beyond_numbers(Tile::put(step, stage, sums))) Tile::put_any(step, stage);
            src.load(step);
        };
        src.load(step);
        prepare(lds);
        Tile::arrive();
        for (int32_t s = 0; s <= last; ++s) {
            const uint8_t *stage = lds + (s & 1) * Tile::STAGE;
            uint8_t *other = lds + (~s & 1) * Tile::STAGE;
            if (early && s < last) prepare(other);
            // The next blocks' elements are on their way out of LDS while one row of blocks is multiplied: left to itself the compiler asks for them when they are needed.
            bf16x8 r[BJ], l[2][PARTS];
            const auto read = [&](int i, bf16x8 (&to)[PARTS]) __attribute__((always_inline)) {
#pragma unroll
                for (int p = 0; p < PARTS; ++p) to[p] = Tile::left(stage + p * (Tile::TI * DEPTH * 2), wi + i * 16, lane);
            };
            read(0, l[0]);
#pragma unroll
            for (int j = 0; j < BJ; ++j) r[j] = Tile::right(stage + Tile::LEFT, wj + j * 16, lane);
#pragma unroll
            for (int i = 0; i < BI; ++i) {
                if (i + 1 < BI) read(i + 1, l[(i + 1) & 1]);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int p = 0; p < PARTS; ++p)
#pragma unroll
                    for (int j = 0; j < BJ; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(r[j], l[i & 1][p], acc[i][j], 0, 0, 0);
                __builtin_amdgcn_sched_barrier(0);
            }
            if (!early && s < last) prepare(other);
            if constexpr (Tile::SUMS)
                if ((s & 7) == 6) keep_sums();                     // (step s + 1 is in)
            Tile::arrive();
        }
    }
    if constexpr (Tile::SUMS) {
        // What the threads have of a column, added up in their order.
        if (a.sums && j0 == 0) {
            const float *parts = reinterpret_cast<const float *>(lds + 2 * Tile::STAGE);           // rows of TI, of which a thread has eight
            constexpr int GROUPS = Tile::THREADS * 8 / Tile::TI;
            keep_sums();
            __syncthreads();
            if (threadIdx.x < Tile::TI && i0 + (int32_t)threadIdx.x < a.n_i) {
                float v = 0.f;
                for (int g = 0; g < GROUPS; ++g) v += parts[g * Tile::TI + threadIdx.x];
                a.sums[(int64_t)split * a.n_i + i0 + threadIdx.x] = v;
            }
        }
    }
#pragma unroll
    for (int i = 0; i < BI; ++i) {
        const int32_t at = i0 + wi + i * 16 + (lane & 15);
        if (at >= a.n_i) continue;
#pragma unroll
        for (int j = 0; j < BJ; ++j) {
            const int32_t col = j0 + wj + j * 16 + (lane >> 4) * 4, n = a.n_j - col;
            if (a.partial) store_four(a.partial + ((int64_t)split * a.n_i + at) * a.n_j + col, acc[i][j], n);
            else if (a.out_type == RG_F32) store_four(row_at<float>(a.out, a.out_stride, at) + col, acc[i][j], n);
            else if (a.out_type == RG_BF16) store_four(row_at<bf16>(a.out, a.out_stride, at) + col, acc[i][j], n);
            else store_four(row_at<f16>(a.out, a.out_stride, at) + col, acc[i][j], n);
        }
    }
}

// dx of many rows and few outputs, which the tiles do at the pace of their starts and ends: w's codes lie in LDS, once for all rows that a workgroup does (where there is more than that holds, each
// has a share of the columns), and a wave by itself takes 16 rows of dy at a time, parted in registers (the next ones' elements on their way beside them spill, and so do 32 rows).  The codes lie by blocks of 16 columns, row after row: what the
// lanes read at a time is contiguous.  Bound as the tiles are, and by the codes, which every wave makes bf16 numbers of
// anew for 16 rows: 199,000 x 256 to 602 in bf16 192 us (960 TFLOP/s of bf16), by tiles 268; 150,000 x 128 to 256 38 and 49.
struct ThinGradArgs {
    GradArgs g;
    int32_t cols;                    // of a workgroup, a multiple of 32
    int32_t shares;                  // of the columns
};

template <typename T, int KS>
__global__ void __launch_bounds__(THIN_THREADS) grad_thin_kernel(ThinGradArgs t)
{
    constexpr int V = 16 / sizeof(T), WAVES = THIN_THREADS / 64, K = KS * 32;
    typedef typename PackOf<T, 8>::type Raw;
    extern __shared__ __align__(16) uint8_t lds[];
    const GradArgs &a = t.g;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int32_t j0 = (int32_t)(blockIdx.x % (uint32_t)t.shares) * t.cols, mine = min(t.cols, a.n_j - j0);
    const int32_t pairs = (mine + 31) / 32, turns = (int32_t)(gridDim.x / (uint32_t)t.shares) * WAVES, n_blocks = (a.n_i + (int32_t)GRAD_THIN_ROWS - 1) / (int32_t)GRAD_THIN_ROWS;
    // Where few blocks are left for a last turn, several waves take one, each a part of the columns.
    const int32_t number = (int32_t)(blockIdx.x / (uint32_t)t.shares) * WAVES + wave, left_over = n_blocks % turns, parts = left_over ? turns / left_over : 1;
    const int32_t whole_turns = n_blocks - left_over;
    int32_t rb = number, from_pair = 0, to_pair = pairs;
    const auto place = [&] {
        if (rb < whole_turns) return;
        if (left_over == 0 || number >= left_over * parts) { rb = n_blocks; return; }
        const int32_t part = number / left_over;
        rb = whole_turns + number % left_over;
        from_pair = part * pairs / parts;
        to_pair = (part + 1) * pairs / parts;
    };
    place();
    float *scales = reinterpret_cast<float *>(lds + (uint32_t)t.cols * K);
    const bool even = a.n_k % 32 == 0 && a.n_k == K;
    Raw next[KS];
    const auto load = [&](int32_t b) {
        const T *row = row_at<T>(a.dy, a.dy_stride, min((int64_t)b * (int64_t)GRAD_THIN_ROWS + (lane & 15), (int64_t)a.n_i - 1));
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            const int32_t k = s * 32 + (lane >> 4) * 8;
            if (even || k + 8 <= a.n_k) {
                next[s] = load_raw<T, 8>(row + k);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) next[s][e] = k + e < a.n_k ? row[k + e] : (T)0.f;
            }
        }
    };
    load(rb);
    // Units of 32 columns of a row of w, eight rows by eight units to a wave.  Of results of 16 bits a lane comes to hold eight side by side, four of either block.
    const int32_t down = (a.n_k + 7) / 8;
    for (int32_t u = wave; u < down * ((pairs + 7) / 8); u += WAVES) {
        const int32_t k = u % down * 8 + (lane >> 3), pair = u / down * 8 + (lane & 7);
        if (k >= a.n_k || pair >= pairs) continue;
        const uint8_t *row = a.held + (uint64_t)k * a.held_stride;
        const int32_t at = j0 + pair * 32;
        const i32x4 u0 = *reinterpret_cast<const i32x4 *>(row + at), u1 = *reinterpret_cast<const i32x4 *>(row + min(at + 16, a.held_bytes - 16));
        i32x4 *to = reinterpret_cast<i32x4 *>(lds + (uint32_t)(pair * 2) * (K * 16) + k * 16);
        if constexpr (V == 8) {
            to[0] = __builtin_shufflevector(u0, u1, 0, 2, 4, 6);
            to[K] = __builtin_shufflevector(u0, u1, 1, 3, 5, 7);
        } else {
            to[0] = u0;
            to[K] = u1;
        }
    }
    for (int32_t k = threadIdx.x; k < K; k += THIN_THREADS) scales[k] = k < a.n_k ? *row_at<float>(a.held + a.held_bytes - 4, a.held_stride, k) : 0.f;
    __syncthreads();
    while (rb < n_blocks) {
        bf16x8 l[KS][PARTS];
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            const f32x4 lo = *reinterpret_cast<const f32x4 *>(scales + s * 32 + (lane >> 4) * 8), hi = *reinterpret_cast<const f32x4 *>(scales + s * 32 + (lane >> 4) * 8 + 4);
            const auto scale = [&](int e) { return e < 4 ? lo[e] : hi[e - 4]; };
            float dy[8], v[8];
            unpack<T, 8>(next[s], dy);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = rounded(dy[e], scale(e));
            if (beyond_numbers(parts_of_numbers(v, l[s]))) parts_of_any(dy, scale, l[s]);
        }
        const int32_t i = rb * (int32_t)GRAD_THIN_ROWS + (lane & 15);
        for (int32_t pair = from_pair; pair < to_pair; ++pair) {
            f32x4 acc[2] = {};
            // The next step's codes are on their way out of LDS while one is multiplied, and no more: all at once they spill.
            const uint8_t *codes = lds + (uint32_t)(pair * 2) * (K * 16) + ((lane >> 4) * 8 + ((lane & 15) >> 1)) * 16 + (lane & 1) * 8;
            i32x2 now[2] = {column_of_codes(codes), column_of_codes(codes + K * 16)};
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                const bf16x8 r[2] = {codes_as_bf16(now[0]), codes_as_bf16(now[1])};
                if (s + 1 < KS) {
                    now[0] = column_of_codes(codes + (s + 1) * 512);
                    now[1] = column_of_codes(codes + (K * 16) + (s + 1) * 512);
                }
#pragma unroll
                for (int p = 0; p < PARTS; ++p)
#pragma unroll
                    for (int b = 0; b < 2; ++b) acc[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(r[b], l[s][p], acc[b], 0, 0, 0);
                __builtin_amdgcn_sched_barrier(0);
            }
            if (i >= a.n_i) continue;
            T *row = row_at<T>(a.out, a.out_stride, i) + j0;
#pragma unroll
            for (int k = 0; k < 8; k += V) {
                const int32_t j = pair * 32 + k * 4 + (lane >> 4) * V;
                float v[V];
#pragma unroll
                for (int e = 0; e < V; ++e) v[e] = acc[(k + e) / 4][(k + e) % 4];
                if (j + V <= mine) {
                    store_pack<T, V>(row + j, v);
                } else {
#pragma unroll
                    for (int e = 0; e < V; ++e)
                        if (j + e < mine) row[j + e] = (T)v[e];
                }
            }
        }
        if (rb >= whole_turns) return;
        rb += turns;
        place();
        if (rb < n_blocks) load(rb);
    }
}

// The scales of held rows side by side.
__global__ void __launch_bounds__(256) scales_kernel(const uint8_t *held, uint64_t stride, int32_t held_bytes, int32_t n, float *scales)
{
    const int32_t r = (int32_t)(blockIdx.x * 256 + threadIdx.x);
    if (r < n) scales[r] = *row_at<float>(held + held_bytes - 4, stride, r);
}

// The splits' sums of a matrix and, in the workgroups behind it, of a vector, added up in a fixed order: four elements of a row to sixteen threads, each of which has every sixteenth
// split.  (All splits to a thread 27 us for 67 MB of them, so 14.)
struct Join {
    const float *partial;            // [splits][n_i][n_j]
    int32_t splits;
    int64_t n_i, n_j;
    uint8_t *out;
    uint64_t out_stride;
};
constexpr int JOIN_GROUPS = 16, JOIN_QUADS = 256 / JOIN_GROUPS;
inline uint32_t join_grid(const Join &j) { return j.out ? (uint32_t)std::min<int64_t>(8192, (j.n_i * ((j.n_j + 3) / 4) + JOIN_QUADS - 1) / JOIN_QUADS) : 0; }
__global__ void __launch_bounds__(256) grad_join_kernel(Join first, Join second, uint32_t first_grid, uint32_t type)
{
    __shared__ f32x4 sums[JOIN_GROUPS][JOIN_QUADS];
    const bool one = blockIdx.x < first_grid;
    const Join &a = one ? first : second;
    const uint32_t block = one ? blockIdx.x : blockIdx.x - first_grid, grid = one ? first_grid : gridDim.x - first_grid;
    const int at = threadIdx.x % JOIN_QUADS, group = threadIdx.x / JOIN_QUADS;
    const int64_t across = (a.n_j + 3) / 4, quads = a.n_i * across;
    for (int64_t q0 = (int64_t)block * JOIN_QUADS; q0 < quads; q0 += (int64_t)grid * JOIN_QUADS) {
        const int64_t q = min(q0 + at, quads - 1), i = q / across, j = q % across * 4;
        const int32_t n = (int32_t)min((int64_t)4, a.n_j - j);
        const float *from = a.partial + i * a.n_j + j;
        f32x4 v = {0.f, 0.f, 0.f, 0.f};
        if (n == 4) {
#pragma unroll 8
            for (int32_t s = group; s < a.splits; s += JOIN_GROUPS) {
                float w[4];
                load_pack<float, 4>(from + s * a.n_i * a.n_j, w);
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] += w[e];
            }
        } else {
            for (int32_t s = group; s < a.splits; s += JOIN_GROUPS)
                for (int e = 0; e < n; ++e) v[e] += from[s * a.n_i * a.n_j + e];
        }
        __syncthreads();
        sums[group][at] = v;
        __syncthreads();
        if (group || q0 + at >= quads) continue;
#pragma unroll
        for (int g = 1; g < JOIN_GROUPS; ++g) v += sums[g][at];
        uint8_t *row = a.out + (uint64_t)i * a.out_stride;
        if (type == RG_F32) store_four(reinterpret_cast<float *>(row) + j, v, n);
        else if (type == RG_BF16) store_four(reinterpret_cast<bf16 *>(row) + j, v, n);
        else store_four(reinterpret_cast<f16 *>(row) + j, v, n);
    }
}

// Sums of dy's columns over a part of its rows, for calls that want no dweight, whose tiles make them on the way: 64 columns to a workgroup, four rows at a time.  Bound by the latency of
// loads of one element a lane: 150,000 x 256 in bf16 44 us (1.7 TB/s), 199,000 x 256 in fp32 59 (3.5).
template <typename T>
__global__ void __launch_bounds__(256) bias_sums_kernel(const uint8_t *dy, uint64_t dy_stride, int32_t n_rows, int32_t n_outs, int32_t each, float *partial)
{
    __shared__ float sums[4][64];
    const int32_t m = (int32_t)blockIdx.x * 64 + (int32_t)(threadIdx.x & 63);
    const int64_t first = (int64_t)blockIdx.y * each;
    float v = 0.f;
    if (m < n_outs)
        for (int64_t n = first + (threadIdx.x >> 6); n < min((int64_t)n_rows, first + each); n += 4) v += (float)row_at<T>(dy, dy_stride, n)[m];
    sums[threadIdx.x >> 6][threadIdx.x & 63] = v;
    __syncthreads();
    if (threadIdx.x < 64 && m < n_outs) partial[(int64_t)blockIdx.y * n_outs + m] = (sums[0][threadIdx.x] + sums[1][threadIdx.x]) + (sums[2][threadIdx.x] + sums[3][threadIdx.x]);
}

rg_status check_product_sizes(uint64_t n_rows, uint64_t n_outs, uint64_t n_cols)
{
    if (n_cols == 0) { set_error("held rows have at least one element"); return RG_EINVAL; }
    if (n_cols > RG_MAX_HELD_COLS || n_rows > 1ull << 30 || n_outs > 1ull << 30) {
        set_error("%llu rows by %llu outputs of %llu elements are beyond the limits (2^30, 2^30, %u)", (unsigned long long)n_rows, (unsigned long long)n_outs, (unsigned long long)n_cols, RG_MAX_HELD_COLS);
        return RG_ERANGE;
    }
    return RG_OK;
}

rg_status check_types(const char *what, const void *p, uint32_t vector_type, uint32_t type)
{
    if (!element_bytes(type)) { set_error("type %u is none of RG_F32, RG_BF16, RG_F16", type); return RG_EINVAL; }
    if (!p) return RG_OK;
    if (vector_type != RG_F32 && vector_type != type) { set_error("%s: its type %u is neither RG_F32 nor the rows' type", what, vector_type); return RG_EINVAL; }
    if (reinterpret_cast<uintptr_t>(p) % element_bytes(vector_type)) { set_error("%s is not aligned for its type", what); return RG_EINVAL; }
    return RG_OK;
}

rg_status check_workspace(const void *workspace, uint64_t got, uint64_t want)
{
    if (!want) return RG_OK;
    if (!workspace || reinterpret_cast<uintptr_t>(workspace) % 16) { set_error("the workspace is null or not aligned to 16 bytes"); return RG_EINVAL; }
    if (got < want) { set_error("the workspace holds %llu bytes of %llu", (unsigned long long)got, (unsigned long long)want); return RG_ERANGE; }
    return RG_OK;
}

// Offsets within a tile's rows have 32 bits.
rg_status check_steps(const char *what, uint64_t stride)
{
    if (stride < 1ull << 24) return RG_OK;
    set_error("%s: a stride of %llu bytes is beyond the products' limit (2^24)", what, (unsigned long long)stride);
    return RG_ERANGE;
}

rg_status check_grid(uint64_t groups, uint32_t threads)
{
    if (groups <= MAX_WORK_ITEMS / threads) return RG_OK;
    set_error("a result of %llu tiles is more than a launch holds", (unsigned long long)groups);
    return RG_ERANGE;
}

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

template <typename T, typename Tile> rg_status launch_tiles(ProductArgs a, int32_t splits, hipStream_t st)
{
    const uint64_t tiles = ((uint64_t)a.n_rows + Tile::TM - 1) / Tile::TM * (((uint64_t)a.n_outs + Tile::TN - 1) / Tile::TN);
    RG_TRY(check_grid(tiles * (uint64_t)splits, Tile::THREADS));
    a.tiles = (uint32_t)tiles;
    static std::atomic<uint64_t> known{0};
    RG_TRY(allow_lds(product_tiles_kernel<T, Tile>, Tile::LDS_BYTES, known));
    hipLaunchKernelGGL((product_tiles_kernel<T, Tile>), dim3((uint32_t)tiles * (uint32_t)splits), dim3(Tile::THREADS), Tile::LDS_BYTES, st, a);
    RG_HIP(hipGetLastError());
    if (splits > 1) {
        hipLaunchKernelGGL(product_join_kernel<T>, dim3((uint32_t)(((uint64_t)a.n_rows * (((uint64_t)a.n_outs + 3) / 4) + 255) / 256)), dim3(256), 0, st, a, splits);
        RG_HIP(hipGetLastError());
    }
    return RG_OK;
}

template <typename T, int KS> rg_status launch_thin(const ProductArgs &a, int n_cu, hipStream_t st)
{
    const ThinShape s = thin_shape((uint64_t)a.n_rows, (uint64_t)a.n_outs, (uint64_t)a.n_cols, n_cu);
    static std::atomic<uint64_t> known{0};
    RG_TRY(allow_lds(product_thin_kernel<T, KS>, (int)THIN_LDS, known));
    hipLaunchKernelGGL((product_thin_kernel<T, KS>), dim3(s.grid), dim3(THIN_THREADS), s.lds, st, ThinArgs{a, (int32_t)s.outs, (int32_t)s.shares});
    RG_HIP(hipGetLastError());
    return RG_OK;
}

template <typename T> rg_status launch_thin_of(const ProductArgs &a, int n_cu, hipStream_t st)
{
    const int steps = (a.n_cols + 63) / 64;
    if (steps <= 1) return launch_thin<T, 1>(a, n_cu, st);
    if (steps <= 2) return launch_thin<T, 2>(a, n_cu, st);
    if (steps <= 4) return launch_thin<T, 4>(a, n_cu, st);
    if (steps <= 6) return launch_thin<T, 6>(a, n_cu, st);
    if (steps <= 8) return launch_thin<T, 8>(a, n_cu, st);
    if (steps <= 10) return launch_thin<T, 10>(a, n_cu, st);
    return launch_thin<T, THIN_COLS / 64>(a, n_cu, st);
}

template <typename T, int WAVES> rg_status launch_few(const ProductArgs &a, hipStream_t st)
{
    const uint64_t tiles = ((uint64_t)a.n_rows + 15) / 16 * (((uint64_t)a.n_outs + 15) / 16);
    RG_TRY(check_grid(tiles, WAVES * 64));
    hipLaunchKernelGGL((product_few_kernel<T, WAVES>), dim3((uint32_t)tiles), dim3(WAVES * 64), 0, st, a);
    RG_HIP(hipGetLastError());
    return RG_OK;
}

template <typename T> rg_status launch_product(const ProductArgs &a, const ProductCut &c, int n_cu, hipStream_t st)
{
    constexpr int PACK = 16 / sizeof(T);
    switch (c.way) {
    case ProductWay::FEW: return launch_few<T, 4>(a, st);
    case ProductWay::FEW_LONG: return launch_few<T, 16>(a, st);
    case ProductWay::THIN: return launch_thin_of<T>(a, n_cu, st);
    case ProductWay::TILES_64: return launch_tiles<T, Tiles<2, 2, 2, 2, 3, PACK>>(a, c.splits, st);
    case ProductWay::TILES_128: return launch_tiles<T, Tiles<4, 2, 2, 4, 2, PACK>>(a, c.splits, st);
    case ProductWay::TILES_128_DEEP: return launch_tiles<T, Tiles<4, 2, 2, 4, 4, PACK>>(a, c.splits, st);
    default: return launch_tiles<T, Tiles<2, 4, 8, 4, 2, PACK>>(a, c.splits, st);
    }
}

uint64_t product_scratch(uint64_t n, uint64_t m, const ProductCut &c) { return c.splits > 1 ? (uint64_t)c.splits * n * (uint64_t)sums_pitch((int64_t)m) * 4 : 0; }

// How the backward pass is cut, and where its scratch lies.
struct GradPlan {
    GradCut dx, dw;
    int32_t bias_parts, bias_each;
    uint64_t scales_at, bias_at, bytes;  // sums of dweight, then of dx in the same place; w's scales; sums of dbias
};

GradPlan grad_plan(uint64_t n, uint64_t m, uint64_t d, int n_cu, bool dx, bool dw, bool db)
{
    GradPlan p{};
    uint64_t bytes = 0;
    if (dx) {
        p.dx = grad_cut(n, d, m, PARTS, n_cu, true);
        if (p.dx.splits > 1) bytes = std::max(bytes, (uint64_t)p.dx.splits * n * d * 4);
    }
    if (dw) {
        p.dw = grad_cut(m, d, n, PARTS, n_cu, false);
        if (p.dw.splits > 1) bytes = std::max(bytes, (uint64_t)p.dw.splits * m * d * 4);
    }
    p.scales_at = (bytes + 15) / 16 * 16;
    if (dx && p.dx.way != GradWay::THIN) bytes = p.scales_at + m * 4;
    p.bias_at = (bytes + 15) / 16 * 16;
    if (db) {
        p.bias_parts = dw ? p.dw.splits : (int32_t)std::max<uint64_t>(1, std::min<uint64_t>(256, n / 64));
        p.bias_each = (int32_t)((n + p.bias_parts - 1) / p.bias_parts);
        bytes = p.bias_at + (uint64_t)p.bias_parts * m * 4;
    }
    p.bytes = bytes;
    return p;
}

template <typename T, typename Tile> rg_status launch_grad(int32_t splits, const GradArgs &g, hipStream_t st)
{
    static std::atomic<uint64_t> known{0};
    RG_TRY(allow_lds(grad_kernel<T, Tile>, Tile::LDS_BYTES, known));
    hipLaunchKernelGGL((grad_kernel<T, Tile>), dim3(g.tiles * (uint32_t)splits), dim3(Tile::THREADS), Tile::LDS_BYTES, st, g);
    RG_HIP(hipGetLastError());
    return RG_OK;
}

template <typename T, bool ALONG, bool SUMS> rg_status launch_grad_by(const GradCut &c, const GradArgs &g, hipStream_t st)
{
    switch (c.way) {
    case GradWay::TILES_256: return launch_grad<T, GradTile<T, ALONG, SUMS, 2, 4, 8, 4>>(c.splits, g, st);
    case GradWay::TILES_128: return launch_grad<T, GradTile<T, ALONG, SUMS, 2, 2, 4, 4>>(c.splits, g, st);
    case GradWay::TILES_64_256: return launch_grad<T, GradTile<T, ALONG, SUMS, 1, 4, 4, 4>>(c.splits, g, st);
    default: return launch_grad<T, GradTile<T, ALONG, SUMS, 2, 2, 2, 2>>(c.splits, g, st);
    }
}

template <typename T, int KS> rg_status launch_grad_thin(const GradArgs &g, int n_cu, hipStream_t st)
{
    const ThinShape s = grad_thin_shape((uint64_t)g.n_i, (uint64_t)g.n_j, KS * 32, GRAD_THIN_ROWS, n_cu);
    static std::atomic<uint64_t> known{0};
    RG_TRY(allow_lds(grad_thin_kernel<T, KS>, (int)THIN_LDS, known));
    hipLaunchKernelGGL((grad_thin_kernel<T, KS>), dim3(s.grid), dim3(THIN_THREADS), s.lds, st, ThinGradArgs{g, (int32_t)s.outs, (int32_t)s.shares});
    RG_HIP(hipGetLastError());
    return RG_OK;
}
template <typename T> rg_status launch_grad_thin_of(const GradArgs &g, int n_cu, hipStream_t st)
{
    if (g.n_k <= 32) return launch_grad_thin<T, 1>(g, n_cu, st);
    if (g.n_k <= 64) return launch_grad_thin<T, 2>(g, n_cu, st);
    if (g.n_k <= 128) return launch_grad_thin<T, 4>(g, n_cu, st);
    return launch_grad_thin<T, GRAD_THIN_OUTS / 32>(g, n_cu, st);
}

template <bool ALONG> rg_status launch_grad_of(uint32_t type, const GradCut &c, const GradArgs &g, hipStream_t st)
{
    constexpr bool MAY = !ALONG;
    if (type == RG_F32) return g.sums ? (launch_grad_by<float, ALONG, MAY>(c, g, st)) : (launch_grad_by<float, ALONG, false>(c, g, st));
    if (type == RG_BF16) return g.sums ? (launch_grad_by<bf16, ALONG, MAY>(c, g, st)) : (launch_grad_by<bf16, ALONG, false>(c, g, st));
    return g.sums ? (launch_grad_by<f16, ALONG, MAY>(c, g, st)) : (launch_grad_by<f16, ALONG, false>(c, g, st));
}

rg_status launch_join(const Join &first, const Join &second, uint32_t type, hipStream_t st)
{
    const uint32_t grid = join_grid(first), more = join_grid(second);
    if (grid + more == 0) return RG_OK;
    hipLaunchKernelGGL(grad_join_kernel, dim3(grid + more), dim3(256), 0, st, first, second, grid, type);
    RG_HIP(hipGetLastError());
    return RG_OK;
}

}  // namespace
}  // namespace rg

using namespace rg;

extern "C" rg_status rg_rows8_product_workspace(uint64_t n_rows, uint64_t n_outs, uint64_t n_cols, uint32_t type, uint64_t *bytes)
{
    if (!bytes) { set_error("null argument"); return RG_EINVAL; }
    RG_TRY(check_product_sizes(n_rows, n_outs, n_cols));
    RG_TRY(check_types("y", nullptr, RG_F32, type));
    *bytes = 0;
    if (n_rows == 0 || n_outs == 0) return RG_OK;
    int n_cu = 0;
    RG_TRY(compute_units(&n_cu));
    *bytes = product_scratch(n_rows, n_outs, product_cut(n_rows, n_outs, n_cols, element_bytes(type), n_cu));
    return RG_OK;
}

extern "C" rg_status rg_rows8_product(const void *x, uint64_t x_stride, uint64_t n_rows, const void *w, uint64_t w_stride, uint64_t n_outs, uint64_t n_cols,
                                      const void *bias, uint32_t bias_type, void *y, uint64_t y_stride, uint32_t type, void *workspace, uint64_t workspace_bytes, void *stream)
{
    RG_TRY(check_product_sizes(n_rows, n_outs, n_cols));
    RG_TRY(check_types("bias", bias, bias_type, type));
    if (n_rows == 0 || n_outs == 0) return RG_OK;
    RG_TRY(check_held("x", x, x_stride, n_rows, n_cols, false));
    RG_TRY(check_held("w", w, w_stride, n_outs, n_cols, false));
    RG_TRY(check_elements("y", y, y_stride, n_rows, n_outs, element_bytes(type), true));
    RG_TRY(check_steps("x", x_stride));
    RG_TRY(check_steps("w", w_stride));
    ProductArgs a{};
    a.x = static_cast<const uint8_t *>(x); a.x_stride = x_stride;
    a.w = static_cast<const uint8_t *>(w); a.w_stride = w_stride;
    a.bias = bias; a.bias_type = bias_type;
    a.y = static_cast<uint8_t *>(y); a.y_stride = y_stride;
    a.n_rows = (int32_t)n_rows; a.n_outs = (int32_t)n_outs; a.n_cols = (int32_t)n_cols; a.held_bytes = (int32_t)held_bytes(n_cols);
    const hipStream_t st = as_stream(stream);
    int n_cu = 0;
    RG_TRY(compute_units(&n_cu));
    const ProductCut c = product_cut(n_rows, n_outs, n_cols, element_bytes(type), n_cu);
    RG_TRY(check_workspace(workspace, workspace_bytes, product_scratch(n_rows, n_outs, c)));
    a.partial = c.splits > 1 ? static_cast<int32_t *>(workspace) : nullptr;
    a.each = c.each;
    if (type == RG_F32) RG_TRY(launch_product<float>(a, c, n_cu, st));
    else if (type == RG_BF16) RG_TRY(launch_product<bf16>(a, c, n_cu, st));
    else RG_TRY(launch_product<f16>(a, c, n_cu, st));
    return RG_OK;
}

extern "C" rg_status rg_rows8_product_backward_workspace(uint64_t n_rows, uint64_t n_outs, uint64_t n_cols, uint32_t type, int want_dx, int want_dweight, int want_dbias,
                                                         uint64_t *bytes)
{
    if (!bytes) { set_error("null argument"); return RG_EINVAL; }
    RG_TRY(check_product_sizes(n_rows, n_outs, n_cols));
    RG_TRY(check_types("dy", nullptr, RG_F32, type));
    int n_cu = 0;
    RG_TRY(compute_units(&n_cu));
    *bytes = grad_plan(n_rows, n_outs, n_cols, n_cu, want_dx, want_dweight, want_dbias).bytes;
    return RG_OK;
}

extern "C" rg_status rg_rows8_product_backward(const void *dy, uint64_t dy_stride, const void *x, uint64_t x_stride, const void *w, uint64_t w_stride, uint64_t n_rows,
                                               uint64_t n_outs, uint64_t n_cols, uint32_t type, void *dx, uint64_t dx_stride, void *dweight, uint64_t dweight_stride, void *dbias,
                                               uint32_t weight_type, void *workspace, uint64_t workspace_bytes, void *stream)
{
    RG_TRY(check_product_sizes(n_rows, n_outs, n_cols));
    RG_TRY(check_types("dweight", dweight, weight_type, type));
    RG_TRY(check_types("dbias", dbias, weight_type, type));
    const uint32_t bytes = element_bytes(type);
    if (n_outs) RG_TRY(check_elements("dy", dy, dy_stride, n_rows, n_outs, bytes, false));
    if (dx) {
        RG_TRY(check_elements("dx", dx, dx_stride, n_rows, n_cols, bytes, true));
        RG_TRY(check_held("w", w, w_stride, n_outs, n_cols, false));
    }
    if (dweight) {
        RG_TRY(check_elements("dweight", dweight, dweight_stride, n_outs, n_cols, element_bytes(weight_type), true));
        RG_TRY(check_held("x", x, x_stride, n_rows, n_cols, false));
    }
    int n_cu = 0;
    RG_TRY(compute_units(&n_cu));
    const GradPlan p = grad_plan(n_rows, n_outs, n_cols, n_cu, dx, dweight, dbias);
    RG_TRY(check_workspace(workspace, workspace_bytes, p.bytes));
    if (p.dx.way == GradWay::TILES_256) RG_TRY(check_grid(p.dx.tiles * (uint64_t)p.dx.splits, 512));         // of the others grad_cut sees to it
    if (p.dw.way == GradWay::TILES_256) RG_TRY(check_grid(p.dw.tiles * (uint64_t)p.dw.splits, 512));
    if (dbias && !dweight) RG_TRY(check_grid((n_outs + 63) / 64, 256));
    const hipStream_t st = as_stream(stream);
    uint8_t *scratch = static_cast<uint8_t *>(workspace);
    float *sums = reinterpret_cast<float *>(scratch), *scales = reinterpret_cast<float *>(scratch + p.scales_at), *bias = reinterpret_cast<float *>(scratch + p.bias_at);
    const bool by_tiles = dx && n_rows && n_outs && p.dx.way != GradWay::THIN;        // which take w's scales side by side
    GradArgs common{};
    common.dy = static_cast<const uint8_t *>(dy); common.dy_stride = dy_stride;
    common.rows_apart = dy_stride >= n_outs * bytes;
    common.n_j = (int32_t)n_cols; common.held_bytes = (int32_t)held_bytes(n_cols);
    Join of_weight{}, of_bias{};
    if (dbias && n_outs) of_bias = Join{bias, p.bias_parts, 1, (int64_t)n_outs, static_cast<uint8_t *>(dbias), 0};
    if (dweight && n_outs) {
        GradArgs g = common;
        g.held = static_cast<const uint8_t *>(x); g.held_stride = x_stride;
        g.out = static_cast<uint8_t *>(dweight); g.out_stride = dweight_stride; g.out_type = weight_type;
        g.n_i = (int32_t)n_outs; g.n_k = (int32_t)n_rows; g.k_each = p.dw.each; g.tiles = (uint32_t)p.dw.tiles;
        g.sums = dbias ? bias : nullptr;
        if (by_tiles) { g.gather = static_cast<const uint8_t *>(w); g.gather_stride = w_stride; g.gathered = scales; g.n_gather = (int32_t)n_outs; }
        if (p.dw.splits > 1) { g.partial = sums; of_weight = Join{sums, p.dw.splits, (int64_t)n_outs, (int64_t)n_cols, g.out, g.out_stride}; }
        RG_TRY(launch_grad_of<false>(type, p.dw, g, st));
    } else if (of_bias.out) {
        const dim3 grid((uint32_t)((n_outs + 63) / 64), (uint32_t)p.bias_parts);
        if (type == RG_F32) hipLaunchKernelGGL(bias_sums_kernel<float>, grid, dim3(256), 0, st, common.dy, dy_stride, (int32_t)n_rows, (int32_t)n_outs, p.bias_each, bias);
        else if (type == RG_BF16) hipLaunchKernelGGL(bias_sums_kernel<bf16>, grid, dim3(256), 0, st, common.dy, dy_stride, (int32_t)n_rows, (int32_t)n_outs, p.bias_each, bias);
        else hipLaunchKernelGGL(bias_sums_kernel<f16>, grid, dim3(256), 0, st, common.dy, dy_stride, (int32_t)n_rows, (int32_t)n_outs, p.bias_each, bias);
        RG_HIP(hipGetLastError());
    }
    RG_TRY(launch_join(of_weight, of_bias, weight_type, st));
    if (dx && n_rows) {
        GradArgs g = common;
        g.held = static_cast<const uint8_t *>(w); g.held_stride = w_stride;
        g.out = static_cast<uint8_t *>(dx); g.out_stride = dx_stride; g.out_type = type;
        g.n_i = (int32_t)n_rows; g.n_k = (int32_t)n_outs; g.k_each = p.dx.each; g.tiles = (uint32_t)p.dx.tiles;
        g.scales = scales;
        if (p.dx.way == GradWay::THIN) {
            if (type == RG_F32) return launch_grad_thin_of<float>(g, n_cu, st);
            return type == RG_BF16 ? launch_grad_thin_of<bf16>(g, n_cu, st) : launch_grad_thin_of<f16>(g, n_cu, st);
        }
        if (by_tiles && !dweight) {
            hipLaunchKernelGGL(scales_kernel, dim3((uint32_t)((n_outs + 255) / 256)), dim3(256), 0, st, g.held, g.held_stride, g.held_bytes, g.n_k, scales);
            RG_HIP(hipGetLastError());
        }
        Join of_rows{};
        if (p.dx.splits > 1) { g.partial = sums; of_rows = Join{sums, p.dx.splits, (int64_t)n_rows, (int64_t)n_cols, g.out, g.out_stride}; }
        RG_TRY(launch_grad_of<true>(type, p.dx, g, st));
        RG_TRY(launch_join(of_rows, Join{}, type, st));
    }
    return RG_OK;
}
