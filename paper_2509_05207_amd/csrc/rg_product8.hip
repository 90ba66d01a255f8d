// Products on rows held in 8 bits: rg_rows8_product, in 8-bit integers with a scale for each row of either side, and its backward pass,
// which takes nothing of the forward pass but the held rows.
#include "rg_internal.h"
#include "rg_elements.h"
#include "rg_launch.h"

namespace rg {

namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef bf16 bf16x8 __attribute__((ext_vector_type(8)));

template <typename T> __device__ __forceinline__ T *row_at(void *p, uint64_t stride, int64_t r) { return reinterpret_cast<T *>(static_cast<uint8_t *>(p) + (uint64_t)r * stride); }
template <typename T> __device__ __forceinline__ const T *row_at(const void *p, uint64_t stride, int64_t r) { return reinterpret_cast<const T *>(static_cast<const uint8_t *>(p) + (uint64_t)r * stride); }

// ---------------------------------------------------------------- y = x w^T + bias
struct ProductArgs {
    const uint8_t *x, *w;
    uint64_t x_stride, w_stride;
    const void *bias;
    uint32_t bias_type;
    uint8_t *y;
    uint64_t y_stride;
    int32_t n_rows, n_outs, n_cols, held_bytes;
};

// A chunk of 16 bytes with codes in it may have the scale's four behind them: where that is so, the scales' own bytes have gone into a sum, and are taken off again.
__device__ __forceinline__ bool scale_in_sum(int32_t n_cols) { const int32_t r = n_cols & 15; return r >= 1 && r <= 12; }

__device__ __forceinline__ float bias_at(const ProductArgs &a, int32_t m)
{
    if (!a.bias) return 0.f;
    return a.bias_type == RG_F32 ? static_cast<const float *>(a.bias)[m] : a.bias_type == RG_BF16 ? (float)static_cast<const bf16 *>(a.bias)[m] : (float)static_cast<const f16 *>(a.bias)[m];
}

// What a sum of codes stands for.  In 64 bits: the sum has up to 31 bits, and two scales' product may leave fp32's range where the result does not.
__device__ __forceinline__ float product_value(int32_t sum, uint32_t sx, uint32_t sw, float bias, bool scales_in)
{
    if (scales_in) sum = sum - __builtin_amdgcn_sdot4((int)sx, (int)sw, 0, false);
    return (float)((double)sum * ((double)__builtin_bit_cast(float, sx) * (double)__builtin_bit_cast(float, sw)) + (double)bias);
}

// Sixteen rows by sixteen outputs to a workgroup, whose waves share out the steps of 64 codes.
template <typename T>
__global__ void __launch_bounds__(256) product_few_kernel(ProductArgs a)
{
    constexpr int WAVES = 4;
    __shared__ i32x4 sums[WAVES][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int32_t down = (a.n_rows + 15) / 16;
    const int32_t n0 = (int32_t)(blockIdx.x % (uint32_t)down) * 16, m0 = (int32_t)(blockIdx.x / (uint32_t)down) * 16;
    const uint8_t *x = a.x + (uint64_t)min(n0 + (lane & 15), a.n_rows - 1) * a.x_stride, *w = a.w + (uint64_t)min(m0 + (lane & 15), a.n_outs - 1) * a.w_stride;
    const int32_t chunks = (a.n_cols + 15) / 16, steps = (chunks + 3) / 4;
    i32x4 acc = {0, 0, 0, 0};
    for (int32_t t = wave; t < steps; t += WAVES) {
        const int32_t c = t * 4 + (lane >> 4);
        i32x4 u = {0, 0, 0, 0}, v = {0, 0, 0, 0};
        if (c < chunks) {
            u = *reinterpret_cast<const i32x4 *>(w + c * 16);
            v = *reinterpret_cast<const i32x4 *>(x + c * 16);
        }
        acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(u, v, acc, 0, 0, 0);
    }
    sums[wave][lane] = acc;
    __syncthreads();
    if (wave) return;
    for (int k = 1; k < WAVES; ++k) acc += sums[k][lane];
    const int32_t n = n0 + (lane & 15), m = m0 + (lane >> 4) * 4;
    if (n >= a.n_rows) return;
    const uint32_t sx = *reinterpret_cast<const uint32_t *>(x + a.held_bytes - 4);
    T *y = row_at<T>(a.y, a.y_stride, n);
    for (int e = 0; e < 4; ++e) {
        if (m + e >= a.n_outs) return;
        const uint32_t s = *row_at<uint32_t>(a.w + a.held_bytes - 4, a.w_stride, m + e);
        y[m + e] = (T)product_value(acc[e], sx, s, bias_at(a, m + e), scale_in_sum(a.n_cols));
    }
}

// ---------------------------------------------------------------- the backward pass
// C[i][j] = sum over k of A(i, k) s[k] code[k][j]: dx (i: rows, k: outputs, held rows w) and dweight (i: outputs, k: rows, held rows x).  A's elements times the scale
// go in as sums of PARTS bf16 numbers.
struct GradArgs {
    const uint8_t *dy, *held;
    uint64_t dy_stride, held_stride;
    uint8_t *out;
    uint64_t out_stride;
    uint32_t out_type;
    float *partial;                  // [splits][n_i][n_j], or NULL: a sum is done by one workgroup
    int32_t n_i, n_j, n_k, held_bytes;
    int32_t k_each;                  // of a split
};

template <int PARTS> __device__ __forceinline__ void parts_of(float v, bf16 (&p)[PARTS])
{
#pragma unroll
    for (int q = 0; q < PARTS; ++q) {
        // cut off, not rounded, but for the last: no part is beyond the range.  What an infinity leaves is nothing.
        const uint32_t bits = __builtin_bit_cast(uint32_t, v) & 0xFFFF0000u;
        const float head = __builtin_bit_cast(float, bits);
        if (q == PARTS - 1) p[q] = (bf16)v;
        else p[q] = __builtin_bit_cast(bf16, (uint16_t)(bits >> 16));
        const bool number = (__builtin_bit_cast(uint32_t, v) & 0x7F800000u) != 0x7F800000u;
        if (!number && q != PARTS - 1) p[q] = (bf16)v;
        v = number ? v - head : 0.f;
    }
}

__device__ __forceinline__ void store_as(void *p, uint32_t type, int64_t at, float v)
{
    if (type == RG_F32) static_cast<float *>(p)[at] = v;
    else if (type == RG_BF16) static_cast<bf16 *>(p)[at] = (bf16)v;
    else static_cast<f16 *>(p)[at] = (f16)v;
}

constexpr int GRAD_TILE = 64, GRAD_DEPTH = 32, GRAD_PITCH = GRAD_DEPTH + 8;

// ALONG: dy's rows run along k (dx); otherwise along i (dweight).
template <typename T, int PARTS, bool ALONG>
__global__ void __launch_bounds__(256) grad_kernel(GradArgs a)
{
    __shared__ __align__(16) bf16 left[PARTS][GRAD_TILE][GRAD_PITCH];
    __shared__ __align__(16) bf16 right[GRAD_TILE][GRAD_PITCH];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int32_t down = (a.n_i + GRAD_TILE - 1) / GRAD_TILE;
    const int32_t i0 = (int32_t)(blockIdx.x % (uint32_t)down) * GRAD_TILE, j0 = (int32_t)(blockIdx.x / (uint32_t)down) * GRAD_TILE;
    const int64_t k_first = (int64_t)blockIdx.y * a.k_each;
    const int32_t k_end = (int32_t)min((int64_t)a.n_k, k_first + a.k_each);
    f32x4 acc[2][2] = {};
    for (int32_t k0 = (int32_t)k_first; k0 < k_end; k0 += GRAD_DEPTH) {
        __syncthreads();
        for (int e = 0; e < 8; ++e) {
            const int q = (int)threadIdx.x * 8 + e;
            const int i = ALONG ? q / GRAD_DEPTH : q % GRAD_TILE, k = ALONG ? q % GRAD_DEPTH : q / GRAD_TILE;
            float v = 0.f;
            if (i0 + i < a.n_i && k0 + k < k_end) {
                const float s = *row_at<float>(a.held + a.held_bytes - 4, a.held_stride, k0 + k);
                v = (float)(ALONG ? row_at<T>(a.dy, a.dy_stride, i0 + i)[k0 + k] : row_at<T>(a.dy, a.dy_stride, k0 + k)[i0 + i]) * s;
            }
            bf16 p[PARTS];
            parts_of<PARTS>(v, p);
            for (int x = 0; x < PARTS; ++x) left[x][i][k] = p[x];
        }
        for (int e = 0; e < 8; ++e) {
            const int q = (int)threadIdx.x * 8 + e, j = q % GRAD_TILE, k = q / GRAD_TILE;
            right[j][k] = (bf16)(float)(j0 + j < a.n_j && k0 + k < k_end ? row_at<int8_t>(a.held, a.held_stride, k0 + k)[j0 + j] : (int8_t)0);
        }
        __syncthreads();
        for (int x = 0; x < PARTS; ++x)
            for (int bi = 0; bi < 2; ++bi)
                for (int bj = 0; bj < 2; ++bj) {
                    const bf16x8 l = *reinterpret_cast<const bf16x8 *>(&left[x][(wave >> 1) * 32 + bi * 16 + (lane & 15)][(lane >> 4) * 8]);
                    const bf16x8 r = *reinterpret_cast<const bf16x8 *>(&right[(wave & 1) * 32 + bj * 16 + (lane & 15)][(lane >> 4) * 8]);
                    acc[bi][bj] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(r, l, acc[bi][bj], 0, 0, 0);
                }
    }
    for (int bi = 0; bi < 2; ++bi)
        for (int bj = 0; bj < 2; ++bj)
            for (int e = 0; e < 4; ++e) {
                const int32_t i = i0 + (wave >> 1) * 32 + bi * 16 + (lane & 15), j = j0 + (wave & 1) * 32 + bj * 16 + (lane >> 4) * 4 + e;
                if (i >= a.n_i || j >= a.n_j) continue;
                if (a.partial) a.partial[((int64_t)blockIdx.y * a.n_i + i) * a.n_j + j] = acc[bi][bj][e];
                else store_as(a.out + (uint64_t)i * a.out_stride, a.out_type, j, acc[bi][bj][e]);
            }
}

// The splits' sums, added up in their order.
__global__ void __launch_bounds__(256) grad_join_kernel(const float *partial, int32_t splits, int64_t n_i, int64_t n_j, uint8_t *out, uint64_t out_stride, uint32_t type)
{
    for (int64_t q = (int64_t)blockIdx.x * 256 + threadIdx.x; q < n_i * n_j; q += (int64_t)gridDim.x * 256) {
        float v = 0.f;
        for (int32_t s = 0; s < splits; ++s) v += partial[s * n_i * n_j + q];
        store_as(out + (uint64_t)(q / n_j) * out_stride, type, q % n_j, v);
    }
}

// Sums of dy's columns over a part of its rows: 64 columns to a workgroup, four rows at a time.
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

rg_status check_grid(uint64_t groups, uint32_t threads)
{
    if (groups <= MAX_WORK_ITEMS / threads) return RG_OK;
    set_error("a result of %llu tiles is more than a launch holds", (unsigned long long)groups);
    return RG_ERANGE;
}

// How the backward pass is cut, and where its scratch lies.
struct GradPlan {
    uint64_t dx_tiles, dw_tiles;
    int32_t dx_splits, dx_each, dw_splits, dw_each, bias_parts, bias_each;
    uint64_t bias_at, bytes;             // sums of dx, then of dweight in the same place; those of dbias
};

int32_t splits_of(uint64_t tiles, uint64_t n_k, int n_cu, int32_t *each)
{
    const uint64_t steps = (n_k + GRAD_DEPTH - 1) / GRAD_DEPTH;
    uint64_t splits = 1;
    while (tiles * splits * 2 <= (uint64_t)n_cu * 2 && steps >= splits * 2 * 4) splits *= 2;
    const uint64_t per = std::max<uint64_t>(1, (steps + splits - 1) / splits);
    *each = (int32_t)(per * GRAD_DEPTH);
    return (int32_t)std::max<uint64_t>(1, (steps + per - 1) / per);
}

GradPlan grad_plan(uint64_t n, uint64_t m, uint64_t d, int n_cu, bool dx, bool dw, bool db)
{
    GradPlan p{};
    uint64_t bytes = 0;
    const auto tiles = [](uint64_t i, uint64_t j) { return (i + GRAD_TILE - 1) / GRAD_TILE * ((j + GRAD_TILE - 1) / GRAD_TILE); };
    if (dx) {
        p.dx_tiles = tiles(n, d);
        p.dx_splits = splits_of(p.dx_tiles, m, n_cu, &p.dx_each);
        if (p.dx_splits > 1) bytes = std::max(bytes, (uint64_t)p.dx_splits * n * d * 4);
    }
    if (dw) {
        p.dw_tiles = tiles(m, d);
        p.dw_splits = splits_of(p.dw_tiles, n, n_cu, &p.dw_each);
        if (p.dw_splits > 1) bytes = std::max(bytes, (uint64_t)p.dw_splits * m * d * 4);
    }
    p.bias_at = (bytes + 15) / 16 * 16;
    if (db) {
        p.bias_parts = (int32_t)std::max<uint64_t>(1, std::min<uint64_t>(256, n / 64));
        p.bias_each = (int32_t)((n + p.bias_parts - 1) / p.bias_parts);
        bytes = p.bias_at + (uint64_t)p.bias_parts * m * 4;
    }
    p.bytes = bytes;
    return p;
}

template <typename T, int PARTS, bool ALONG> void launch_grad(uint64_t tiles, int32_t splits, const GradArgs &g, hipStream_t st)
{
    hipLaunchKernelGGL((grad_kernel<T, PARTS, ALONG>), dim3((uint32_t)tiles, (uint32_t)splits), dim3(256), 0, st, g);
}

template <bool ALONG> rg_status launch_grad_of(uint32_t type, uint64_t tiles, int32_t splits, GradArgs g, void *workspace, hipStream_t st)
{
    g.partial = splits > 1 ? static_cast<float *>(workspace) : nullptr;
    if (type == RG_F32) launch_grad<float, 3, ALONG>(tiles, splits, g, st);
    else if (type == RG_BF16) launch_grad<bf16, 2, ALONG>(tiles, splits, g, st);
    else launch_grad<f16, 2, ALONG>(tiles, splits, g, st);
    RG_HIP(hipGetLastError());
    if (splits > 1) {
        hipLaunchKernelGGL(grad_join_kernel, dim3((uint32_t)std::min<int64_t>(2048, ((int64_t)g.n_i * g.n_j + 255) / 256)), dim3(256), 0, st, g.partial, splits, (int64_t)g.n_i, (int64_t)g.n_j, g.out,
                           g.out_stride, g.out_type);
        RG_HIP(hipGetLastError());
    }
    return RG_OK;
}

}  // namespace
}  // namespace rg

using namespace rg;

extern "C" rg_status rg_rows8_product_workspace(uint64_t n_rows, uint64_t n_outs, uint64_t n_cols, uint64_t *bytes)
{
    if (!bytes) { set_error("null argument"); return RG_EINVAL; }
    RG_TRY(check_product_sizes(n_rows, n_outs, n_cols));
    *bytes = 0;
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
    RG_TRY(check_workspace(workspace, workspace_bytes, 0));
    ProductArgs a{};
    a.x = static_cast<const uint8_t *>(x); a.x_stride = x_stride;
    a.w = static_cast<const uint8_t *>(w); a.w_stride = w_stride;
    a.bias = bias; a.bias_type = bias_type;
    a.y = static_cast<uint8_t *>(y); a.y_stride = y_stride;
    a.n_rows = (int32_t)n_rows; a.n_outs = (int32_t)n_outs; a.n_cols = (int32_t)n_cols; a.held_bytes = (int32_t)held_bytes(n_cols);
    const hipStream_t st = as_stream(stream);
    const uint64_t tiles = (n_rows + 15) / 16 * ((n_outs + 15) / 16);
    RG_TRY(check_grid(tiles, 256));
    if (type == RG_F32) hipLaunchKernelGGL(product_few_kernel<float>, dim3((uint32_t)tiles), dim3(256), 0, st, a);
    else if (type == RG_BF16) hipLaunchKernelGGL(product_few_kernel<bf16>, dim3((uint32_t)tiles), dim3(256), 0, st, a);
    else hipLaunchKernelGGL(product_few_kernel<f16>, dim3((uint32_t)tiles), dim3(256), 0, st, a);
    RG_HIP(hipGetLastError());
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
    RG_TRY(check_grid(p.dx_tiles, 256));
    RG_TRY(check_grid(p.dw_tiles, 256));
    RG_TRY(check_grid((n_outs + 63) / 64, 256));
    const hipStream_t st = as_stream(stream);
    GradArgs g{};
    g.dy = static_cast<const uint8_t *>(dy); g.dy_stride = dy_stride;
    g.n_j = (int32_t)n_cols; g.held_bytes = (int32_t)held_bytes(n_cols);
    if (dx && n_rows) {
        g.held = static_cast<const uint8_t *>(w); g.held_stride = w_stride;
        g.out = static_cast<uint8_t *>(dx); g.out_stride = dx_stride; g.out_type = type;
        g.n_i = (int32_t)n_rows; g.n_k = (int32_t)n_outs; g.k_each = p.dx_each;
        RG_TRY(launch_grad_of<true>(type, p.dx_tiles, p.dx_splits, g, workspace, st));
    }
    if (dweight && n_outs) {
        g.held = static_cast<const uint8_t *>(x); g.held_stride = x_stride;
        g.out = static_cast<uint8_t *>(dweight); g.out_stride = dweight_stride; g.out_type = weight_type;
        g.n_i = (int32_t)n_outs; g.n_k = (int32_t)n_rows; g.k_each = p.dw_each;
        RG_TRY(launch_grad_of<false>(type, p.dw_tiles, p.dw_splits, g, workspace, st));
    }
    if (dbias && n_outs) {
        float *partial = reinterpret_cast<float *>(static_cast<uint8_t *>(workspace) + p.bias_at);
        const dim3 grid((uint32_t)((n_outs + 63) / 64), (uint32_t)p.bias_parts);
        const uint8_t *from = static_cast<const uint8_t *>(dy);
        if (type == RG_F32) hipLaunchKernelGGL(bias_sums_kernel<float>, grid, dim3(256), 0, st, from, dy_stride, (int32_t)n_rows, (int32_t)n_outs, p.bias_each, partial);
        else if (type == RG_BF16) hipLaunchKernelGGL(bias_sums_kernel<bf16>, grid, dim3(256), 0, st, from, dy_stride, (int32_t)n_rows, (int32_t)n_outs, p.bias_each, partial);
        else hipLaunchKernelGGL(bias_sums_kernel<f16>, grid, dim3(256), 0, st, from, dy_stride, (int32_t)n_rows, (int32_t)n_outs, p.bias_each, partial);
        RG_HIP(hipGetLastError());
        hipLaunchKernelGGL(grad_join_kernel, dim3((uint32_t)std::min<uint64_t>(2048, (n_outs + 255) / 256)), dim3(256), 0, st, partial, p.bias_parts, (int64_t)1, (int64_t)n_outs,
                           static_cast<uint8_t *>(dbias), (uint64_t)0, weight_type);
        RG_HIP(hipGetLastError());
    }
    return RG_OK;
}
