// Rows held in 8 bits: written (rg_quantize_rows) and read back (rg_dequantize_rows).
//
// A held row is its codes, zeros, and its scale in the last four bytes, so that everything that moves rows moves held ones: a quarter of the bytes of fp32 through the
// cache, the gather and the host link.  With s = max|x| / 127 (rounded to fp32; at least 2^-126, and 127 s is a number) a code is the whole number nearest to the exact quotient x / s, ties to
// even: what is read back is off by s / 2 at most.
//
// Both directions are bound by HBM: a row is read once into registers and written once.  It belongs to 8 to 64 lanes of a wave, or to a workgroup, whatever holds
// it in 32 elements a lane or fewer; rows beyond that are read twice.
#include "rg_internal.h"
#include "rg_elements.h"
#include "rg_launch.h"

namespace rg {

namespace {

struct HoldArgs {
    const uint8_t *from;             // elements, or held rows
    uint64_t from_stride;
    uint8_t *to;
    uint64_t to_stride;
    const int64_t *rows;             // positions in `from`, or NULL: every row in its place
    int64_t n_from, n_out;
    int32_t n_cols, held_bytes;
};

// The row that output i is made of: its address, or NULL with `none` (position -1: zeros) or without (a position beyond the rows: all NaN).
__device__ __forceinline__ const uint8_t *row_from(const HoldArgs &a, int64_t i, bool &none)
{
    const int64_t r = a.rows ? a.rows[i] : i;
    none = r == -1;
    return r >= 0 && r < a.n_from ? a.from + (uint64_t)r * a.from_stride : nullptr;
}

__device__ __forceinline__ uint32_t magnitude(float v) { return __builtin_bit_cast(uint32_t, v) & 0x7FFFFFFFu; }   // compares as |v| does; infinities and NaN above all numbers

template <int CTRL> __device__ __forceinline__ uint32_t dpp_max(uint32_t v)
{
    return max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, CTRL, 0xF, 0xF, true));
}
// The largest over groups of LANES lanes (up to 64), in every lane of the group.
template <int LANES> __device__ __forceinline__ uint32_t lanes_max(uint32_t v)
{
    v = dpp_max<0xB1>(v);                          // quad_perm 1 0 3 2
    v = dpp_max<0x4E>(v);                          // quad_perm 2 3 0 1
    v = dpp_max<0x141>(v);                         // row_half_mirror
    if constexpr (LANES >= 16) v = dpp_max<0x140>(v);        // row_mirror
    if constexpr (LANES >= 32) v = max(v, (uint32_t)__shfl_xor((int)v, 16));
    if constexpr (LANES >= 64) v = max(v, (uint32_t)__shfl_xor((int)v, 32));
    return v;
}
// The same over a row's lanes; beyond a wave they meet in LDS, in slots taken by turns: whoever writes a slot again has passed a barrier that every
// wave reaches only after it has read that slot.
template <int LANES> __device__ __forceinline__ uint32_t row_max(uint32_t v, uint32_t (*slots)[16], uint32_t &turn)
{
    v = lanes_max<(LANES < 64 ? LANES : 64)>(v);
    if constexpr (LANES > 64) {
        uint32_t *s = slots[turn & 1];
        ++turn;
        if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
        __syncthreads();
        v = 0;
#pragma unroll
        for (int w = 0; w < LANES / 64; ++w) v = max(v, s[w]);
    }
    return v;
}

constexpr float SCALE_MOST = 0x1.020406p+121f;      // the largest of which 127 are a number
struct Scale {
    float s, inverse, half;
    bool finite;
    __device__ __forceinline__ explicit Scale(uint32_t largest)
    {
        finite = largest < 0x7F800000u;
        s = fminf(fmaxf(__builtin_bit_cast(float, largest) / 127.f, 0x1p-126f), SCALE_MOST);
        inverse = 1.f / s;
        half = 0.5f * s;
    }
    __device__ __forceinline__ float stored() const { return finite ? s : __builtin_nanf(""); }
    // The whole number nearest to x / s, ties to even, of the exact quotient: q from the rounded one is off by one at most, and what it leaves, x - q s, is exact
    // in 32 bits (a multiple of the coarser of both units, and not much more than s / 2).
    __device__ __forceinline__ int code(float x) const
    {
        float q = rintf(x * inverse);
        const float rest = fmaf(-q, s, x), off = fabsf(rest);
        if (off >= half && (off > half || ((int)q & 1))) q += copysignf(1.f, rest);
        return finite ? (int)q : 0;
    }
};

// Elements [c, c + V) of a row, zeros beyond it.
template <typename T, int V> __device__ __forceinline__ void load_inside(const uint8_t *row, int32_t c, int32_t n_cols, float (&v)[V])
{
    const T *p = reinterpret_cast<const T *>(row) + c;
    if (row && c + V <= n_cols) {
        load_pack<T, V>(p, v);
    } else {
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = row && c + e < n_cols ? (float)p[e] : 0.f;
    }
}

// The codes of V elements from c on, as they lie in a held row: four to a word, the row's last word the scale.
template <int V> __device__ __forceinline__ void store_codes(uint8_t *row, int32_t c, int32_t held_bytes, const Scale &s, const float (&v)[V])
{
    typedef uint32_t Words __attribute__((ext_vector_type(V / 4)));
    uint32_t w[V / 4];
#pragma unroll
    for (int k = 0; k < V / 4; ++k) {
        w[k] = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) w[k] |= ((uint32_t)s.code(v[k * 4 + e]) & 0xFFu) << (8 * e);
    }
    if (c + V == held_bytes) w[V / 4 - 1] = __builtin_bit_cast(uint32_t, s.stored());
    if constexpr (V == 4) {
        *reinterpret_cast<uint32_t *>(row + c) = w[0];
    } else {
        Words x;
#pragma unroll
        for (int k = 0; k < V / 4; ++k) x[k] = w[k];
        *reinterpret_cast<Words *>(row + c) = x;
    }
}

// (NaN where a position is beyond the rows.)
__device__ __forceinline__ uint32_t with_missing(uint32_t largest, const uint8_t *row, bool none) { return row || none ? largest : 0x7FC00000u; }

template <typename T, int LANES, int NV>
__global__ void __launch_bounds__(LANES > 256 ? LANES : 256) quantize_rows_kernel(HoldArgs a)
{
    constexpr int V = 16 / sizeof(T), THREADS = LANES > 256 ? LANES : 256, GROUPS = THREADS / LANES;
    __shared__ uint32_t slots[2][16];
    uint32_t turn = 0;
    const int32_t lane = (int32_t)(threadIdx.x % LANES);
    for (int64_t i = (int64_t)blockIdx.x * GROUPS + threadIdx.x / LANES; i < a.n_out; i += (int64_t)gridDim.x * GROUPS) {
        bool none;
        const uint8_t *row = row_from(a, i, none);
        float v[NV][V];
#pragma unroll
        for (int j = 0; j < NV; ++j) load_inside<T, V>(row, (j * LANES + lane) * V, a.n_cols, v[j]);
        uint32_t largest = 0;
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int e = 0; e < V; ++e) largest = max(largest, magnitude(v[j][e]));
        const Scale s(with_missing(row_max<LANES>(largest, slots, turn), row, none));
        uint8_t *to = a.to + (uint64_t)i * a.to_stride;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int32_t c = (j * LANES + lane) * V;
            if (c < a.held_bytes) store_codes<V>(to, c, a.held_bytes, s, v[j]);
        }
    }
}

// Rows beyond what registers hold: read once for the largest, and again, out of the caches, for the codes.
template <typename T>
__global__ void __launch_bounds__(1024) quantize_long_rows_kernel(HoldArgs a)
{
    constexpr int V = 16 / sizeof(T), STEP = 1024 * V;
    __shared__ uint32_t slots[2][16];
    uint32_t turn = 0;
    for (int64_t i = blockIdx.x; i < a.n_out; i += gridDim.x) {
        bool none;
        const uint8_t *row = row_from(a, i, none);
        uint32_t largest = 0;
        for (int32_t c = (int32_t)threadIdx.x * V; c < a.n_cols; c += STEP) {
            float v[V];
            load_inside<T, V>(row, c, a.n_cols, v);
#pragma unroll
            for (int e = 0; e < V; ++e) largest = max(largest, magnitude(v[e]));
        }
        const Scale s(with_missing(row_max<1024>(largest, slots, turn), row, none));
        uint8_t *to = a.to + (uint64_t)i * a.to_stride;
        for (int32_t c = (int32_t)threadIdx.x * V; c < a.held_bytes; c += STEP) {
            float v[V];
            load_inside<T, V>(row, c, a.n_cols, v);
            store_codes<V>(to, c, a.held_bytes, s, v);
        }
    }
}

// V codes of a held row at a time.  The last pack of a row is the one that ends at the row's end: it overlaps its predecessor, and both write the same there.
template <typename T, int V, int LANES>
__global__ void __launch_bounds__(256) dequantize_rows_kernel(HoldArgs a)
{
    constexpr int GROUPS = 256 / LANES;
    const int32_t lane = (int32_t)(threadIdx.x % LANES);
    for (int64_t i = (int64_t)blockIdx.x * GROUPS + threadIdx.x / LANES; i < a.n_out; i += (int64_t)gridDim.x * GROUPS) {
        bool none;
        const uint8_t *row = row_from(a, i, none);
        const float s = row ? *reinterpret_cast<const float *>(row + a.held_bytes - 4) : none ? 0.f : __builtin_nanf("");
        T *to = reinterpret_cast<T *>(a.to + (uint64_t)i * a.to_stride);
        for (int32_t at = lane * V; at < a.n_cols; at += LANES * V) {
            const int32_t c = min(at, a.n_cols - V);
            typename PackOf<int8_t, V>::type q = {};
            if (row) q = load_raw<int8_t, V>(reinterpret_cast<const int8_t *>(row) + c);
            float v[V];
            unpack<int8_t, V>(q, v);
#pragma unroll
            for (int e = 0; e < V; ++e) v[e] *= s;
            store_pack<T, V>(to + c, v);
        }
    }
}

template <typename T, int LANES, int NV> void launch_quantize(const HoldShape &s, const HoldArgs &a, hipStream_t st)
{
    hipLaunchKernelGGL((quantize_rows_kernel<T, LANES, NV>), dim3(s.grid), dim3(LANES > 256 ? LANES : 256), 0, st, a);
}

template <typename T> bool launch_quantize_of(const HoldShape &s, const HoldArgs &a, hipStream_t st)
{
    switch (s.lanes * 16 + s.packs) {
    case 0: hipLaunchKernelGGL(quantize_long_rows_kernel<T>, dim3(s.grid), dim3(1024), 0, st, a); return true;
    case 8 * 16 + 1: launch_quantize<T, 8, 1>(s, a, st); return true;
    case 16 * 16 + 1: launch_quantize<T, 16, 1>(s, a, st); return true;
    case 32 * 16 + 1: launch_quantize<T, 32, 1>(s, a, st); return true;
    case 64 * 16 + 1: launch_quantize<T, 64, 1>(s, a, st); return true;
    case 64 * 16 + 2: launch_quantize<T, 64, 2>(s, a, st); return true;
    case 64 * 16 + 3: launch_quantize<T, 64, 3>(s, a, st); return true;
    case 64 * 16 + 4: launch_quantize<T, 64, 4>(s, a, st); return true;
    case 256 * 16 + 2: launch_quantize<T, 256, 2>(s, a, st); return true;
    case 256 * 16 + 3: launch_quantize<T, 256, 3>(s, a, st); return true;
    case 256 * 16 + 4: launch_quantize<T, 256, 4>(s, a, st); return true;
    case 1024 * 16 + 2: launch_quantize<T, 1024, 2>(s, a, st); return true;
    case 1024 * 16 + 3: launch_quantize<T, 1024, 3>(s, a, st); return true;
    case 1024 * 16 + 4: launch_quantize<T, 1024, 4>(s, a, st); return true;
    }
    return false;
}

template <typename T, int V> void launch_dequantize(const HoldShape &s, const HoldArgs &a, hipStream_t st)
{
    if (s.lanes == 8) hipLaunchKernelGGL((dequantize_rows_kernel<T, V, 8>), dim3(s.grid), dim3(256), 0, st, a);
    else if (s.lanes == 16) hipLaunchKernelGGL((dequantize_rows_kernel<T, V, 16>), dim3(s.grid), dim3(256), 0, st, a);
    else if (s.lanes == 32) hipLaunchKernelGGL((dequantize_rows_kernel<T, V, 32>), dim3(s.grid), dim3(256), 0, st, a);
    else if (s.lanes == 64) hipLaunchKernelGGL((dequantize_rows_kernel<T, V, 64>), dim3(s.grid), dim3(256), 0, st, a);
    else hipLaunchKernelGGL((dequantize_rows_kernel<T, V, 256>), dim3(s.grid), dim3(256), 0, st, a);
}

template <typename T> void launch_dequantize_of(const HoldShape &s, const HoldArgs &a, hipStream_t st)
{
    if (s.pack == 1) launch_dequantize<T, 1>(s, a, st);
    else launch_dequantize<T, 16 / sizeof(T)>(s, a, st);
}

rg_status check_hold(uint64_t n_rows, uint64_t n_cols, uint32_t type, const int64_t *rows, uint64_t n_out)
{
    if (!element_bytes(type)) { set_error("type %u is none of RG_F32, RG_BF16, RG_F16", type); return RG_EINVAL; }
    if (n_cols == 0) { set_error("rows of no elements are not held"); return RG_EINVAL; }
    if (n_cols > RG_MAX_HELD_COLS || n_rows >= 1ull << 40 || n_out >= 1ull << 40) {
        set_error("%llu rows of %llu elements, %llu of them wanted, are beyond the limits (2^40, %u, 2^40)", (unsigned long long)n_rows, (unsigned long long)n_cols, (unsigned long long)n_out, RG_MAX_HELD_COLS);
        return RG_ERANGE;
    }
    if (!rows && n_out && n_out != n_rows) { set_error("%llu rows of %llu without their positions", (unsigned long long)n_out, (unsigned long long)n_rows); return RG_EINVAL; }
    if (reinterpret_cast<uintptr_t>(rows) % 8) { set_error("rows is not aligned for its type"); return RG_EINVAL; }
    return RG_OK;
}

HoldArgs hold_args(const void *from, uint64_t from_stride, uint64_t n_from, const int64_t *rows, uint64_t n_out, uint64_t n_cols, void *to, uint64_t to_stride)
{
    HoldArgs a{};
    a.from = static_cast<const uint8_t *>(from); a.from_stride = from_stride; a.n_from = (int64_t)n_from;
    a.to = static_cast<uint8_t *>(to); a.to_stride = to_stride; a.n_out = (int64_t)n_out;
    a.rows = rows;
    a.n_cols = (int32_t)n_cols; a.held_bytes = (int32_t)held_bytes(n_cols);
    return a;
}

}  // namespace

rg_status check_elements(const char *what, const void *p, uint64_t stride, uint64_t n_rows, uint64_t n_cols, uint32_t bytes, bool output)
{
    if (n_rows == 0) return RG_OK;
    if (!p) { set_error("%s is null", what); return RG_EINVAL; }
    if ((reinterpret_cast<uintptr_t>(p) | stride) % bytes) { set_error("%s: address and stride have to be multiples of %u bytes", what, bytes); return RG_EINVAL; }
    if (output && n_rows > 1 && stride < n_cols * bytes) { set_error("%s: a stride of %llu bytes is less than a row", what, (unsigned long long)stride); return RG_EINVAL; }
    if (stride > 1ull << 40) { set_error("%s: a stride of %llu bytes is beyond the limit (2^40)", what, (unsigned long long)stride); return RG_ERANGE; }
    return RG_OK;
}

rg_status check_held(const char *what, const void *p, uint64_t stride, uint64_t n_rows, uint64_t n_cols, bool output)
{
    if (n_rows == 0) return RG_OK;
    if (!p) { set_error("%s is null", what); return RG_EINVAL; }
    if ((reinterpret_cast<uintptr_t>(p) | stride) % 16) { set_error("%s: address and stride of held rows have to be multiples of 16 bytes", what); return RG_EINVAL; }
    if (output && n_rows > 1 && stride < held_bytes(n_cols)) { set_error("%s: a stride of %llu bytes is less than a held row", what, (unsigned long long)stride); return RG_EINVAL; }
    if (stride > 1ull << 40) { set_error("%s: a stride of %llu bytes is beyond the limit (2^40)", what, (unsigned long long)stride); return RG_ERANGE; }
    return RG_OK;
}

}  // namespace rg

using namespace rg;

extern "C" rg_status rg_rows8_bytes(uint64_t n_cols, uint64_t *bytes)
{
    if (!bytes) { set_error("null argument"); return RG_EINVAL; }
    RG_TRY(check_hold(0, n_cols, RG_F32, nullptr, 0));
    *bytes = held_bytes(n_cols);
    return RG_OK;
}

extern "C" rg_status rg_quantize_rows(const void *x, uint64_t x_stride, uint64_t n_rows, uint64_t n_cols, uint32_t type, const int64_t *rows, uint64_t n_out,
                                      void *held, uint64_t held_stride, void *stream)
{
    RG_TRY(check_hold(n_rows, n_cols, type, rows, n_out));
    const uint32_t bytes = element_bytes(type);
    RG_TRY(check_elements("x", x, x_stride, n_rows, n_cols, bytes, false));
    RG_TRY(check_held("held", held, held_stride, n_out, n_cols, true));
    if (n_out == 0) return RG_OK;
    int n_cu = 0;
    RG_TRY(compute_units(&n_cu));
    const HoldArgs a = hold_args(x, x_stride, n_rows, rows, n_out, n_cols, held, held_stride);
    const HoldShape s = hold_shape((int64_t)n_out, (int64_t)n_cols, (int)bytes, n_cu);
    const hipStream_t st = as_stream(stream);
    const bool found = type == RG_F32 ? launch_quantize_of<float>(s, a, st) : type == RG_BF16 ? launch_quantize_of<bf16>(s, a, st) : launch_quantize_of<f16>(s, a, st);
    if (!found) { set_error("no kernel for rows of %llu elements", (unsigned long long)n_cols); return RG_EHIP; }
    RG_HIP(hipGetLastError());
    return RG_OK;
}

extern "C" rg_status rg_dequantize_rows(const void *held, uint64_t held_stride, uint64_t n_rows, uint64_t n_cols, const int64_t *rows, uint64_t n_out,
                                        uint32_t type, void *out, uint64_t out_stride, void *stream)
{
    RG_TRY(check_hold(n_rows, n_cols, type, rows, n_out));
    const uint32_t bytes = element_bytes(type);
    RG_TRY(check_held("held", held, held_stride, n_rows, n_cols, false));
    RG_TRY(check_elements("out", out, out_stride, n_out, n_cols, bytes, true));
    if (n_out == 0) return RG_OK;
    int n_cu = 0;
    RG_TRY(compute_units(&n_cu));
    const HoldArgs a = hold_args(held, held_stride, n_rows, rows, n_out, n_cols, out, out_stride);
    const HoldShape s = read_shape((int64_t)n_out, (int64_t)n_cols, (int)bytes, n_cu);
    const hipStream_t st = as_stream(stream);
    if (type == RG_F32) launch_dequantize_of<float>(s, a, st);
    else if (type == RG_BF16) launch_dequantize_of<bf16>(s, a, st);
    else launch_dequantize_of<f16>(s, a, st);
    RG_HIP(hipGetLastError());
    return RG_OK;
}
