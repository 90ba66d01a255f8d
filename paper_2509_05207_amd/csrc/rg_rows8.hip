// Rows held in 8 bits: written (rg_quantize_rows) and read back (rg_dequantize_rows).
//
// A held row is its codes, zeros, and its scale in the last four bytes, so that everything that moves rows moves held ones: a quarter of the bytes of fp32 through the
// cache, the gather and the host link.  With s = max|x| / 127 (the fp32 product with the fp32 number next to 1 / 127, as torch divides by 127 on this
// device, so that rows held by either are the same; at least 2^-126, and 127 s is a number) a code is the whole number nearest to the exact quotient x / s, ties to
// even: what is read back is off by s / 2 at most.
//
// Both directions are bound by HBM: a row is read once into registers and written once.  It belongs to 8 to 64 lanes of a wave, or to a workgroup, whatever holds
// it in 40 elements a lane or fewer; rows beyond that are read twice.
// 199,000 x 602 in fp32: written 111 us (5.4 TB/s), read back 137 (4.4 TB/s; results past the caches), where a copy reaches 5.1; 200,000 x 256 in bf16 by positions out of a million rows
// 48 and 25; 199,000 x 602 to bf16 out of 233,000 rows 78 (4.6 TB/s).
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

// The position of output i's row.
__device__ __forceinline__ int64_t position(const HoldArgs &a, int64_t i) { return a.rows ? a.rows[i] : i; }

// The row at a position: its address, or NULL with `none` (position -1: zeros) or without (a position beyond the rows: all NaN).
__device__ __forceinline__ const uint8_t *row_from(const HoldArgs &a, int64_t r, bool &none)
{
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

constexpr float ONE_127TH = 0x1.020408p-7f;         // the largest element over the scale stays within 2^-22 of 127, so codes do
constexpr float SCALE_MOST = 0x1.020406p+121f;      // the largest of which 127 are a number
constexpr float ROUNDER = 12582912.f;               // 1.5 * 2^23: a sum with it is a whole number, which is in its last bits
struct Scale {
    float s, inverse, half;
    bool finite;
    __device__ __forceinline__ explicit Scale(uint32_t largest)
    {
        finite = largest < 0x7F800000u;
        s = fminf(fmaxf(__builtin_bit_cast(float, largest) * ONE_127TH, 0x1p-126f), SCALE_MOST);
        inverse = __builtin_amdgcn_rcpf(s);
        half = 0.5f * s;
    }
    __device__ __forceinline__ float stored() const { return finite ? s : __builtin_nanf(""); }
    // x plus ROUNDER where x / s is the whole number that the rounded quotient says, and what that leaves, x - q s.  q is off from the exact quotient's nearest whole number by one at
    // most, and the rest, which is exact in 32 bits (x itself where q is zero; else a multiple of half of s's unit, and not much more than s / 2), tells.
    __device__ __forceinline__ float near(float x, float &rest) const
    {
        const float q = fmaf(x, inverse, ROUNDER);
        rest = fmaf(ROUNDER - q, s, x);
        return q;
    }
    // The whole number nearest to the exact quotient, ties to even.
    __device__ __forceinline__ float exact(float x) const
    {
        float rest;
        const float q = near(x, rest), off = fabsf(rest);
        return off > half || (off == half && (__builtin_bit_cast(uint32_t, q) & 1)) ? q + copysignf(1.f, rest) : q;
    }
};

// Four codes out of the last bytes of their numbers.
__device__ __forceinline__ uint32_t four_codes(float a, float b, float c, float d)
{
    const uint32_t lo = __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, b), __builtin_bit_cast(uint32_t, a), 0x0C0C0400u);
    const uint32_t hi = __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, d), __builtin_bit_cast(uint32_t, c), 0x0C0C0400u);
    return lo | hi << 16;
}

// The codes of V elements, four to a word.
template <int V> __device__ __forceinline__ void codes_of(const Scale &s, const float (&v)[V], uint32_t (&w)[V / 4])
{
    float q[V], worst = 0.f;
#pragma unroll
    for (int e = 0; e < V; ++e) {
        float rest;
        q[e] = s.near(v[e], rest);
        worst = fmaxf(worst, fabsf(rest));
    }
    if (__builtin_expect(__ballot(worst >= s.half) != 0, 0))           // next to the border between two codes: one element of some thousands
#pragma unroll
        for (int e = 0; e < V; ++e) q[e] = s.exact(v[e]);
#pragma unroll
    for (int k = 0; k < V / 4; ++k) w[k] = s.finite ? four_codes(q[k * 4], q[k * 4 + 1], q[k * 4 + 2], q[k * 4 + 3]) : 0;
}

// Elements [c, c + V) of a row as they are, zeros beyond it.
template <typename T, int V> __device__ __forceinline__ typename PackOf<T, V>::type load_inside(const uint8_t *row, int32_t c, int32_t n_cols)
{
    typename PackOf<T, V>::type raw = {};
    const T *p = reinterpret_cast<const T *>(row) + c;
    if (row && c + V <= n_cols) {
        raw = load_raw<T, V>(p);
    } else if (row) {
#pragma unroll
        for (int e = 0; e < V; ++e)
            if (c + e < n_cols) raw[e] = p[e];
    }
    return raw;
}

// Words from c on as they lie in a held row, of which the last is the scale.
template <int V> __device__ __forceinline__ void store_codes(uint8_t *row, int32_t c, int32_t held_bytes, const Scale &s, uint32_t (&w)[V / 4])
{
    typedef uint32_t Two __attribute__((ext_vector_type(2)));
    if (c >= held_bytes) return;
    if (c + V == held_bytes) w[V / 4 - 1] = __builtin_bit_cast(uint32_t, s.stored());
    if constexpr (V == 4) *reinterpret_cast<uint32_t *>(row + c) = w[0];
    else *reinterpret_cast<Two *>(row + c) = Two{w[0], w[1]};
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
    const int64_t step = (int64_t)gridDim.x * GROUPS;
    int64_t i = (int64_t)blockIdx.x * GROUPS + threadIdx.x / LANES;
    typename PackOf<T, V>::type next[NV];
    const uint8_t *row = nullptr;
    bool none = true;
    // The position of the next row; the one behind it is asked for ahead of the row's elements, since what is asked for first arrives first.
    int64_t at = i < a.n_out ? position(a, i) : 0;
    const auto load = [&] {
        row = row_from(a, at, none);
        if (i + step < a.n_out) at = position(a, i + step);
#pragma unroll
        for (int j = 0; j < NV; ++j) next[j] = load_inside<T, V>(row, (j * LANES + lane) * V, a.n_cols);
    };
    if (i < a.n_out) load();
    while (i < a.n_out) {
        float v[NV][V];
        uint32_t largest = 0;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            unpack<T, V>(next[j], v[j]);
#pragma unroll
            for (int e = 0; e < V; ++e) largest = max(largest, magnitude(v[j][e]));
        }
        largest = with_missing(row_max<LANES>(largest, slots, turn), row, none);
        uint8_t *to = a.to + (uint64_t)i * a.to_stride;
        i += step;
        if (i < a.n_out) load();                                       // the next row is on its way while this one's codes are made
        const Scale s(largest);
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            uint32_t w[V / 4];
            codes_of<V>(s, v[j], w);
            store_codes<V>(to, (j * LANES + lane) * V, a.held_bytes, s, w);
        }
    }
}

// Rows beyond what registers hold: read once for the largest, and again, backwards, so that what the first pass read last is in the caches still, for the codes.  704 x 131,072 in fp32: 141 us, where bytes
// read once would take 90.
template <typename T>
__global__ void __launch_bounds__(1024) quantize_long_rows_kernel(HoldArgs a)
{
    constexpr int V = 16 / sizeof(T), STEP = 1024 * V;
    __shared__ uint32_t slots[2][16];
    uint32_t turn = 0;
    for (int64_t i = blockIdx.x; i < a.n_out; i += gridDim.x) {
        bool none;
        const uint8_t *row = row_from(a, position(a, i), none);
        uint32_t largest = 0;
        for (int32_t c = (int32_t)threadIdx.x * V; c < a.n_cols; c += STEP) {
            float v[V];
            unpack<T, V>(load_inside<T, V>(row, c, a.n_cols), v);
#pragma unroll
            for (int e = 0; e < V; ++e) largest = max(largest, magnitude(v[e]));
        }
        const Scale s(with_missing(row_max<1024>(largest, slots, turn), row, none));
        uint8_t *to = a.to + (uint64_t)i * a.to_stride;
        for (int32_t c = (int32_t)threadIdx.x * V + (a.held_bytes - 1) / STEP * STEP; c >= 0; c -= STEP) {       // backwards: what was read last is in the caches still
            float v[V];
            uint32_t w[V / 4];
            unpack<T, V>(load_inside<T, V>(row, c, a.n_cols), v);
            codes_of<V>(s, v, w);
            store_codes<V>(to, c, a.held_bytes, s, w);
        }
    }
}

// V codes of a held row at a time.  The last pack of a row is the one that ends at the row's end: it overlaps its predecessor, and both write the same there.
// PAST: past the caches.
template <typename T, int V, bool PAST> __device__ __forceinline__ void store_values(T *to, const typename PackOf<int8_t, V>::type &q, float s)
{
    typedef typename PackOf<T, V>::type P __attribute__((aligned(alignof(T))));
    float v[V];
    unpack<int8_t, V>(q, v);
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] *= s;
    if constexpr (PAST && V > 1) {
        P raw;
#pragma unroll
        for (int e = 0; e < V; ++e) raw[e] = (T)v[e];
        __builtin_nontemporal_store(raw, reinterpret_cast<P *>(to));
    } else {
        store_pack<T, V>(to, v);
    }
}

template <typename T, int V, int LANES, int NV, bool PAST>
__global__ void __launch_bounds__(256) dequantize_rows_kernel(HoldArgs a)
{
    constexpr int GROUPS = 256 / LANES;
    typedef typename PackOf<int8_t, V>::type Codes;
    const int32_t lane = (int32_t)(threadIdx.x % LANES);
    const int64_t step = (int64_t)gridDim.x * GROUPS;
    int64_t i = (int64_t)blockIdx.x * GROUPS + threadIdx.x / LANES;
    if (i >= a.n_out) return;
    Codes next[NV];
    float next_scale = 0.f;
    int64_t from = position(a, i);
    const auto load = [&] {
        bool none;
        const uint8_t *row = row_from(a, from, none);
        if (i + step < a.n_out) from = position(a, i + step);              // ahead of the row's codes, as above
        next_scale = row ? *reinterpret_cast<const float *>(row + a.held_bytes - 4) : none ? 0.f : __builtin_nanf("");
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int32_t at = (j * LANES + lane) * V;
            next[j] = Codes{};
            if (row && at < a.n_cols) next[j] = load_raw<int8_t, V>(reinterpret_cast<const int8_t *>(row) + min(at, a.n_cols - V));
        }
    };
    load();
    while (i < a.n_out) {
        Codes now[NV];
#pragma unroll
        for (int j = 0; j < NV; ++j) now[j] = next[j];
        const float s = next_scale;
        T *to = reinterpret_cast<T *>(a.to + (uint64_t)i * a.to_stride);
        i += step;
        if (i < a.n_out) load();
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int32_t at = (j * LANES + lane) * V;
            if (at < a.n_cols) store_values<T, V, PAST>(to + min(at, a.n_cols - V), now[j], s);
        }
    }
}

// Long rows, by parts of four packs a thread.
template <typename T, int V, bool PAST>
__global__ void __launch_bounds__(256) dequantize_long_rows_kernel(HoldArgs a)
{
    typedef typename PackOf<int8_t, V>::type Codes;
    constexpr int PACKS = 4;
    const int32_t parts = (a.n_cols + 256 * V * PACKS - 1) / (256 * V * PACKS);
    for (int64_t u = blockIdx.x; u < a.n_out * parts; u += gridDim.x) {
        const int64_t i = u / parts;
        const int32_t at = (int32_t)(u - i * parts) * (256 * V * PACKS) + (int32_t)threadIdx.x * V;
        bool none;
        const uint8_t *row = row_from(a, position(a, i), none);
        const float s = row ? *reinterpret_cast<const float *>(row + a.held_bytes - 4) : none ? 0.f : __builtin_nanf("");
        T *to = reinterpret_cast<T *>(a.to + (uint64_t)i * a.to_stride);
        Codes q[PACKS];
#pragma unroll
        for (int j = 0; j < PACKS; ++j) {
            q[j] = Codes{};
            if (row && at + j * 256 * V < a.n_cols) q[j] = load_raw<int8_t, V>(reinterpret_cast<const int8_t *>(row) + min(at + j * 256 * V, a.n_cols - V));
        }
#pragma unroll
        for (int j = 0; j < PACKS; ++j)
            if (at + j * 256 * V < a.n_cols) store_values<T, V, PAST>(to + min(at + j * 256 * V, a.n_cols - V), q[j], s);
    }
}

template <typename T, int LANES, int NV> bool launch_quantize(const HoldShape &s, const HoldArgs &a, hipStream_t st)
{
    hipLaunchKernelGGL((quantize_rows_kernel<T, LANES, NV>), dim3(s.grid), dim3(LANES > 256 ? LANES : 256), 0, st, a);
    return true;
}

template <typename T> bool launch_quantize_of(const HoldShape &s, const HoldArgs &a, hipStream_t st)
{
    switch (s.lanes * 16 + s.packs) {
    case 0: hipLaunchKernelGGL(quantize_long_rows_kernel<T>, dim3(s.grid), dim3(1024), 0, st, a); return true;
    case 8 * 16 + 1: return launch_quantize<T, 8, 1>(s, a, st);
    case 16 * 16 + 1: return launch_quantize<T, 16, 1>(s, a, st);
    case 32 * 16 + 1: return launch_quantize<T, 32, 1>(s, a, st);
    case 32 * 16 + 2: return launch_quantize<T, 32, 2>(s, a, st);
    case 32 * 16 + 3: return launch_quantize<T, 32, 3>(s, a, st);
    case 32 * 16 + 4: return launch_quantize<T, 32, 4>(s, a, st);
    case 32 * 16 + 5: return launch_quantize<T, 32, 5>(s, a, st);
    case 64 * 16 + 3: return launch_quantize<T, 64, 3>(s, a, st);
    case 64 * 16 + 4: return launch_quantize<T, 64, 4>(s, a, st);
    case 64 * 16 + 5: return launch_quantize<T, 64, 5>(s, a, st);
    case 256 * 16 + 2: return launch_quantize<T, 256, 2>(s, a, st);
    case 256 * 16 + 3: return launch_quantize<T, 256, 3>(s, a, st);
    case 256 * 16 + 4: return launch_quantize<T, 256, 4>(s, a, st);
    case 256 * 16 + 5: return launch_quantize<T, 256, 5>(s, a, st);
    case 1024 * 16 + 2: return launch_quantize<T, 1024, 2>(s, a, st);
    case 1024 * 16 + 3: return launch_quantize<T, 1024, 3>(s, a, st);
    case 1024 * 16 + 4: return launch_quantize<T, 1024, 4>(s, a, st);
    case 1024 * 16 + 5: return launch_quantize<T, 1024, 5>(s, a, st);
    }
    return false;
}

template <typename T, int V, int LANES, int NV, bool PAST> bool launch_dequantize(const HoldShape &s, const HoldArgs &a, hipStream_t st)
{
    hipLaunchKernelGGL((dequantize_rows_kernel<T, V, LANES, NV, PAST>), dim3(s.grid), dim3(256), 0, st, a);
    return true;
}

template <typename T, bool PAST> bool launch_dequantize_of(const HoldShape &s, const HoldArgs &a, hipStream_t st)
{
    constexpr int V = 16 / sizeof(T);
    if (s.pack == 1) return launch_dequantize<T, 1, 8, 1, false>(s, a, st);
    switch (s.lanes * 16 + s.packs) {
    case 0: hipLaunchKernelGGL((dequantize_long_rows_kernel<T, V, PAST>), dim3(s.grid), dim3(256), 0, st, a); return true;
    case 8 * 16 + 1: return launch_dequantize<T, V, 8, 1, PAST>(s, a, st);
    case 16 * 16 + 1: return launch_dequantize<T, V, 16, 1, PAST>(s, a, st);
    case 32 * 16 + 1: return launch_dequantize<T, V, 32, 1, PAST>(s, a, st);
    case 32 * 16 + 2: return launch_dequantize<T, V, 32, 2, PAST>(s, a, st);
    case 32 * 16 + 3: return launch_dequantize<T, V, 32, 3, PAST>(s, a, st);
    case 32 * 16 + 4: return launch_dequantize<T, V, 32, 4, PAST>(s, a, st);
    case 32 * 16 + 5: return launch_dequantize<T, V, 32, 5, PAST>(s, a, st);
    case 64 * 16 + 3: return launch_dequantize<T, V, 64, 3, PAST>(s, a, st);
    case 64 * 16 + 4: return launch_dequantize<T, V, 64, 4, PAST>(s, a, st);
    }
    return false;
}

template <typename T> bool launch_dequantize_as(bool past, const HoldShape &s, const HoldArgs &a, hipStream_t st)
{
    return past ? launch_dequantize_of<T, true>(s, a, st) : launch_dequantize_of<T, false>(s, a, st);
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
    // Results that fill more than half of the caches (256 MB) are read from memory by whoever takes them, and go there faster past them (199,000 x 602, us: fp32 164, past
    // them 142; bf16 picked by positions 90 and 84; 700 x 131,072 fp32 83 and 68).
    const bool past = n_out * n_cols * bytes > 128ull << 20;
    const HoldShape s = read_shape((int64_t)n_out, (int64_t)n_cols, (int)bytes, n_cu);
    const hipStream_t st = as_stream(stream);
    const bool found = type == RG_F32 ? launch_dequantize_as<float>(past, s, a, st) : type == RG_BF16 ? launch_dequantize_as<bf16>(past, s, a, st) : launch_dequantize_as<f16>(past, s, a, st);
    if (!found) { set_error("no kernel for rows of %llu elements", (unsigned long long)n_cols); return RG_EHIP; }
    RG_HIP(hipGetLastError());
    return RG_OK;
}
