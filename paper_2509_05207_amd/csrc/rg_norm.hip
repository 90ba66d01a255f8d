// Layer norm of rows and its gradients: the norm a trainer runs on the gathered blocks (Sec. 4 par. (8)).
//
// Both directions are bound by HBM: a row is read once into registers, its sums are taken there, and the result is written once.  The mean comes first, then
// the squares around it and the sum of what it leaves, by which it is corrected: y of rows far from zero has the digits of their deviations, and of a constant row is
// nothing.  (The gradients take the mean as it was given out, rounded to fp32.)  A row belongs to 8 to 64 lanes of a wave, or to
// a workgroup, whatever holds it in 32 elements a lane or fewer; rows beyond that are read twice.  The last pack of a row is the one that
// ENDS at the row's end: it overlaps its predecessor, both write the same values there, and the elements that it repeats count in
// no sum.
//
// The gradients of weight and bias are sums over all rows.  A workgroup takes rows from the whole range by turns and keeps the sums of
// its columns in registers; their partial sums go to the workspace, one row a workgroup, and a second launch adds them up in a fixed
// order (no atomics: the same bits every time).
#include "rg_internal.h"
#include "rg_elements.h"
#include "rg_launch.h"

#include <cmath>

namespace rg {

namespace {

struct NormArgs {
    const uint8_t *x;
    uint64_t x_stride;
    const uint8_t *dy;
    uint64_t dy_stride;
    uint8_t *out;                    // y, or dx (NULL: not wanted)
    uint64_t out_stride;
    const void *weight, *bias;       // or NULL
    uint32_t weight_type;
    float eps, cols, inv_cols;         // inv_cols: 1 / cols
    float *mean, *rstd;              // written by the forward pass (or NULL), read by the backward pass
    float *partial;                  // [2][n_partial][n_cols], or NULL: neither dweight nor dbias is wanted
    uint32_t n_partial;
    uint32_t parts;                  // workgroups to a row of those that do not fit registers
    int64_t n_rows, n_cols;
};

// Elements [c, c + V) of a vector of one of the three types.
template <int V>
__device__ __forceinline__ void load_weights(const void *p, uint32_t type, int64_t c, float (&v)[V])
{
    if (type == RG_F32) load_pack(static_cast<const float *>(p) + c, v);
    else if (type == RG_BF16) load_pack(static_cast<const bf16 *>(p) + c, v);
    else load_pack(static_cast<const f16 *>(p) + c, v);
}

// A product that is rounded before it goes into a sum or a difference.  In dx what is rounded cancels: of a row of one column nothing is left, of one of two a part of
// eps / variance, and a product that were fused with the difference behind it would leave its own rounding there instead.
__device__ __forceinline__ float rounded(float a, float b)
{
#pragma clang fp contract(off)
    return a * b;
}

// 1 / sqrt(v), rounded once: the device's approximation r, corrected by what v r^2 is off from one (r^2 in two parts).  Where that leaves the range, r as it is.
__device__ __forceinline__ float inverse_root(float v)
{
    const float r = rsqrtf(v), p = rounded(r, r), off = fmaf(-v, fmaf(r, r, -p), fmaf(-v, p, 1.f));
    return fabsf(off) < 0.5f ? fmaf(0.5f * r, off, r) : r;
}

// Squares around the mean out of those around a point near it: sum is what is left over of that point, rest its share to an element.  (Not below zero, and a NaN stays.)
__device__ __forceinline__ float squares_around(float squares, float sum, float rest)
{
    const float m2 = fmaf(-sum, rest, squares);
    return m2 < 0.f ? 0.f : m2;
}

// Sums over all lanes of a row.  Beyond a wave they meet in LDS, in slots taken by turns: whoever writes a slot again has passed a barrier
// that every wave reaches only after it has read that slot.
template <int LANES, int N>
__device__ __forceinline__ void row_sums(float (&v)[N], float (*slots)[2][16], uint32_t &turn)
{
    static_assert(N <= 2, "");
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = lanes_sum<(LANES < 64 ? LANES : 64)>(v[k]);
    if constexpr (LANES > 64) {
        float(*s)[16] = slots[turn & 1];
        ++turn;
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int k = 0; k < N; ++k) s[k][threadIdx.x >> 6] = v[k];
        __syncthreads();
#pragma unroll
        for (int k = 0; k < N; ++k) {
            float t = 0.f;
#pragma unroll
            for (int w = 0; w < LANES / 64; ++w) t += s[k][w];
            v[k] = t;
        }
    }
}

// Where the packs of a lane lie.  Only the last of a row's NV packs a lane can leave the row (the shape has as many as the row needs).
template <int V, int LANES, int NV>
struct RowLane {
    int32_t last;            // first column of the last pack
    int32_t skip;            // its leading elements that belong to other packs; V: all of them
    int32_t lane;
    __device__ __forceinline__ RowLane(int32_t n_cols)
    {
        lane = (int32_t)(threadIdx.x % LANES);
        const int32_t c = ((NV - 1) * LANES + lane) * V;
        last = min(c, n_cols - V);
        skip = min(c - last, V);
    }
    __device__ __forceinline__ int32_t column(int j) const { return j == NV - 1 ? last : (j * LANES + lane) * V; }
    __device__ __forceinline__ bool counts(int j, int e) const { return j != NV - 1 || e >= skip; }
    __device__ __forceinline__ bool stores(int j) const { return j != NV - 1 || skip < V; }
};

constexpr int norm_threads(int lanes) { return lanes > 256 ? lanes : 256; }

// y, and the rows' statistics.  (us: 199,000 x 602 fp32 181, 5.3 TB/s; 150,000 x 256 bf16 29, 5.2 TB/s; 8,192 x 8,192 bf16 52, 5.2 TB/s; 256 x 64 fp32 3.0,
// a launch's latency.)
template <typename T, int V, int LANES, int NV>
__global__ void __launch_bounds__(norm_threads(LANES)) norm_rows_kernel(NormArgs a)
{
    __shared__ float slots[2][2][16];
    uint32_t turn = 0;
    const RowLane<V, LANES, NV> at((int32_t)a.n_cols);
    float w[NV][V], b[NV][V];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
#pragma unroll
        for (int e = 0; e < V; ++e) { w[j][e] = 1.f; b[j][e] = 0.f; }
        if (a.weight) load_weights<V>(a.weight, a.weight_type, at.column(j), w[j]);
        if (a.bias) load_weights<V>(a.bias, a.weight_type, at.column(j), b[j]);
    }
    constexpr int GROUPS = norm_threads(LANES) / LANES;
    for (int64_t row = (int64_t)blockIdx.x * GROUPS + threadIdx.x / LANES; row < a.n_rows; row += (int64_t)gridDim.x * GROUPS) {
        const T *x = reinterpret_cast<const T *>(a.x + (uint64_t)row * a.x_stride);
        T *y = reinterpret_cast<T *>(a.out + (uint64_t)row * a.out_stride);
        float v[NV][V], s[1] = {0.f};
#pragma unroll
        for (int j = 0; j < NV; ++j) load_pack(x + at.column(j), v[j]);
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int e = 0; e < V; ++e) s[0] += at.counts(j, e) ? v[j][e] : 0.f;
        row_sums<LANES>(s, slots, turn);
        // What the mean leaves of a constant row are a few units of its last place, whose sums are exact, and so are the quotient (of a division, not of a rounded inverse) and the difference.
        const float about = s[0] / a.cols;
        float t[2] = {0.f, 0.f};
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                v[j][e] -= about;
                t[0] += at.counts(j, e) ? v[j][e] : 0.f;
                t[1] += at.counts(j, e) ? rounded(v[j][e], v[j][e]) : 0.f;
            }
        row_sums<LANES>(t, slots, turn);
        // Up to the differences' own roundings what is left is nothing but these.
        const float left = t[0] / a.cols, rest = fabsf(left) <= 0x1p-23f * sqrtf(t[1] * a.inv_cols) ? 0.f : left;
        const float mean = about + rest, rstd = inverse_root(squares_around(t[1], t[0], rest) * a.inv_cols + a.eps);
#pragma unroll
        for (int j = 0; j < NV; ++j) {
#pragma unroll
            for (int e = 0; e < V; ++e) v[j][e] = (v[j][e] - rest) * rstd * w[j][e] + b[j][e];
            if (at.stores(j)) store_pack(y + at.column(j), v[j]);
        }
        if (at.lane == 0) {
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
    }
}

// dx and the workgroup's sums of dy xhat and dy, from x, dy and the rows' statistics.  A wave has the next row under way while it works on one: without that a row's
// way from memory and its sums follow one another.  (us: 199,000 x 602 fp32 without dx 199, 4.8 TB/s; 150,000 x 256 bf16 40, 5.8 TB/s; 8,192 x 8,192 bf16 86, 4.7 TB/s.)
template <typename T, int V, int LANES, int NV>
__global__ void __launch_bounds__(norm_threads(LANES), LANES > 256 ? 1 : V * NV > 8 ? 3 : 4) norm_grad_kernel(NormArgs a)
{
    __shared__ float slots[2][2][16];
    uint32_t turn = 0;
    const RowLane<V, LANES, NV> at((int32_t)a.n_cols);
    float w[NV][V], dw[NV][V], db[NV][V];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
#pragma unroll
        for (int e = 0; e < V; ++e) { w[j][e] = 1.f; dw[j][e] = 0.f; db[j][e] = 0.f; }
        if (a.weight) load_weights<V>(a.weight, a.weight_type, at.column(j), w[j]);
    }
    constexpr int GROUPS = norm_threads(LANES) / LANES;
    // The next row is under way while this one is worked on (behind the last row that one again), where there are registers for it.
    constexpr bool AHEAD_OF_ROW = LANES < 1024 || NV * V <= 8;
    typename PackOf<T, V>::type raw_x[NV], raw_dy[NV];
    float mean = 0.f, rstd = 0.f;
    const auto fetch = [&](int64_t row) {
        const T *x = reinterpret_cast<const T *>(a.x + (uint64_t)row * a.x_stride);
        const T *dy = reinterpret_cast<const T *>(a.dy + (uint64_t)row * a.dy_stride);
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            raw_x[j] = load_raw<T, V>(x + at.column(j));
            raw_dy[j] = load_raw<T, V>(dy + at.column(j));
        }
        mean = a.mean[row];
        rstd = a.rstd[row];
    };
    const int64_t step = (int64_t)gridDim.x * GROUPS;
    int64_t row = (int64_t)blockIdx.x * GROUPS + threadIdx.x / LANES;
    if (AHEAD_OF_ROW && row < a.n_rows) fetch(row);
    for (; row < a.n_rows; row += step) {
        if (!AHEAD_OF_ROW) fetch(row);
        float h[NV][V], g[NV][V];
        const float this_mean = mean, this_rstd = rstd;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            unpack<T, V>(raw_x[j], h[j]);
            unpack<T, V>(raw_dy[j], g[j]);
        }
        if (AHEAD_OF_ROW) fetch(row + step < a.n_rows ? row + step : row);
        float s[2] = {0.f, 0.f};
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                h[j][e] = rounded(h[j][e] - this_mean, this_rstd);
                const float counted = at.counts(j, e) ? g[j][e] : 0.f;
                db[j][e] += counted;
                dw[j][e] += at.counts(j, e) ? g[j][e] * h[j][e] : 0.f;
                g[j][e] = rounded(g[j][e], w[j][e]);               // q from here on
                s[0] += at.counts(j, e) ? g[j][e] : 0.f;
                s[1] += at.counts(j, e) ? rounded(g[j][e], h[j][e]) : 0.f;
            }
        if (!a.out) continue;
        row_sums<LANES>(s, slots, turn);
        const float m0 = rounded(s[0], a.inv_cols), m1 = rounded(s[1], a.inv_cols);
        T *dx = reinterpret_cast<T *>(a.out + (uint64_t)row * a.out_stride);
#pragma unroll
        for (int j = 0; j < NV; ++j) {
#pragma unroll
            for (int e = 0; e < V; ++e) g[j][e] = this_rstd * (g[j][e] - m0 - rounded(h[j][e], m1));
            if (at.stores(j)) store_pack(dx + at.column(j), g[j]);
        }
    }
    if (!a.partial) return;
    float *to_dw = a.partial + (uint64_t)blockIdx.x * (uint64_t)a.n_cols, *to_db = to_dw + (uint64_t)a.n_partial * (uint64_t)a.n_cols;
    // Rows of a wave's groups, then of the workgroup's waves.
    if constexpr (LANES < 64) {
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int e = 0; e < V; ++e)
#pragma unroll
                for (int m = LANES; m < 64; m <<= 1) {
                    dw[j][e] += __shfl_xor(dw[j][e], m);
                    db[j][e] += __shfl_xor(db[j][e], m);
                }
    }
    if constexpr (LANES <= 64) {
        __shared__ float waves[3][2][V][64];
        const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            if (wave > 0)
#pragma unroll
                for (int e = 0; e < V; ++e) { waves[wave - 1][0][e][lane] = dw[j][e]; waves[wave - 1][1][e][lane] = db[j][e]; }
            __syncthreads();
            if (wave == 0)
#pragma unroll
                for (int e = 0; e < V; ++e)
#pragma unroll
                    for (int k = 0; k < 3; ++k) { dw[j][e] += waves[k][0][e][lane]; db[j][e] += waves[k][1][e][lane]; }
            __syncthreads();
        }
        if (wave > 0 || lane >= LANES) return;
    }
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int e = 0; e < V; ++e)
            if (at.counts(j, e)) {
                to_dw[at.column(j) + e] = dw[j][e];
                to_db[at.column(j) + e] = db[j][e];
            }
}

// ---------------------------------------------------------------- rows that do not fit a workgroup's registers
constexpr int LONG_THREADS = 1024;
constexpr int AHEAD = 8;                 // packs that a thread has under way

// Count, mean (mean + low, what the first rounded away) and squares around it of two disjoint parts put together.  The counts come in before the difference is squared: of
// an empty q it is a whole mean, whose square may be beyond the range.
struct Moments { float n, mean, low, m2; };
__device__ __forceinline__ Moments join(const Moments &p, const Moments &q)
{
    if (p.n == 0.f) return q;
    const float n = p.n + q.n;
    const float part = q.n / n, d = (q.mean - p.mean) + (q.low - p.low);
    const float step = rounded(d, part), mean = p.mean + step, moved = mean - p.mean;
    return Moments{n, mean, p.low + ((p.mean - (mean - moved)) + (step - moved)), p.m2 + q.m2 + d * (d * (p.n * part))};
}

// Few rows are shared out among `parts` workgroups each: all of them take the row's sums (which they read from their L2: workgroup g runs on XCD g mod
// 8, and a row's workgroups are on one), and each writes its own part.  (61 rows of 131,071 fp32, us: a workgroup a row 26, four 21.)
struct Part {
    int64_t row, rows;                   // the first row, and how far the next one is
    int64_t from, to;                    // packs of the part
    bool last;
};
__device__ __forceinline__ Part part_of(uint32_t parts, int64_t packs)
{
    const uint32_t q = blockIdx.x / 8, k = q % parts;
    return Part{(int64_t)(q / parts) * 8 + blockIdx.x % 8, (int64_t)(gridDim.x / parts), packs * k / parts, packs * (k + 1) / parts, k + 1 == parts};
}

template <typename T>
__global__ void __launch_bounds__(LONG_THREADS) norm_long_rows_kernel(NormArgs a)
{
    constexpr int V = 16 / (int)sizeof(T);
    __shared__ Moments waves[2][LONG_THREADS / 64];
    uint32_t turn = 0;
    const int64_t packs = a.n_cols / V;
    const int64_t rest = packs * V + threadIdx.x;              // what no pack holds: an element a thread
    const Part part = part_of(a.parts, packs);
    for (int64_t row = part.row; row < a.n_rows; row += part.rows) {
        const T *x = reinterpret_cast<const T *>(a.x + (uint64_t)row * a.x_stride);
        T *y = reinterpret_cast<T *>(a.out + (uint64_t)row * a.out_stride);
        Moments m{0.f, 0.f, 0.f, 0.f};
        for (int64_t first = threadIdx.x; first < packs; first += LONG_THREADS * AHEAD) {
            typename PackOf<T, V>::type raw[AHEAD];
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) raw[k] = load_raw<T, V>(x + min(first + k * LONG_THREADS, packs - 1) * V);
            float v[AHEAD][V], s = 0.f, n = 0.f;
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                unpack<T, V>(raw[k], v[k]);
                const bool there = first + k * LONG_THREADS < packs;
                n += there ? (float)V : 0.f;
#pragma unroll
                for (int e = 0; e < V; ++e) s += there ? v[k][e] : 0.f;
            }
            Moments q{n, s / n, 0.f, 0.f};
            s = 0.f;
#pragma unroll
            for (int k = 0; k < AHEAD; ++k)
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float c = first + k * LONG_THREADS < packs ? v[k][e] - q.mean : 0.f;
                    s += c;
                    q.m2 += rounded(c, c);
                }
            q.low = s / n;
            q.m2 = squares_around(q.m2, s, q.low);
            m = join(m, q);
        }
        if (rest < a.n_cols) m = join(m, Moments{1.f, (float)x[rest], 0.f, 0.f});
#pragma unroll
        for (int k = 1; k < 64; k <<= 1) m = join(m, Moments{__shfl_xor(m.n, k), __shfl_xor(m.mean, k), __shfl_xor(m.low, k), __shfl_xor(m.m2, k)});
        Moments *s = waves[turn & 1];
        ++turn;
        if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = m;
        __syncthreads();
        m = s[0];
        for (int k = 1; k < LONG_THREADS / 64; ++k) m = join(m, s[k]);
        const float mean = m.mean, low = m.low, rstd = inverse_root(m.m2 * a.inv_cols + a.eps);
        for (int64_t first = part.from + threadIdx.x; first < part.to; first += LONG_THREADS * AHEAD) {
            typename PackOf<T, V>::type raw[AHEAD];
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) raw[k] = load_raw<T, V>(x + min(first + k * LONG_THREADS, packs - 1) * V);
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                const int64_t c = (first + k * LONG_THREADS) * V;
                if (c >= part.to * V) break;
                float v[V], w[V], b[V];
                unpack<T, V>(raw[k], v);
#pragma unroll
                for (int e = 0; e < V; ++e) { w[e] = 1.f; b[e] = 0.f; }
                if (a.weight) load_weights<V>(a.weight, a.weight_type, c, w);
                if (a.bias) load_weights<V>(a.bias, a.weight_type, c, b);
#pragma unroll
                for (int e = 0; e < V; ++e) v[e] = (v[e] - mean - low) * rstd * w[e] + b[e];
                store_pack(y + c, v);
            }
        }
        if (part.last && rest < a.n_cols) {
            float v[1], w[1] = {1.f}, b[1] = {0.f};
            load_pack(x + rest, v);
            if (a.weight) load_weights<1>(a.weight, a.weight_type, rest, w);
            if (a.bias) load_weights<1>(a.bias, a.weight_type, rest, b);
            v[0] = (v[0] - mean - low) * rstd * w[0] + b[0];
            store_pack(y + rest, v);
        }
        if (threadIdx.x == 0 && part.last) {
            if (a.mean) a.mean[row] = mean + low;
            if (a.rstd) a.rstd[row] = rstd;
        }
    }
}

// dx alone; the columns' sums are taken by the kernel below.  (512 rows of 65,536 bf16, us: 50; 201 MB, of which x and dy are read twice, from cache then.)
template <typename T>
__global__ void __launch_bounds__(LONG_THREADS) norm_long_dx_kernel(NormArgs a)
{
    constexpr int V = 16 / (int)sizeof(T);
    __shared__ float slots[2][2][16];
    uint32_t turn = 0;
    const int64_t packs = a.n_cols / V;
    const int64_t rest = packs * V + threadIdx.x;
    const Part part = part_of(a.parts, packs);
    for (int64_t row = part.row; row < a.n_rows; row += part.rows) {
        const T *x = reinterpret_cast<const T *>(a.x + (uint64_t)row * a.x_stride);
        const T *dy = reinterpret_cast<const T *>(a.dy + (uint64_t)row * a.dy_stride);
        T *dx = reinterpret_cast<T *>(a.out + (uint64_t)row * a.out_stride);
        const float mean = a.mean[row], rstd = a.rstd[row];
        float s[2] = {0.f, 0.f};
        const auto add = [&](auto c, auto &h, auto &g) {
            constexpr int N = sizeof(h) / sizeof(float);
            float w[N];
            load_pack(x + c, h);
            load_pack(dy + c, g);
#pragma unroll
            for (int e = 0; e < N; ++e) w[e] = 1.f;
            if (a.weight) load_weights<N>(a.weight, a.weight_type, c, w);
#pragma unroll
            for (int e = 0; e < N; ++e) { h[e] = (h[e] - mean) * rstd; g[e] *= w[e]; }
        };
#pragma unroll 4
        for (int64_t p = threadIdx.x; p < packs; p += LONG_THREADS) {
            float h[V], g[V];
            add(p * V, h, g);
#pragma unroll
            for (int e = 0; e < V; ++e) { s[0] += g[e]; s[1] += g[e] * h[e]; }
        }
        if (rest < a.n_cols) {
            float h[1], g[1];
            add(rest, h, g);
            s[0] += g[0];
            s[1] += g[0] * h[0];
        }
        row_sums<LONG_THREADS>(s, slots, turn);
        const float m0 = s[0] * a.inv_cols, m1 = s[1] * a.inv_cols;
        #pragma unroll 2
        for (int64_t p = part.from + threadIdx.x; p < part.to; p += LONG_THREADS) {
            float h[V], g[V];
            add(p * V, h, g);
#pragma unroll
            for (int e = 0; e < V; ++e) g[e] = rstd * (g[e] - m0 - h[e] * m1);
            store_pack(dx + p * V, g);
        }
        if (part.last && rest < a.n_cols) {
            float h[1], g[1];
            add(rest, h, g);
            g[0] = rstd * (g[0] - m0 - h[0] * m1);
            store_pack(dx + rest, g);
        }
    }
}

// Partial column sums of the rows blockIdx.y, blockIdx.y + gridDim.y, ...: a pack of columns a thread.  (512 x 65,536 bf16, us: 31, 4.3 TB/s.)
template <typename T>
__global__ void __launch_bounds__(256) norm_columns_kernel(NormArgs a)
{
    constexpr int V = 16 / (int)sizeof(T);
    const int64_t c = ((int64_t)blockIdx.x * 256 + threadIdx.x) * V;
    if (c >= a.n_cols) return;
    const int n = (int)min((int64_t)V, a.n_cols - c);
    float dw[V], db[V];
#pragma unroll
    for (int e = 0; e < V; ++e) { dw[e] = 0.f; db[e] = 0.f; }
    for (int64_t row = blockIdx.y; row < a.n_rows; row += gridDim.y) {
        const T *x = reinterpret_cast<const T *>(a.x + (uint64_t)row * a.x_stride) + c;
        const T *dy = reinterpret_cast<const T *>(a.dy + (uint64_t)row * a.dy_stride) + c;
        const float mean = a.mean[row], rstd = a.rstd[row];
        float h[V], g[V];
        if (n == V) {
            load_pack(x, h);
            load_pack(dy, g);
        } else {
#pragma unroll
            for (int e = 0; e < V; ++e) { h[e] = e < n ? (float)x[e] : 0.f; g[e] = e < n ? (float)dy[e] : 0.f; }
        }
#pragma unroll
        for (int e = 0; e < V; ++e) { dw[e] += g[e] * ((h[e] - mean) * rstd); db[e] += g[e]; }
    }
    float *to_dw = a.partial + (uint64_t)blockIdx.y * (uint64_t)a.n_cols + c, *to_db = to_dw + (uint64_t)a.n_partial * (uint64_t)a.n_cols;
#pragma unroll
    for (int e = 0; e < V; ++e)
        if (e < n) { to_dw[e] = dw[e]; to_db[e] = db[e]; }
}

// ---------------------------------------------------------------- the partial sums put together
// 32 columns a workgroup at a time, 32 threads to a column; blockIdx.y 0: dweight, 1: dbias.  (4 to 5 us for up to 8,192 columns, most of it a launch's latency; 13 for 65,536.)
__global__ void __launch_bounds__(NORM_SUM_THREADS) norm_partials_kernel(const float *__restrict__ partial, uint32_t n_partial, int64_t n_cols, void *dweight, void *dbias, uint32_t type)
{
    static_assert(NORM_SUM_COLUMNS == 32 && NORM_SUM_THREADS == 32 * 32, "");
    void *out = blockIdx.y == 0 ? dweight : dbias;
    if (!out) return;
    __shared__ float part[32][33];
    const float *src = partial + (uint64_t)blockIdx.y * n_partial * (uint64_t)n_cols;
    const uint32_t k = threadIdx.x >> 5;
    for (int64_t first = (int64_t)blockIdx.x * 32; first < n_cols; first += (int64_t)gridDim.x * 32) {
        const int64_t c = first + (threadIdx.x & 31);
        float s = 0.f;
        if (c < n_cols)
#pragma unroll 8
            for (uint32_t p = k; p < n_partial; p += 32) s += src[(uint64_t)p * (uint64_t)n_cols + c];
        part[k][threadIdx.x & 31] = s;
        __syncthreads();
        if (threadIdx.x < 32 && c < n_cols) {
            s = 0.f;
#pragma unroll
            for (int j = 0; j < 32; ++j) s += part[j][threadIdx.x];
            if (type == RG_F32) static_cast<float *>(out)[c] = s;
            else if (type == RG_BF16) static_cast<bf16 *>(out)[c] = (bf16)s;
            else static_cast<f16 *>(out)[c] = (f16)s;
        }
        __syncthreads();                                       // part is read, and may be written
    }
}

// ---------------------------------------------------------------- launches
enum class Pass { FORWARD, BACKWARD };

template <Pass PASS, typename T, int V, int LANES, int NV>
void launch_one(const NormShape &s, const NormArgs &a, hipStream_t st)
{
    if constexpr (PASS == Pass::FORWARD) hipLaunchKernelGGL((norm_rows_kernel<T, V, LANES, NV>), dim3(s.grid), dim3(norm_threads(LANES)), 0, st, a);
    else hipLaunchKernelGGL((norm_grad_kernel<T, V, LANES, NV>), dim3(s.grid), dim3(norm_threads(LANES)), 0, st, a);
}

template <Pass PASS, typename T>
bool launch_rows(const NormShape &s, const NormArgs &a, hipStream_t st)
{
    constexpr int V = 16 / (int)sizeof(T);
    const auto is = [&](int v, int lanes, int packs) { return s.pack == v && s.lanes == lanes && s.packs == packs; };
#define RG_NORM_SHAPE(v, lanes, packs)                                                                                    \
    if constexpr ((v) * (packs) <= norm_elements(PASS == Pass::BACKWARD))                                                 \
        if (is(v, lanes, packs)) { launch_one<PASS, T, v, lanes, packs>(s, a, st); return true; }
    RG_NORM_SHAPE(1, 8, 1)
    RG_NORM_SHAPE(V, 8, 1)
    RG_NORM_SHAPE(V, 16, 1)
    RG_NORM_SHAPE(V, 32, 1)
    RG_NORM_SHAPE(V, 64, 1)
    RG_NORM_SHAPE(V, 64, 2)
    RG_NORM_SHAPE(V, 64, 3)
    RG_NORM_SHAPE(V, 64, 4)
    RG_NORM_SHAPE(V, 256, 1)
    RG_NORM_SHAPE(V, 256, 2)
    RG_NORM_SHAPE(V, 256, 3)
    RG_NORM_SHAPE(V, 256, 4)
    RG_NORM_SHAPE(V, 1024, 1)
    RG_NORM_SHAPE(V, 1024, 2)
    RG_NORM_SHAPE(V, 1024, 3)
    RG_NORM_SHAPE(V, 1024, 4)
#undef RG_NORM_SHAPE
    return false;
}

template <Pass PASS>
bool launch_rows_of(uint32_t type, const NormShape &s, const NormArgs &a, hipStream_t st)
{
    return type == RG_F32 ? launch_rows<PASS, float>(s, a, st) : type == RG_BF16 ? launch_rows<PASS, bf16>(s, a, st) : launch_rows<PASS, f16>(s, a, st);
}

#define RG_BY_TYPE(kernel, grid, threads, st, a)                                                                   \
    do {                                                                                                           \
        if (type == RG_F32) hipLaunchKernelGGL(kernel<float>, grid, dim3(threads), 0, st, a);                      \
        else if (type == RG_BF16) hipLaunchKernelGGL(kernel<bf16>, grid, dim3(threads), 0, st, a);                 \
        else hipLaunchKernelGGL(kernel<f16>, grid, dim3(threads), 0, st, a);                                       \
    } while (0)

rg_status check_sizes(uint64_t n_rows, uint64_t n_cols, uint32_t type)
{
    if (!element_bytes(type)) { set_error("type %u is none of RG_F32, RG_BF16, RG_F16", type); return RG_EINVAL; }
    if (n_cols == 0) { set_error("rows of no elements have no mean"); return RG_EINVAL; }
    if (n_cols >= 1ull << 31 || n_rows >= 1ull << 40) { set_error("%llu rows of %llu elements are beyond the limits (2^40, 2^31)", (unsigned long long)n_rows, (unsigned long long)n_cols); return RG_ERANGE; }
    return RG_OK;
}

// A matrix of rows: address and stride in whole elements; an output's rows apart from each other.
rg_status check_rows(const char *what, const void *p, uint64_t stride, uint64_t n_rows, uint64_t n_cols, uint32_t bytes, bool output)
{
    if (n_rows == 0) return RG_OK;
    if (!p) { set_error("%s is null", what); return RG_EINVAL; }
    if ((reinterpret_cast<uintptr_t>(p) | stride) % bytes) { set_error("%s: address and stride have to be multiples of %u bytes", what, bytes); return RG_EINVAL; }
    if (output && n_rows > 1 && stride < n_cols * bytes) { set_error("%s: a stride of %llu bytes is less than a row", what, (unsigned long long)stride); return RG_EINVAL; }
    if (stride > 1ull << 40) { set_error("%s: a stride of %llu bytes is beyond the limit (2^40)", what, (unsigned long long)stride); return RG_ERANGE; }
    return RG_OK;
}

// A result in the place of an input has its rows where the input has them.
rg_status check_place(const char *what, const void *out, uint64_t out_stride, const void *in, uint64_t in_stride, uint64_t n_rows)
{
    if (out != in || out_stride == in_stride || n_rows <= 1) return RG_OK;
    set_error("%s: in place, but with another stride", what);
    return RG_EINVAL;
}

rg_status check_vector(const char *what, const void *p, uint32_t weight_type, uint32_t type)
{
    if (!p) return RG_OK;
    if (weight_type != RG_F32 && weight_type != type) { set_error("%s: weight_type %u is neither RG_F32 nor the rows' type", what, weight_type); return RG_EINVAL; }
    if (reinterpret_cast<uintptr_t>(p) % element_bytes(weight_type)) { set_error("%s is not aligned for its type", what); return RG_EINVAL; }
    return RG_OK;
}

}  // namespace
}  // namespace rg

using namespace rg;

extern "C" rg_status rg_layer_norm(const void *x, uint64_t x_stride, uint64_t n_rows, uint64_t n_cols, uint32_t type, const void *weight, const void *bias,
                                   uint32_t weight_type, float eps, void *y, uint64_t y_stride, float *mean, float *rstd, void *stream)
{
    RG_TRY(check_sizes(n_rows, n_cols, type));
    const uint32_t bytes = element_bytes(type);
    RG_TRY(check_rows("x", x, x_stride, n_rows, n_cols, bytes, false));
    RG_TRY(check_rows("y", y, y_stride, n_rows, n_cols, bytes, true));
    RG_TRY(check_place("y", y, y_stride, x, x_stride, n_rows));
    RG_TRY(check_vector("weight", weight, weight_type, type));
    RG_TRY(check_vector("bias", bias, weight_type, type));
    RG_TRY(check_vector("mean", mean, RG_F32, type));
    RG_TRY(check_vector("rstd", rstd, RG_F32, type));
    if (!(eps >= 0.f) || std::isinf(eps)) { set_error("eps has to be a number >= 0"); return RG_EINVAL; }
    if (n_rows == 0) return RG_OK;
    int n_cu = 0;
    RG_TRY(compute_units(&n_cu));
    NormArgs a{};
    a.x = static_cast<const uint8_t *>(x); a.x_stride = x_stride;
    a.out = static_cast<uint8_t *>(y); a.out_stride = y_stride;
    a.weight = weight; a.bias = bias; a.weight_type = weight_type;
    a.eps = eps; a.cols = (float)n_cols; a.inv_cols = (float)(1.0 / (double)n_cols);
    a.mean = mean; a.rstd = rstd;
    a.n_rows = (int64_t)n_rows; a.n_cols = (int64_t)n_cols;
    const hipStream_t st = as_stream(stream);
    const NormShape s = norm_shape((int64_t)n_rows, (int64_t)n_cols, (int)bytes, n_cu, false, y == x);
    a.parts = s.parts;
    if (s.lanes == 0) RG_BY_TYPE(norm_long_rows_kernel, dim3(s.grid), LONG_THREADS, st, a);
    else if (!launch_rows_of<Pass::FORWARD>(type, s, a, st)) { set_error("no kernel for rows of %llu elements", (unsigned long long)n_cols); return RG_EHIP; }
    RG_HIP(hipGetLastError());
    return RG_OK;
}

extern "C" rg_status rg_layer_norm_workspace(uint64_t n_rows, uint64_t n_cols, uint32_t type, uint64_t *bytes)
{
    if (!bytes) { set_error("null argument"); return RG_EINVAL; }
    RG_TRY(check_sizes(n_rows, n_cols, type));
    int n_cu = 0;
    RG_TRY(compute_units(&n_cu));
    const NormShape s = norm_shape((int64_t)n_rows, (int64_t)n_cols, (int)element_bytes(type), n_cu, true, false);
    *bytes = 2ull * s.n_partial * n_cols * sizeof(float);
    return RG_OK;
}

extern "C" rg_status rg_layer_norm_backward(const void *dy, uint64_t dy_stride, const void *x, uint64_t x_stride, uint64_t n_rows, uint64_t n_cols, uint32_t type,
                                            const void *weight, uint32_t weight_type, const float *mean, const float *rstd, void *dx, uint64_t dx_stride,
                                            void *dweight, void *dbias, void *workspace, uint64_t workspace_bytes, void *stream)
{
    RG_TRY(check_sizes(n_rows, n_cols, type));
    const uint32_t bytes = element_bytes(type);
    RG_TRY(check_rows("dy", dy, dy_stride, n_rows, n_cols, bytes, false));
    RG_TRY(check_rows("x", x, x_stride, n_rows, n_cols, bytes, false));
    if (dx) {
        RG_TRY(check_rows("dx", dx, dx_stride, n_rows, n_cols, bytes, true));
        RG_TRY(check_place("dx", dx, dx_stride, dy, dy_stride, n_rows));
        RG_TRY(check_place("dx", dx, dx_stride, x, x_stride, n_rows));
    }
    RG_TRY(check_vector("weight", weight, weight_type, type));
    RG_TRY(check_vector("dweight", dweight, weight_type, type));
    RG_TRY(check_vector("dbias", dbias, weight_type, type));
    RG_TRY(check_rows("mean", mean, 0, n_rows, 1, 4, false));
    RG_TRY(check_rows("rstd", rstd, 0, n_rows, 1, 4, false));
    int n_cu = 0;
    RG_TRY(compute_units(&n_cu));
    const NormShape s = norm_shape((int64_t)n_rows, (int64_t)n_cols, (int)bytes, n_cu, true, dx == dy || dx == x);
    const bool columns = dweight || dbias;
    if (columns && s.n_partial) {
        const uint64_t want = 2ull * s.n_partial * n_cols * sizeof(float);
        if (!workspace || reinterpret_cast<uintptr_t>(workspace) % 16) { set_error("the workspace is null or not aligned to 16 bytes"); return RG_EINVAL; }
        if (workspace_bytes < want) { set_error("the workspace holds %llu bytes of %llu", (unsigned long long)workspace_bytes, (unsigned long long)want); return RG_ERANGE; }
    }
    NormArgs a{};
    a.x = static_cast<const uint8_t *>(x); a.x_stride = x_stride;
    a.dy = static_cast<const uint8_t *>(dy); a.dy_stride = dy_stride;
    a.out = static_cast<uint8_t *>(dx); a.out_stride = dx_stride;
    a.weight = weight; a.weight_type = weight_type;
    a.cols = (float)n_cols; a.inv_cols = (float)(1.0 / (double)n_cols);
    a.mean = const_cast<float *>(mean); a.rstd = const_cast<float *>(rstd);
    a.partial = columns ? static_cast<float *>(workspace) : nullptr;
    a.n_partial = s.n_partial;
    a.parts = s.parts;
    a.n_rows = (int64_t)n_rows; a.n_cols = (int64_t)n_cols;
    const hipStream_t st = as_stream(stream);
    if (n_rows && (dx || columns)) {
        if (s.lanes == 0) {
            if (columns) {                                     // first: dx may take dy's place
                RG_BY_TYPE(norm_columns_kernel, dim3(s.column_grid, s.n_partial), 256, st, a);
                RG_HIP(hipGetLastError());
            }
            if (dx) RG_BY_TYPE(norm_long_dx_kernel, dim3(s.grid), LONG_THREADS, st, a);
        } else if (!launch_rows_of<Pass::BACKWARD>(type, s, a, st)) { set_error("no kernel for rows of %llu elements", (unsigned long long)n_cols); return RG_EHIP; }
        RG_HIP(hipGetLastError());
    }
    if (columns) {
        hipLaunchKernelGGL(norm_partials_kernel, dim3(s.sum_grid, 2), dim3(NORM_SUM_THREADS), 0, st, static_cast<const float *>(workspace), s.n_partial, (int64_t)n_cols, dweight, dbias,
                           weight_type);
        RG_HIP(hipGetLastError());
    }
    return RG_OK;
}
