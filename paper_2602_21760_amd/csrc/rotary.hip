// Rotary positions with several axes on queries and keys: pair (x, y) of a token's head -> (x cos a - y sin a, x sin a + y cos a).
//
// Bound by memory: every value of q and k is read and written once (65537 tokens, 24 / 8 heads of 128, 1.07 GB: 5.4 TB/s; 4429 tokens, 24 / 24 of 64, 54 MB: 5.5).  With one or two heads the fp64 angles count as much
// (half a million tokens, one head of 128: 3.8 TB/s).  The angles of a token are the same for all of its heads, so a
// workgroup forms the sines and cosines of its tokens once, in LDS, and turns all heads with them.  Angles are kept in turns and in fp64
// (position x frequency, minus the nearest whole number of quarter turns): a position of 10^6 keeps 10 digits behind the point where fp32
// would keep none; the rest, at most an eighth of a turn, goes to fp32 Taylor polynomials.
#include "common.h"

#include <math.h>

namespace {

constexpr int kThreads = 256;
constexpr int kMaxPairs = 128;          // head_dim <= 256
constexpr int kUnroll = 4;              // units of a thread whose loads are in flight together

struct RotaryArgs {
    const int* positions;
    const void *q, *k;
    void *q_out, *k_out;
    unsigned q_stride, k_stride, q_out_stride, k_out_stride;   // elements
    int tokens, axes;
    int head_dim, half;                 // half: pairs that turn
    int q_units, units;                 // units per token: of q, of q and k
    int tile;                           // tokens per workgroup
    int head_units;                     // units per head
    unsigned unit_magic, head_magic;    // magic_of() units and head_units
    float q_scale;
    unsigned char axis[kMaxPairs];
    double turns[kMaxPairs];            // turns per position of each pair
};

// i / d for i < 2^16 and d <= 2^16, magic = floor(2^32 / d) + 1 (0 stands for d = 1): the product is off by less than 1 / d.
unsigned magic_of(unsigned d) { return d == 1 ? 0u : (unsigned)((1ull << 32) / d) + 1; }
__device__ __forceinline__ int quotient(int i, unsigned magic) { return magic == 0 ? i : (int)__umulhi((unsigned)i, magic); }

template <typename T> struct Vec;
template <> struct Vec<bf16_t> { typedef bf16x8 type; static constexpr int n = 8; };
template <> struct Vec<float> { typedef f32x4 type; static constexpr int n = 4; };

// cos and sin of 2 pi t.  t minus its nearest quarter leaves |x| <= pi / 4, where the Taylor polynomials' remainders are below 2e-9 (sine: x^11 / 11!) and 2e-10
// (cosine: x^12 / 12!), far inside fp32.
__device__ __forceinline__ f32x2 cos_sin_turns(double t) {
    const double quarters = t * 4.0, whole = rint(quarters);
    const float x = (float)(quarters - whole) * 1.5707963267948966f;
    const int n = (int)(whole - 4.0 * floor(whole * 0.25));
    const float z = x * x;
    const float s = fmaf(x * z, fmaf(z, fmaf(z, fmaf(z, 2.7557319224e-6f, -1.9841269841e-4f), 8.3333333333e-3f), -1.6666666667e-1f), x);
    const float c = fmaf(z, fmaf(z, fmaf(z, fmaf(z, fmaf(z, -2.7557319224e-7f, 2.4801587302e-5f), -1.3888888889e-3f), 4.1666666667e-2f), -0.5f), 1.0f);
    const float a = n & 1 ? s : c, b = n & 1 ? c : s;
    return f32x2{n == 1 || n == 2 ? -a : a, n >= 2 ? -b : b};
}

// A kernel argument in a scalar register: a choice between two arguments is then one between values, not a load per lane from the chosen place.
template <typename P> __device__ __forceinline__ P pinned(P x) {
    asm("" : "+s"(x));
    return x;
}

// A unit is what a thread turns at a time: HALVES: two 16-byte vectors half the rotated width apart (behind it two that are only scaled);
// otherwise one vector of neighbouring pairs.  FULL: all features of a head turn; then the queries' table holds the scale as well.
template <typename T, bool HALVES, bool FULL>
__global__ __launch_bounds__(kThreads) void rotary_kernel(RotaryArgs a) {
    typedef typename Vec<T>::type vec;
    constexpr int N = Vec<T>::n, PAIRS = HALVES ? N : N / 2;
    extern __shared__ __attribute__((aligned(16))) f32x2 turn[];     // [tile][half] for k, and (FULL) the same times q_scale for q
    const long long first = (long long)(blockIdx.y * gridDim.x + blockIdx.x) * a.tile;
    if (first >= a.tokens) return;
    const int t0 = (int)first, tokens = min(a.tile, a.tokens - t0);
    const int total = tokens * a.units;
    const T* q_in = pinned(static_cast<const T*>(a.q) + (size_t)t0 * a.q_stride);
    const T* k_in = pinned(static_cast<const T*>(a.k) + (size_t)t0 * a.k_stride);
    T* q_to = pinned(static_cast<T*>(a.q_out) + (size_t)t0 * a.q_out_stride);
    T* k_to = pinned(static_cast<T*>(a.k_out) + (size_t)t0 * a.k_out_stride);
    const unsigned q_step = pinned(a.q_stride), k_step = pinned(a.k_stride), q_to_step = pinned(a.q_out_stride), k_to_step = pinned(a.k_out_stride);
    const int apart = a.half, apart_rest = a.head_dim / 2 - a.half;  // HALVES: elements between the two vectors of a unit that turns / does not
    const int q_table = FULL ? tokens * a.half : 0;
    T* out[kUnroll];
    vec x[kUnroll], y[kUnroll];
    int pair[kUnroll], table[kUnroll];      // first pair (-1: no unit; FULL aside, >= half: does not turn); its place in `turn`
    float scale[kUnroll];
    auto load = [&](int i0) {
#pragma unroll
        for (int j = 0; j < kUnroll; j++) {
            const int i = i0 + j * kThreads;
            if (i >= total) { pair[j] = -1; continue; }
            const int tok = quotient(i, a.unit_magic);
            int u = i - tok * a.units;
            const bool is_q = u < a.q_units;
            u -= is_q ? 0 : a.q_units;
            const int head = quotient(u, a.head_magic), v = u - head * a.head_units;
            scale[j] = is_q ? a.q_scale : 1.f;
            pair[j] = v * PAIRS;
            int off = u * N;
            if constexpr (HALVES) off = head * a.head_dim + (FULL || pair[j] < a.half ? v * N : a.half + v * N);   // (behind the rotated width R = 2 half: R + (v N - half))
            const T* in = (is_q ? q_in : k_in) + (size_t)(unsigned)tok * (is_q ? q_step : k_step) + off;
            out[j] = (is_q ? q_to : k_to) + (size_t)(unsigned)tok * (is_q ? q_to_step : k_to_step) + off;
            table[j] = (is_q ? q_table : 0) + tok * a.half + pair[j];
            x[j] = *reinterpret_cast<const vec*>(in);
            if constexpr (HALVES) y[j] = *reinterpret_cast<const vec*>(in + (FULL || pair[j] < a.half ? apart : apart_rest));
        }
    };
    auto finish = [&]() {
#pragma unroll
        for (int j = 0; j < kUnroll; j++) {
            if (pair[j] < 0) continue;
            float p[PAIRS], q[PAIRS];
#pragma unroll
            for (int e = 0; e < PAIRS; e++) {
                p[e] = to_f32<T>(HALVES ? x[j][e] : x[j][2 * e]);
                q[e] = to_f32<T>(HALVES ? y[j][e] : x[j][2 * e + 1]);
            }
            if constexpr (!FULL) {
#pragma unroll
                for (int e = 0; e < PAIRS; e++) {
                    p[e] *= scale[j];
                    q[e] *= scale[j];
                }
            }
            if (FULL || pair[j] < a.half) {
                const f32x2* cs = turn + table[j];
#pragma unroll
                for (int e = 0; e < PAIRS; e++) {
                    if (!FULL && !HALVES && pair[j] + e >= a.half) continue;       // (a vector may hold the last pairs that turn and the first that do not)
                    const f32x2 c = cs[e];
                    const float u = p[e];
                    p[e] = fmaf(u, c[0], -q[e] * c[1]);
                    q[e] = fmaf(u, c[1], q[e] * c[0]);
                }
            }
            vec u, w;
#pragma unroll
            for (int e = 0; e < PAIRS; e++) {
                if constexpr (HALVES) {
                    u[e] = from_f32<T>(p[e]);
                    w[e] = from_f32<T>(q[e]);
                } else {
                    u[2 * e] = from_f32<T>(p[e]);
                    u[2 * e + 1] = from_f32<T>(q[e]);
                }
            }
            *reinterpret_cast<vec*>(out[j]) = u;
            if constexpr (HALVES) *reinterpret_cast<vec*>(out[j] + (FULL || pair[j] < a.half ? apart : apart_rest)) = w;
        }
    };
    load(threadIdx.x);                  // on their way while the angles are formed
    for (int i = threadIdx.x; i < tokens * a.half; i += kThreads) {
        const int tok = i / a.half, p = i - tok * a.half;
        const double pos = (double)a.positions[(size_t)(t0 + tok) * a.axes + a.axis[p]];
        const f32x2 c = cos_sin_turns(pos * a.turns[p]);
        turn[i] = c;
        if constexpr (FULL) turn[q_table + i] = f32x2{c[0] * a.q_scale, c[1] * a.q_scale};
    }
    __syncthreads();
    finish();
    for (int i0 = threadIdx.x + kThreads * kUnroll; i0 < total; i0 += kThreads * kUnroll) {
        load(i0);
        finish();
    }
}

template <typename T>
int launch(RotaryArgs& a, bool halves, int q_heads, int k_heads, hipStream_t st) {
    constexpr int N = Vec<T>::n;
    a.head_units = a.head_dim / (halves ? 2 * N : N);
    a.q_units = q_heads * a.head_units;
    a.units = (q_heads + k_heads) * a.head_units;
    // Tokens per workgroup: of those that make two to four units per thread the number that leaves the fewest threads without one in the last round, the smaller for
    // the same (32 / 8 heads of 128, 65537 tokens: 512 units 200 us, 1024 203, 2048 206; 256 units 399: workgroups are then not started fast enough.  24 / 24
    // heads of 64 have 384 units a token: 4429 tokens two at a time 10.9 us, one 11.7; 12 / 12 in fp32 as many: 2102 tokens 6.0 and 6.3); and few tokens spread over the chip (16 tokens of 32 / 8
    // heads of 128: one a workgroup 3.2 us, two 3.8, three 4.3).  (Launches one after the other in a graph.)
    a.tile = 1;
    int best = 0;
    for (int t = 1; t <= 16 && (t == 1 || (t * a.units <= 4 * kThreads && t * 400 <= a.tokens)); t++) {      // (16 x 128 pairs, twice: 32 KB of LDS)
        const int n = t * a.units, share = 100 * n / ((n + kThreads - 1) / kThreads * kThreads);
        if (share > best + 3 || (n > kThreads && (t - 1) * a.units <= kThreads)) {
            a.tile = t;
            best = share;
        }
    }
    a.unit_magic = magic_of((unsigned)a.units);
    a.head_magic = magic_of((unsigned)a.head_units);
    const bool full = 2 * a.half == a.head_dim;
    // (a grid dimension holds less than 2^32 threads: what goes beyond 2^23 workgroups goes into the second one)
    const unsigned groups = (unsigned)(((size_t)a.tokens + a.tile - 1) / a.tile), x = groups < 1u << 23 ? groups : 1u << 23;
    const dim3 grid(x, (groups + x - 1) / x);
    const size_t lds = (size_t)a.tile * a.half * sizeof(f32x2) * (full ? 2 : 1);
    HybTraceScope trace("rotary", "byte", 2.0 * a.tokens * (q_heads + k_heads) * (double)a.head_dim * sizeof(T), st);
    if (halves && full) hipLaunchKernelGGL((rotary_kernel<T, true, true>), grid, dim3(kThreads), lds, st, a);
    else if (halves) hipLaunchKernelGGL((rotary_kernel<T, true, false>), grid, dim3(kThreads), lds, st, a);
    else if (full) hipLaunchKernelGGL((rotary_kernel<T, false, true>), grid, dim3(kThreads), lds, st, a);
    else hipLaunchKernelGGL((rotary_kernel<T, false, false>), grid, dim3(kThreads), lds, st, a);
    return hyb_check_launch("rotary");
}

}  // namespace

extern "C" int hyb_rotary(const hyb_rotary_desc* desc, const int* positions, const void* q, void* q_out, const void* k, void* k_out, void* stream) {
    HYB_REQUIRE(desc != nullptr, HYB_ERR_NULL, "hyb_rotary: argument 'desc' is NULL");
    const hyb_rotary_desc& d = *desc;
    HYB_CHECK_DTYPE(d.dtype);
    HYB_REQUIRE(d.pairs == HYB_ROTARY_NEIGHBOURS || d.pairs == HYB_ROTARY_HALVES, HYB_ERR_DTYPE, "hyb_rotary: unknown pairs %d", (int)d.pairs);
    HYB_REQUIRE(d.tokens >= 0 && d.q_heads >= 0 && d.k_heads >= 0, HYB_ERR_SHAPE, "hyb_rotary: negative size");
    HYB_REQUIRE(d.q_heads <= 512 && d.k_heads <= 512, HYB_ERR_SHAPE, "hyb_rotary: at most 512 heads each");
    HYB_REQUIRE(d.head_dim > 0 && d.head_dim <= 256 && d.head_dim % 16 == 0, HYB_ERR_SHAPE, "hyb_rotary: head_dim %d is not a multiple of 16 up to 256", d.head_dim);
    HYB_REQUIRE(d.axes >= 1 && d.axes <= HYB_ROTARY_MAX_AXES, HYB_ERR_SHAPE, "hyb_rotary: %d axes (1 to %d are possible)", d.axes, HYB_ROTARY_MAX_AXES);
    int width = 0;
    for (int i = 0; i < d.axes; i++) {
        HYB_REQUIRE(d.axis_dims[i] > 0 && d.axis_dims[i] % 2 == 0 && d.axis_dims[i] <= 256, HYB_ERR_SHAPE, "hyb_rotary: axis_dims[%d] = %d is not even and positive", i, d.axis_dims[i]);
        HYB_REQUIRE(isfinite(d.axis_scale[i]), HYB_ERR_SHAPE, "hyb_rotary: axis_scale[%d] is not finite", i);
        width += d.axis_dims[i];
    }
    HYB_REQUIRE(width <= d.head_dim, HYB_ERR_SHAPE, "hyb_rotary: axis_dims add up to %d features of %d", width, d.head_dim);
    HYB_REQUIRE(d.pairs != HYB_ROTARY_HALVES || width % 16 == 0, HYB_ERR_SHAPE, "hyb_rotary: halves need axis_dims that add up to a multiple of 16, not %d", width);
    HYB_REQUIRE(d.theta > 0.f && isfinite(d.theta), HYB_ERR_SHAPE, "hyb_rotary: theta must be positive");
    HYB_REQUIRE(isfinite(d.q_scale), HYB_ERR_SHAPE, "hyb_rotary: q_scale is not finite");
    if (d.tokens == 0 || d.q_heads + d.k_heads == 0) return HYB_OK;
    HYB_CHECK_PTR(positions); HYB_CHECK_ALIGN(positions);
    const size_t vec = 16 / hyb_dtype_size(d.dtype);
    const struct { int heads; const void* in; const void* out; size_t in_stride, out_stride; const char* name; } side[2] = {
        {d.q_heads, q, q_out, d.q_stride, d.q_out_stride, "q"}, {d.k_heads, k, k_out, d.k_stride, d.k_out_stride, "k"}};
    for (const auto& s : side) {
        if (s.heads == 0) continue;
        HYB_REQUIRE(s.in != nullptr && s.out != nullptr, HYB_ERR_NULL, "hyb_rotary: argument '%s' or '%s_out' is NULL", s.name, s.name);
        HYB_REQUIRE((((uintptr_t)s.in | (uintptr_t)s.out) & 15u) == 0, HYB_ERR_ALIGN, "hyb_rotary: argument '%s' or '%s_out' is not 16-byte aligned", s.name, s.name);
        const size_t row = (size_t)s.heads * d.head_dim;
        HYB_REQUIRE(s.in_stride >= row && s.out_stride >= row, HYB_ERR_SHAPE, "hyb_rotary: strides of %s are smaller than its %zu elements per token", s.name, row);
        HYB_REQUIRE(s.in_stride % vec == 0 && s.out_stride % vec == 0, HYB_ERR_ALIGN, "hyb_rotary: strides of %s are not multiples of 16 bytes", s.name);
        HYB_REQUIRE(s.in_stride < ((size_t)1 << 31) && s.out_stride < ((size_t)1 << 31), HYB_ERR_SHAPE, "hyb_rotary: strides of %s are not below 2^31", s.name);
        HYB_REQUIRE(s.in != s.out || s.in_stride == s.out_stride, HYB_ERR_SHAPE, "hyb_rotary: %s_out is %s with another stride", s.name, s.name);
    }
    RotaryArgs a = {};
    a.positions = positions;
    a.q = q; a.k = k; a.q_out = q_out; a.k_out = k_out;
    a.q_stride = (unsigned)d.q_stride; a.k_stride = (unsigned)d.k_stride; a.q_out_stride = (unsigned)d.q_out_stride; a.k_out_stride = (unsigned)d.k_out_stride;
    a.tokens = d.tokens; a.axes = d.axes; a.head_dim = d.head_dim; a.half = width / 2;
    a.q_scale = d.q_scale == 0.f ? 1.f : d.q_scale;
    // turns per position, theta^(-2 j / n) / (2 pi), by repeated multiplication in fp64: j roundings of 2^-53
    int p = 0;
    for (int i = 0; i < d.axes; i++) {
        const double step = pow((double)d.theta, -2.0 / d.axis_dims[i]);
        double f = (d.axis_scale[i] == 0.f ? 1.0 : (double)d.axis_scale[i]) / (d.inverse ? -6.283185307179586476925 : 6.283185307179586476925);
        for (int j = 0; j < d.axis_dims[i] / 2; j++, p++, f *= step) {
            a.axis[p] = (unsigned char)i;
            a.turns[p] = f;
        }
    }
    const bool halves = d.pairs == HYB_ROTARY_HALVES;
    return d.dtype == HYB_BF16 ? launch<bf16_t>(a, halves, d.q_heads, d.k_heads, (hipStream_t)stream) : launch<float>(a, halves, d.q_heads, d.k_heads, (hipStream_t)stream);
}
