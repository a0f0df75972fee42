// Rotary positions with several axes on queries and keys: pair (x, y) of a token's head -> (x cos a - y sin a, x sin a + y cos a).
//
// Bound by memory: every value of q and k is read and written once.  The angles of a token are the same for all of its heads, so a
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
    size_t q_stride, k_stride, q_out_stride, k_out_stride;   // elements
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

// A unit is what a thread turns at a time: HALVES: two 16-byte vectors half the rotated width apart (behind it two that are only scaled);
// otherwise one vector of neighbouring pairs.
template <typename T, bool HALVES>
__global__ __launch_bounds__(kThreads) void rotary_kernel(RotaryArgs a) {
    typedef typename Vec<T>::type vec;
    constexpr int N = Vec<T>::n;
    extern __shared__ f32x2 turn[];     // [tile][half]
    const int t0 = blockIdx.x * a.tile, tokens = min(a.tile, a.tokens - t0);
    const int total = tokens * a.units;
    const T* in[kUnroll];
    T* out[kUnroll];
    vec x[kUnroll], y[kUnroll];
    int pair[kUnroll], token[kUnroll];
    float scale[kUnroll];
    int apart = 0, apart_rest = 0;      // HALVES: elements between the two vectors
    if constexpr (HALVES) {
        apart = a.half;
        apart_rest = a.head_dim / 2 - a.half;
    }
    auto load = [&](int i0) {
#pragma unroll
        for (int j = 0; j < kUnroll; j++) {
            const int i = i0 + j * kThreads;
            if (i >= total) { pair[j] = -1; continue; }
            const int tok = quotient(i, a.unit_magic);
            int u = i - tok * a.units;
            const bool is_q = u < a.q_units;
            const size_t at = t0 + tok;
            const T* src = static_cast<const T*>(is_q ? a.q : a.k) + at * (is_q ? a.q_stride : a.k_stride);
            T* dst = static_cast<T*>(is_q ? a.q_out : a.k_out) + at * (is_q ? a.q_out_stride : a.k_out_stride);
            if (!is_q) u -= a.q_units;
            scale[j] = is_q ? a.q_scale : 1.f;
            token[j] = tok;
            const int head = quotient(u, a.head_magic), v = u - head * a.head_units;
            int off;
            if constexpr (HALVES) {
                const bool turned = v * N < a.half;
                off = head * a.head_dim + (turned ? v * N : a.half + v * N);      // behind the rotated width R = 2 half: R + (v N - half)
                pair[j] = turned ? v * N : kMaxPairs;
            } else {
                off = u * N;
                pair[j] = v * (N / 2);
            }
            in[j] = src + off;
            out[j] = dst + off;
            x[j] = *reinterpret_cast<const vec*>(in[j]);
            if constexpr (HALVES) y[j] = *reinterpret_cast<const vec*>(in[j] + (pair[j] < kMaxPairs ? apart : apart_rest));
        }
    };
    auto finish = [&]() {
#pragma unroll
        for (int j = 0; j < kUnroll; j++) {
            if (pair[j] < 0) continue;
            const f32x2* cs = turn + token[j] * a.half;
            vec u, w;
            if constexpr (HALVES) {
                const bool turned = pair[j] < kMaxPairs;
#pragma unroll
                for (int e = 0; e < N; e++) {
                    const float p = to_f32<T>(x[j][e]) * scale[j], q = to_f32<T>(y[j][e]) * scale[j];
                    const f32x2 c = cs[turned ? pair[j] + e : 0];
                    u[e] = from_f32<T>(turned ? fmaf(p, c[0], -q * c[1]) : p);
                    w[e] = from_f32<T>(turned ? fmaf(p, c[1], q * c[0]) : q);
                }
                *reinterpret_cast<vec*>(out[j]) = u;
                *reinterpret_cast<vec*>(out[j] + (turned ? apart : apart_rest)) = w;
            } else {
#pragma unroll
                for (int e = 0; e < N / 2; e++) {
                    const float p = to_f32<T>(x[j][2 * e]) * scale[j], q = to_f32<T>(x[j][2 * e + 1]) * scale[j];
                    const bool turned = pair[j] + e < a.half;
                    const f32x2 c = cs[turned ? pair[j] + e : 0];
                    u[2 * e] = from_f32<T>(turned ? fmaf(p, c[0], -q * c[1]) : p);
                    u[2 * e + 1] = from_f32<T>(turned ? fmaf(p, c[1], q * c[0]) : q);
                }
                *reinterpret_cast<vec*>(out[j]) = u;
            }
        }
    };
    load(threadIdx.x);                  // on their way while the angles are formed
    for (int i = threadIdx.x; i < tokens * a.half; i += kThreads) {
        const int tok = i / a.half, p = i - tok * a.half;
        const double pos = (double)a.positions[(size_t)(t0 + tok) * a.axes + a.axis[p]];
        turn[i] = cos_sin_turns(pos * a.turns[p]);
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
    // tokens per workgroup: about one round of loads, so that a long batch runs many workgroups and a short one still spreads over the chip
    const int round = kThreads * kUnroll;
    a.tile = a.units >= round ? 1 : round / a.units;
    if (a.tile > 32) a.tile = 32;       // (32 x 128 pairs: 32 KB of LDS)
    a.unit_magic = magic_of((unsigned)a.units);
    a.head_magic = magic_of((unsigned)a.head_units);
    const dim3 grid((unsigned)(((size_t)a.tokens + a.tile - 1) / a.tile));
    const size_t lds = (size_t)a.tile * (a.half > 0 ? a.half : 1) * sizeof(f32x2);
    HybTraceScope trace("rotary", "byte", 2.0 * a.tokens * (q_heads + k_heads) * (double)a.head_dim * sizeof(T), st);
    if (halves) hipLaunchKernelGGL((rotary_kernel<T, true>), grid, dim3(kThreads), lds, st, a);
    else hipLaunchKernelGGL((rotary_kernel<T, false>), grid, dim3(kThreads), lds, st, a);
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
    a.q_stride = d.q_stride; a.k_stride = d.k_stride; a.q_out_stride = d.q_out_stride; a.k_out_stride = d.k_out_stride;
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
