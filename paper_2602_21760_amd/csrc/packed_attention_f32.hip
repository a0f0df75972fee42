// fp32 attention over packed batches on the fp32 matrix cores (reference precision), the merge of cut keys for both types, and the entry point.
//
// A workgroup of 4 waves owns 32 rows (small launches at head_dim 128: 16) of one (sequence, key head) and splits the KEYS: wave w takes the 32-key tiles w, w + 4, ... with a running reference and normaliser of
// its own; the four partial results are merged in LDS in a fixed order.  Keys and values go straight from memory (L2) to registers, the queries, which all waves share, lie in LDS.
// S^T = K Q^T and O^T += V^T P^T on v_mfma_f32_16x16x4_f32: a 16-byte load gives a lane 4 features of its key for 4 MFMAs, and register i of the exponentiated S^T is the B operand of
// the MFMA over the keys 4 q4 + i, with rows 4 q4 + i of V as the A operand.
//
// Bound by the matrix cores, which share their issue with everything else here: fp32 MFMAs and vector instructions of the waves of a SIMD do not overlap (busy 75 % and 22 % of the time
// at head_dim 64, no better with waves of different priority).  So a tile has few others: a probability is one fma and one
// v_exp_f32, 2^(c score - reference), whose error is that of an argument near 0 wherever the probability counts; masks, maxima across lanes and rescaling only where a tile asks for them;
// offsets of buffer loads that no tile changes.  One sequence of 4096, 8 heads: head_dim 64 130 TFLOP/s, 128 118 (a large library product in fp32 reaches 139); with 16 rows 110 and 107.
// The queries in LDS make room for a third workgroup at head_dim 64 (in registers, with the next tile's keys requested ahead: 314, 1302 and 259 tokens, 12 / 4 heads, 65 us, so 61) and for
// 32 rows at 128 (16 rows: 800, 300 and 1200 tokens, causal, 16 / 8 heads, 115 us, so 99; three sequences of 142 to 605, 4 heads: 25 and 34).  Ragged and small launches are held by the 10 us that a workgroup takes beside its tiles.
#include "packed_attention.h"

#include <math.h>

namespace {

constexpr int BKV = 32;
constexpr int WAVES = 4;
constexpr float RESCALE_LOG2 = 8.0f;

__device__ __forceinline__ f32x4 load16(__amdgpu_buffer_rsrc_t rsrc, int offset) { return __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(rsrc, offset, 0, 0)); }

template <int D, int BQ>
__global__ __launch_bounds__(256, D == 64 ? 3 : 2) void packed_attention_f32_kernel(PackedAttnArgs a) {
    constexpr int QT = BQ / 16, DT = D / 16, VH = D / 64;
    __shared__ f32x4 part_o[WAVES][QT][DT][64];      // [wave][row tile][feature tile][lane]
    __shared__ float part_ml[WAVES][QT][2][16];      // [wave][row tile][maximum, normaliser][row]
    const PackedUnit u = packed_unit<BQ, true>(a, packed_group_id());
    if (u.rows == 0) return;
    const int lane = threadIdx.x % 64, l16 = lane % 16, q4 = lane / 16;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const char* kp = static_cast<const char*>(a.k) + (size_t)u.k0 * a.k_token + (size_t)u.head * a.k_head;
    const char* vp = static_cast<const char*>(a.v) + (size_t)u.k0 * a.v_token + (size_t)u.head * a.v_head;

    const float c = a.prescaled ? 1.f : a.scale * 1.4426950408889634f;
    int last[QT];
#pragma unroll
    for (int qt = 0; qt < QT; qt++) last[qt] = packed_last_key(a, u, packed_div(u.row0 + min(qt * 16 + l16, u.rows - 1), a.by_group));
    // the queries in LDS, where the waves' results go later: 16-byte slot s of row r at s ^ (r % 16)
    f32x4* const q = &part_o[0][0][0][0];
#pragma unroll
    for (int i = 0; i < BQ * D / 4 / 256; i++) {
        const int r = (threadIdx.x + 256 * i) / (D / 4), slot = threadIdx.x % (D / 4), row = u.row0 + min(r, u.rows - 1), t = packed_div(row, a.by_group);
        q[r * (D / 4) + (slot ^ (r % 16))] =
            *reinterpret_cast<const f32x4*>(static_cast<const char*>(a.q) + (size_t)(u.q0 + t) * a.q_token + (size_t)(u.head * a.group + row - t * a.group) * a.q_head + 16 * slot);
    }
    __syncthreads();
    const int block_min = packed_last_key(a, u, packed_div(u.row0, a.by_group)), block_max = packed_last_key(a, u, packed_div(u.row0 + u.rows - 1, a.by_group));
    const int nt = (block_max + BKV) / BKV, part_tiles = packed_part_tiles(a, nt, BKV);
    const int t_begin = min(u.part * part_tiles, nt), t_end = min(t_begin + part_tiles, nt);

    float m[QT], l[QT];
    f32x4 o[DT][QT];     // [feature tile][row tile]
#pragma unroll
    for (int qt = 0; qt < QT; qt++) {
        m[qt] = -__builtin_inff();
        l[qt] = 0.f;
#pragma unroll
        for (int dt = 0; dt < DT; dt++) o[dt][qt] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    // byte offsets of the lane's rows in a tile; rows behind the last key lie outside the resource and come as zeros
    int k_off[2], v_off[2][4];
#pragma unroll
    for (int kt = 0; kt < 2; kt++) {
        k_off[kt] = (kt * 16 + l16) * (int)a.k_token + 16 * q4;
#pragma unroll
        for (int i = 0; i < 4; i++) v_off[kt][i] = (kt * 16 + 4 * q4 + i) * (int)a.v_token + 16 * l16;
    }
    for (int t = t_begin + wave; t < t_end; t += WAVES) {
        const int key0 = t * BKV, more = min(u.n_k - key0, BKV) - 1;
        const __amdgpu_buffer_rsrc_t k_rsrc = __builtin_amdgcn_make_buffer_rsrc((void*)(kp + (size_t)key0 * a.k_token), 0, more * (int)a.k_token + 4 * D, 0x00020000);
        const __amdgpu_buffer_rsrc_t v_rsrc = __builtin_amdgcn_make_buffer_rsrc((void*)(vp + (size_t)key0 * a.v_token), 0, more * (int)a.v_token + 4 * D, 0x00020000);
        f32x4 k[2][DT], v[2][4][VH];     // K: [key tile][16-feature step]; V: [key tile][row 4 q4 + i][64 features]
#pragma unroll
        for (int kt = 0; kt < 2; kt++)
#pragma unroll
            for (int s = 0; s < DT; s++) k[kt][s] = load16(k_rsrc, k_off[kt] + 64 * s);
        auto load_v = [&](int kt) {
#pragma unroll
            for (int i = 0; i < 4; i++)
#pragma unroll
                for (int h = 0; h < VH; h++) v[kt][i][h] = load16(v_rsrc, v_off[kt][i] + 256 * h);
        };
        load_v(0);
        if constexpr (D == 64 || BQ == 16) load_v(1);
        f32x4 s[2][QT];      // [key tile][row tile]: keys 16 kt + 4 q4 + i
#pragma unroll
        for (int kt = 0; kt < 2; kt++)
#pragma unroll
            for (int qt = 0; qt < QT; qt++) s[kt][qt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int st = 0; st < DT; st++) {
            f32x4 qs[QT];
#pragma unroll
            for (int qt = 0; qt < QT; qt++) qs[qt] = q[(qt * 16 + l16) * (D / 4) + ((4 * st + q4) ^ l16)];
#pragma unroll
            for (int j = 0; j < 4; j++)
#pragma unroll
                for (int kt = 0; kt < 2; kt++)
#pragma unroll
                    for (int qt = 0; qt < QT; qt++) s[kt][qt] = __builtin_amdgcn_mfma_f32_16x16x4f32(k[kt][st][j], qs[qt][j], s[kt][qt], 0, 0, 0);
        }
        if constexpr (D == 128 && BQ == 32) load_v(1);       // (into registers that the keys leave)
        const bool masked = key0 + BKV - 1 > block_min;
        if (masked) {
#pragma unroll
            for (int qt = 0; qt < QT; qt++) {
                const int seen = last[qt] - key0 - 4 * q4;      // keys 16 kt + i > seen are hidden
#pragma unroll
                for (int kt = 0; kt < 2; kt++)
#pragma unroll
                    for (int i = 0; i < 4; i++) s[kt][qt][i] = kt * 16 + i > seen ? -__builtin_inff() : s[kt][qt][i];
            }
        }
        // the reference m (in base 2) only advances when a score exceeds it by more than 2^RESCALE_LOG2; it is the same for the four lanes of a row
        float mx[QT];
        bool grows = false;
#pragma unroll
        for (int qt = 0; qt < QT; qt++) {
            mx[qt] = fmaxf(fmaxf(fmaxf(s[0][qt][0], s[0][qt][1]), fmaxf(s[0][qt][2], s[0][qt][3])), fmaxf(fmaxf(s[1][qt][0], s[1][qt][1]), fmaxf(s[1][qt][2], s[1][qt][3])));
            grows |= fmaf(mx[qt], c, -m[qt]) > RESCALE_LOG2;
        }
        if (__any(grows)) {
#pragma unroll
            for (int qt = 0; qt < QT; qt++) {
                mx[qt] = fmaxf(mx[qt], __shfl_xor(mx[qt], 16, 64));
                mx[qt] = fmaxf(mx[qt], __shfl_xor(mx[qt], 32, 64)) * c;
                const bool grow = mx[qt] - m[qt] > RESCALE_LOG2;
                const float corr = grow ? __builtin_amdgcn_exp2f(m[qt] - mx[qt]) : 1.f;      // first tile: 2^-inf = 0
                m[qt] = grow ? mx[qt] : m[qt];
                l[qt] *= corr;
#pragma unroll
                for (int dt = 0; dt < DT; dt++) o[dt][qt] *= corr;
            }
        }
#pragma unroll
        for (int qt = 0; qt < QT; qt++) {
            const float ref = m[qt] == -__builtin_inff() ? 0.f : m[qt];          // only hidden keys so far: all probabilities 0
#pragma unroll
            for (int kt = 0; kt < 2; kt++)
#pragma unroll
                for (int i = 0; i < 4; i++) {
                    s[kt][qt][i] = __builtin_amdgcn_exp2f(fmaf(s[kt][qt][i], c, -ref));
                    l[qt] += s[kt][qt][i];
                }
        }
        // a probability of 0 does not keep an infinity or NaN of a hidden key's value out of the MFMA: such values are added to the rows that see them by hand
        if (masked) {
            unsigned any = 0;
#pragma unroll
            for (int kt = 0; kt < 2; kt++)
#pragma unroll
                for (int i = 0; i < 4; i++)
#pragma unroll
                    for (int h = 0; h < VH; h++)
#pragma unroll
                        for (int e = 0; e < 4; e++) any |= odd_bits_f32(__float_as_uint(v[kt][i][h][e]));
            if (__any(any != 0)) {
#pragma unroll 1
                for (int key = key0; key < min(key0 + BKV, u.n_k); key++) {
#pragma unroll
                    for (int dt = 0; dt < DT; dt++)
#pragma unroll
                        for (int i = 0; i < 4; i++) {
                            __builtin_amdgcn_sched_barrier(0);      // (one value at a time: this path's registers count for the whole kernel)
                            unsigned x = *reinterpret_cast<const unsigned*>(vp + (size_t)key * a.v_token + 4 * ((dt / 4) * 64 + 16 * q4 + 4 * i + dt % 4));
                            x &= odd_mask_f32(x);
#pragma unroll
                            for (int qt = 0; qt < QT; qt++) o[dt][qt][i] += __uint_as_float(x & (key <= last[qt] ? ~0u : 0u));
                        }
                }
#pragma unroll
                for (int kt = 0; kt < 2; kt++)
#pragma unroll
                    for (int i = 0; i < 4; i++)
#pragma unroll
                        for (int h = 0; h < VH; h++)
#pragma unroll
                            for (int e = 0; e < 4; e++) v[kt][i][h][e] = __uint_as_float(__float_as_uint(v[kt][i][h][e]) & ~odd_mask_f32(__float_as_uint(v[kt][i][h][e])));
            }
        }
#pragma unroll
        for (int kt = 0; kt < 2; kt++)
#pragma unroll
            for (int i = 0; i < 4; i++)
#pragma unroll
                for (int dt = 0; dt < DT; dt++)
#pragma unroll
                    for (int qt = 0; qt < QT; qt++) o[dt][qt] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[kt][i][dt / 4][dt % 4], s[kt][qt][i], o[dt][qt], 0, 0, 0);
    }

    __syncthreads();         // everyone is done with the queries
    // merge of the waves: row = sum_p o_p 2^(m_p - M) / sum_p l_p 2^(m_p - M), p in order
#pragma unroll
    for (int qt = 0; qt < QT; qt++) {
        l[qt] += __shfl_xor(l[qt], 16, 64);
        l[qt] += __shfl_xor(l[qt], 32, 64);
        if (q4 == 0) {
            part_ml[wave][qt][0][l16] = m[qt];
            part_ml[wave][qt][1][l16] = l[qt];
        }
#pragma unroll
        for (int dt = 0; dt < DT; dt++) part_o[wave][qt][dt][lane] = o[dt][qt];
    }
    __syncthreads();
    // a wave finishes one row tile's 64 features, or half of their registers: register i of feature tiles 4 h .. 4 h + 3 is features 64 h + 16 q4 + 4 i .. + 3 of row l16
    constexpr int SPLIT = WAVES / (QT * VH), NI = 4 / SPLIT;
    typedef float regs __attribute__((ext_vector_type(NI)));
    const int qt = wave / SPLIT / VH, h = wave / SPLIT % VH, i0 = wave % SPLIT * NI;
    if (qt * 16 + l16 >= u.rows) return;
    float m_all = part_ml[0][qt][0][l16], l_all = 0.f;
#pragma unroll
    for (int p = 1; p < WAVES; p++) m_all = fmaxf(m_all, part_ml[p][qt][0][l16]);
    f32x4 r[NI];
#pragma unroll
    for (int i = 0; i < NI; i++) r[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int p = 0; p < WAVES; p++) {
        const float mp = part_ml[p][qt][0][l16], lp = part_ml[p][qt][1][l16];
        if (lp == 0.f) continue;     // a wave without keys for this row counts nothing
        const float w = mp == m_all ? 1.f : __builtin_amdgcn_exp2f(mp - m_all);
        l_all = fmaf(lp, w, l_all);
#pragma unroll
        for (int e = 0; e < 4; e++) {
            const regs y = *reinterpret_cast<const regs*>(reinterpret_cast<const float*>(&part_o[p][qt][4 * h + e][lane]) + i0);
#pragma unroll
            for (int i = 0; i < NI; i++) r[i][e] = fmaf(y[i], w, r[i][e]);
        }
    }
    const int row = u.row0 + qt * 16 + l16, tok = packed_div(row, a.by_group), head = u.head * a.group + (row - tok * a.group);
    const int feature = 64 * h + 16 * q4 + 4 * i0;
    if (a.parts > 1) {
        const size_t at = ((size_t)(u.q0 + tok) * a.q_heads + head) * a.parts + u.part;
        if (feature == 0) *reinterpret_cast<f32x2*>(a.part + (size_t)a.total_q * a.q_heads * a.parts * D + at * 2) = f32x2{m_all, l_all};
#pragma unroll
        for (int i = 0; i < NI; i++) *reinterpret_cast<f32x4*>(a.part + at * D + feature + 4 * i) = r[i];
        return;
    }
    float* op = reinterpret_cast<float*>(static_cast<char*>(a.o) + (size_t)(u.q0 + tok) * a.o_token + (size_t)head * a.o_head) + feature;
#pragma unroll
    for (int i = 0; i < NI; i++) *reinterpret_cast<f32x4*>(op + 4 * i) = l_all == 0.f ? f32x4{0.f, 0.f, 0.f, 0.f} : r[i] / l_all;
}

// Joins the parts of cut keys: with references m_p, normalisers l_p and accumulators o_p a row is sum_p o_p w_p / sum_p l_p w_p, w_p = 2^(m_p - M),
// M = max m_p over the parts with keys, parts in index order.  D / 4 lanes per row, four features each; lane f has the weights of parts f, f + D / 4, ...
// Rows are those of all offsets (they do not decrease), so no sequence has to be found: one trip to memory for the pairs and the first accumulators, one for every eight more.  Bound
// by that latency and, for many rows, by the partial results it reads.
template <typename T, int D>
__global__ __launch_bounds__(256) void packed_merge_kernel(PackedAttnArgs a, PackedDivisor by_q_heads) {
    constexpr int G = D / 4, ROWS = 64 / G, E = kPackedMaxParts / G, U = 8;
    typedef T tx4 __attribute__((ext_vector_type(4)));
    const int lane = threadIdx.x % 64, g = lane / G, f = lane % G, parts = a.parts;
    const unsigned all = (unsigned)a.total_q * (unsigned)a.q_heads, row = (packed_group_id() * 4 + threadIdx.x / 64) * ROWS + g, r = min(row, all - 1);
    const float* o = a.part + (size_t)r * parts * D + 4 * f;
    const f32x2* pairs = reinterpret_cast<const f32x2*>(a.part + (size_t)all * parts * D) + (size_t)r * parts;
    f32x2 e[E];
#pragma unroll
    for (int i = 0; i < E; i++) e[i] = pairs[min(f + i * G, parts - 1)];
    const int begin = packed_offset(a.offsets_q, 0, a.total_q), end = packed_offset(a.offsets_q, a.sequences, a.total_q);
    float m = -__builtin_inff(), l = 0.f, w[E];
    bool any[E];
#pragma unroll
    for (int i = 0; i < E; i++) {
        any[i] = f + i * G < parts && e[i][1] != 0.f;      // (a part without keys for this row: its accumulators were not written)
        m = fmaxf(m, any[i] ? e[i][0] : -__builtin_inff());
    }
#pragma unroll
    for (int s = G / 2; s > 0; s >>= 1) m = fmaxf(m, __shfl_xor(m, s, 64));
#pragma unroll
    for (int i = 0; i < E; i++) {
        w[i] = !any[i] ? -1.f : e[i][0] == m ? 1.f : __builtin_amdgcn_exp2f(e[i][0] - m);
        l += any[i] ? e[i][1] * w[i] : 0.f;
    }
#pragma unroll
    for (int s = G / 2; s > 0; s >>= 1) l += __shfl_xor(l, s, 64);
    f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < E; i++) {
        for (int p0 = i * G; p0 < min((i + 1) * G, parts); p0 += U) {
            f32x4 v[U];
#pragma unroll
            for (int j = 0; j < U; j++) v[j] = *reinterpret_cast<const f32x4*>(o + (size_t)min(p0 + j, parts - 1) * D);
#pragma unroll
            for (int j = 0; j < U; j++) {
                const float wp = p0 + j < parts ? __shfl(w[i], g * G + p0 + j - i * G, 64) : -1.f;
#pragma unroll
                for (int k = 0; k < 4; k++) x[k] = wp >= 0.f ? fmaf(v[j][k], wp, x[k]) : x[k];
            }
        }
    }
    const int tok = packed_div((int)r, by_q_heads), head = (int)r - tok * a.q_heads;
    if (row >= all || tok < begin || tok >= end) return;
    const float inv = l == 0.f ? 0.f : 1.0f / l;
    *reinterpret_cast<tx4*>(static_cast<char*>(a.o) + (size_t)tok * a.o_token + (size_t)head * a.o_head + 4 * f * sizeof(T)) =
        tx4{from_f32<T>(x[0] * inv), from_f32<T>(x[1] * inv), from_f32<T>(x[2] * inv), from_f32<T>(x[3] * inv)};
}

template <typename T, int D>
int launch_merge(const PackedAttnArgs& a, hipStream_t st) {
    constexpr size_t kRows = 4 * (64 / (D / 4));         // of a workgroup
    HybTraceScope trace("packed_attention_merge", "byte", 4.0 * packed_part_floats(a.total_q, a.q_heads, a.parts, D), st);
    hipLaunchKernelGGL((packed_merge_kernel<T, D>), packed_grid_of(((size_t)a.total_q * a.q_heads + kRows - 1) / kRows), dim3(256), 0, st, a, packed_divisor((unsigned)a.q_heads));
    return hyb_check_launch("packed_attention_merge");
}

// How many parts the keys of a block are cut into; each block deals its own keys out to them.  The least over an estimate of a launch's length in us: the longest part's keys at the pace of a
// workgroup that is alone on its CU, or all blocks' at the pace of a full chip, whatever is longer; the start of the workgroups; the merge: a launch, a share per row, the partial results that are
// written and read.  Fitted to 344 launches of 1 to 64 sequences of 50 to 9000 keys, in caches and out of them, each in 1 to 32 parts: 1.4 % above the best on average, 3 % where the keys come from
// memory (as many parts as fill the chip: 7 and 9 %; 10 heads of 64, 8 sequences of 648: not cut 21 us, in two 43; 17 tokens over 2031 to 3695 keys, 16 / 8 heads of 128: 69 and, in six, 22).
// Never more than the chip holds at once.  max_k == 0: half as many again as the mean; it decides the number of parts only.
void choose_parts(PackedAttnArgs& a, int max_k, bool f32, int head_dim) {
    const double mean = (double)a.total_k / a.sequences, most = max_k > 0 ? max_k : 1.5 * mean, keys = most < a.total_k ? most : a.total_k;
    if (!f32 && keys <= 512) return;                // (bf16 blocks of so few keys gain nothing: 10.5 us, cut 12.9)
    const double key = f32 ? (head_dim == 64 ? 0.015 : 0.025) : head_dim == 64 ? 0.009 : 0.014;
    const double blocks = ((double)a.total_q * a.group / a.rows + 0.5 * a.sequences) * a.k_heads;
    const double seen = a.causal && a.total_q == a.total_k ? 0.5 * mean : mean, all = blocks * seen * key / (hyb_cu_count() * (f32 ? 1.2 : 1.6));
    const double rows = (double)a.total_q * a.q_heads;
    if (rows > 1 << 30) return;                     // (the merge counts rows in 32 bits)
    double best = 0;
    const int slots = hyb_cu_count() * (f32 ? 2 : head_dim == 64 ? 4 : 3);
    for (int parts = 1; parts <= kPackedMaxParts && (parts == 1 || ((parts - 1) * kPackedPartKeys < keys && parts * blocks <= slots)); parts++) {
        const double share = keys / parts > kPackedPartKeys ? keys / parts : kPackedPartKeys, own = (parts == 1 ? keys : share) * key;
        const double merge = parts == 1 ? 0 : 2.4 + rows * (0.1e-3 + 0.1e-3 * parts * head_dim / 64);
        const double us = (own > all ? own : all) + 0.003 * blocks * parts + merge;
        if (parts == 1 || us < best) {
            best = us;
            a.parts = parts;
        }
    }
}

// Pieces of the few-rows kernel: all keys dealt out over the chip, two pieces for every workgroup that fits it (one: 11 % slower over caches of 100 to 8000 keys, three: the same), of at
// least 256 keys (8000 keys of one sequence, 8 heads of 128: 11.7 us; of 512: 13.0), or 512 where the sequences alone fill the chip.  Sequences of which the caller says that none is
// longer than a piece are one piece each, whatever their length, and need no join.  So are those of up to 1024 keys (head_dim 128: 768; the join costs more than they take: 16 caches of up to 600, 32 / 8
// heads of 64, 11.3 us, so 8.3; one of 1024 9.7 both, of 2000 9.7 and 13.9), and those of up to 2048 and much the same length that keep a quarter of the CUs busy: what pieces cost in starts
// and join is more than what they even out (8 heads of 128: 40 caches of 630 to 700 keys 24.8 us, in pieces 31.0; 87 of 1080 to 1200 77 / 97; 16 of up to 2000 22.3 / 24.6; 4 of up to 2000 19.1 / 13.4;
// 53 of 2700 to 3000 125 / 132, but 40 of them 110 / 103.  256 caches of which every second has 2000 keys, the others 50, 4 heads: 130 / 118).
void choose_pieces(PackedAttnArgs& a, int max_k, int head_dim) {
    const int slots = hyb_cu_count() * (head_dim == 64 ? 4 : 2);
    long long len = ((long long)a.total_k * a.k_heads / (2 * slots) + 63) / 64 * 64;
    const int least = (long long)a.sequences * a.k_heads >= slots ? 512 : 256;
    if (len < least) len = least;
    const bool alike = max_k <= 2048 && 4ll * a.sequences * max_k <= 7ll * a.total_k && 4ll * a.total_k * a.k_heads >= (long long)max_k * hyb_cu_count();
    if (max_k > 0 && (max_k <= len || max_k <= (head_dim == 64 ? 1024 : 768) || alike)) len = 1 << 30;
    a.part_keys = (int)len;
    a.by_piece = packed_divisor((unsigned)len);
    a.pieces = (int)(a.total_k / len) + a.sequences;
    a.rests_last = a.sequences <= 64 && (long long)a.pieces * a.k_heads > slots;
    a.blocks = (int)packed_blocks(a, 1);       // of the join
}

int fill_args(const char* who, const hyb_packed_attention_desc* desc, PackedAttnArgs& a) {
    HYB_REQUIRE(desc != nullptr, HYB_ERR_NULL, "%s: argument 'desc' is NULL", who);
    const hyb_packed_attention_desc& d = *desc;
    HYB_ARG_DTYPE(who, d.dtype);
    HYB_REQUIRE(d.sequences >= 0 && d.total_q >= 0 && d.total_k >= 0 && d.max_q >= 0 && d.max_k >= 0, HYB_ERR_SHAPE, "%s: negative size", who);
    HYB_REQUIRE(d.head_dim == 64 || d.head_dim == 128, HYB_ERR_SHAPE, "%s: head_dim %d is not supported (only 64 and 128)", who, d.head_dim);
    HYB_REQUIRE(d.q_heads > 0 && d.k_heads > 0 && d.q_heads <= 65535 && d.q_heads % d.k_heads == 0, HYB_ERR_SHAPE, "%s: %d query heads are no multiple of %d key heads", who, d.q_heads, d.k_heads);
    HYB_REQUIRE(d.prescaled != 0 || d.scale <= 0.f || isfinite(d.scale * 1.4426950408889634f), HYB_ERR_SHAPE, "%s: scale %g is not finite in base 2", who, (double)d.scale);
    const size_t es = hyb_dtype_size(d.dtype), vec = 16 / es;
    const size_t strides[8] = {d.q_token_stride, d.q_head_stride, d.k_token_stride, d.k_head_stride, d.v_token_stride, d.v_head_stride, d.o_token_stride, d.o_head_stride};
    for (size_t s : strides) {
        HYB_REQUIRE(s % vec == 0, HYB_ERR_ALIGN, "%s: a stride of %zu elements is not a multiple of 16 bytes", who, s);
        HYB_REQUIRE(s < ((size_t)1 << 40), HYB_ERR_SHAPE, "%s: a stride of %zu elements is too large", who, s);
    }
    for (int i = 0; i < 8; i += 2) HYB_REQUIRE(strides[i] < ((size_t)1 << 23), HYB_ERR_SHAPE, "%s: a token stride of %zu elements is not below 2^23", who, strides[i]);
    a = {};
    a.sequences = d.sequences; a.total_q = d.total_q; a.total_k = d.total_k;
    a.q_heads = d.q_heads; a.k_heads = d.k_heads; a.group = d.q_heads / d.k_heads;
    a.by_group = packed_divisor((unsigned)a.group);
    a.scale = d.scale > 0.f ? d.scale : (d.head_dim == 64 ? 0.125f : 0.08838834764831845f);
    a.causal = d.causal != 0; a.prescaled = d.prescaled != 0;
    a.q_token = d.q_token_stride * es; a.q_head = d.q_head_stride * es; a.k_token = d.k_token_stride * es; a.k_head = d.k_head_stride * es;
    a.v_token = d.v_token_stride * es; a.v_head = d.v_head_stride * es; a.o_token = d.o_token_stride * es; a.o_head = d.o_head_stride * es;
    HYB_REQUIRE(d.total_k <= 1 << 30, HYB_ERR_SHAPE, "%s: more than 2^30 rows of keys (%d)", who, d.total_k);
    HYB_REQUIRE((long long)d.total_q * a.group < (1ll << 31) && packed_blocks(a, 1) * a.k_heads < (1ll << 31) && ((long long)d.total_k / 256 + d.sequences) * a.k_heads < (1ll << 29), HYB_ERR_SHAPE, "%s: too many rows (%d of queries, %d of keys, %d heads)", who, d.total_q, d.total_k, d.q_heads);
    a.xcd_heads = d.k_heads % 8 == 0 ? 8 : d.k_heads % 4 == 0 ? 4 : d.k_heads % 2 == 0 ? 2 : 1;
    a.xcd_share = 8 / a.xcd_heads;
    a.xcd_shift = a.xcd_heads == 8 ? 3 : a.xcd_heads / 2;
    a.parts = 1;
    // at most 16 rows per sequence: the kernel whose waves split the keys (only the sizes that the caller names can say so; any others are right, too)
    if (d.dtype == HYB_BF16 && d.max_q > 0 && (long long)d.max_q * a.group <= kPackedRowsFew) {
        choose_pieces(a, d.max_k, d.head_dim);
    } else {
        // fp32, head_dim 128: blocks of 32 rows where they fill three quarters of the chip's two workgroups a CU, of 16 otherwise
        const bool small = d.head_dim == 128 && ((long long)d.total_q * a.group / 32 + d.sequences / 2) * a.k_heads * 2 < 3 * hyb_cu_count();
        a.rows = d.dtype == HYB_BF16 ? kPackedRowsMfma : small ? 16 : 32;
        a.blocks = (int)packed_blocks(a, a.rows);
        if (d.sequences > 0) choose_parts(a, d.max_k, d.dtype == HYB_F32, d.head_dim);
    }
    return HYB_OK;
}

size_t scratch_bytes(const PackedAttnArgs& a, int head_dim) {
    const size_t floats = a.pieces > a.sequences ? packed_piece_rows(a.pieces, a.k_heads) * (head_dim + 2) : a.parts > 1 ? packed_part_floats(a.total_q, a.q_heads, a.parts, head_dim) : 0;
    return hyb_align_up(floats * sizeof(float), 256);
}

}  // namespace

int hyb_launch_packed_attention_f32(PackedAttnArgs& a, int head_dim, hipStream_t st) {
    const dim3 grid = packed_grid(a);
    HybTraceScope trace("packed_attention_f32", "byte", 8.0 * head_dim * ((double)a.total_q * a.q_heads + (double)a.total_k * a.k_heads), st);
    if (head_dim == 64) hipLaunchKernelGGL((packed_attention_f32_kernel<64, 32>), grid, dim3(256), 0, st, a);
    else if (a.rows == 32) hipLaunchKernelGGL((packed_attention_f32_kernel<128, 32>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((packed_attention_f32_kernel<128, 16>), grid, dim3(256), 0, st, a);
    return hyb_check_launch("packed_attention_f32");
}

extern "C" size_t hyb_packed_attention_workspace_bytes(const hyb_packed_attention_desc* desc) {
    PackedAttnArgs a;
    if (fill_args("hyb_packed_attention_workspace_bytes", desc, a) != HYB_OK) return 0;
    return scratch_bytes(a, desc->head_dim);
}

extern "C" int hyb_packed_attention(const hyb_packed_attention_desc* desc, const void* q, const void* k, const void* v, void* o,
                                    const int* offsets_q, const int* offsets_k, void* workspace, size_t workspace_bytes, void* stream) {
    PackedAttnArgs a;
    int rc = fill_args("hyb_packed_attention", desc, a);
    if (rc) return rc;
    const hyb_packed_attention_desc& d = *desc;
    if (d.sequences == 0 || d.total_q == 0) return HYB_OK;
    HYB_CHECK_PTR(q); HYB_CHECK_PTR(o); HYB_CHECK_PTR(offsets_q); HYB_CHECK_PTR(offsets_k);
    HYB_CHECK_ALIGN(q); HYB_CHECK_ALIGN(o); HYB_CHECK_ALIGN(offsets_q); HYB_CHECK_ALIGN(offsets_k);
    if (d.total_k > 0) { HYB_CHECK_PTR(k); HYB_CHECK_PTR(v); }
    HYB_CHECK_ALIGN(k); HYB_CHECK_ALIGN(v);
    const size_t heads = (size_t)d.q_heads, row = (size_t)d.head_dim;
    HYB_REQUIRE((d.o_head_stride >= row && d.o_token_stride >= (heads - 1) * d.o_head_stride + row) ||
                    (d.o_token_stride >= row && d.o_head_stride >= ((size_t)d.total_q - 1) * d.o_token_stride + row),
                HYB_ERR_SHAPE, "hyb_packed_attention: the strides of o let its rows overlap");
    const size_t need = scratch_bytes(a, d.head_dim);
    if (need > 0) {
        HYB_CHECK_PTR(workspace); HYB_CHECK_ALIGN(workspace);
        HYB_REQUIRE(workspace_bytes >= need, HYB_ERR_WORKSPACE, "hyb_packed_attention: workspace of %zu bytes is smaller than the %zu required", workspace_bytes, need);
        a.part = static_cast<float*>(workspace);
    }
    a.q = q; a.k = k; a.v = v; a.o = o; a.offsets_q = offsets_q; a.offsets_k = offsets_k;
    const hipStream_t st = (hipStream_t)stream;
    rc = a.pieces ? hyb_launch_packed_attention_few(a, d.head_dim, st) : d.dtype == HYB_BF16 ? hyb_launch_packed_attention_mfma(a, d.head_dim, st) : hyb_launch_packed_attention_f32(a, d.head_dim, st);
    if (rc || a.pieces || a.parts == 1) return rc;
    if (d.dtype == HYB_BF16) return d.head_dim == 64 ? launch_merge<bf16_t, 64>(a, st) : launch_merge<bf16_t, 128>(a, st);
    return d.head_dim == 64 ? launch_merge<float, 64>(a, st) : launch_merge<float, 128>(a, st);
}
