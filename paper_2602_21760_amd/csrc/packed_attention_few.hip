// Attention over packed batches for at most 16 rows a block (single new tokens, their heads of a group as rows), bf16, head_dim 64 or 128.
//
// Bound by memory: every key and value is read once, with 8 multiply-adds a byte at most, one for each of 16 rows and 2 bytes (64 caches of 100 to 8000 keys, 8 heads of 128, 368 MB: 5.1 TB/s, and 5.6 us for the join; without
// cuts, 215 caches of 3000: 5.6 TB/s).  So nothing is shared between waves: a workgroup of 4
// waves owns the rows of one (sequence, key head) and a part of its keys, wave w takes the 32-key tiles w, w + 4, ... of it and streams them without a
// barrier through an LDS tile of its own each for keys and values: the fragments of a tile go to registers at once, and the next tile's copy into the same
// place is under way during this tile's arithmetic.  (Keys loaded straight to registers, 64 bytes of a row per instruction, reach 10 % less bandwidth.)  Running maximum and normaliser per wave, in fp32; probabilities are rounded to bf16 for the
// product with the values, and the normaliser is the sum of the rounded ones, as where blocks have many rows; the four partial results are joined in LDS, in a
// fixed order, and those of a sequence's parts by a second kernel.
//
// Caches are of all lengths, so workgroups are numbered by pieces of part_keys keys (as blocks of rows are elsewhere, see packed_find): a launch holds
// at most one workgroup without work per sequence and head, and long sequences are spread over as many workgroups as they have pieces.
#include "packed_attention.h"

namespace {

constexpr int BQ = kPackedRowsFew;
constexpr int BKV = 32;
constexpr int WAVES = 4;
constexpr float RESCALE_LOG2 = 8.0f;

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef void __attribute__((address_space(3)))* lptr_t;

template <int D> __device__ __forceinline__ int swz(int r) { return D == 64 ? (r & 6) | ((r >> 3) & 1) : ((r & 7) << 1) | ((r >> 3) & 1); }

// At most N of the wave's memory requests are outstanding: everything older has landed.
template <int N> __device__ __forceinline__ void memory_wait() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }
__device__ __forceinline__ void lds_done() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// K fragments of a tile (key tile kt, 32-feature step ks): LDS reads and the wait for them, through which every result passes.
template <int D>
__device__ __forceinline__ void k_fragments(unsigned at, bf16x8 (&kf)[2][D / 32]) {
#pragma unroll
    for (int ks = 0; ks < D / 32; ks++) {
        asm volatile("ds_read_b128 %0, %1 offset:0" : "=v"(kf[0][ks]) : "v"(at ^ (ks * 64u)));
        asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(kf[1][ks]) : "v"(at ^ (ks * 64u)), "i"(16 * D * 2));
    }
#pragma unroll
    for (int ks = 0; ks < D / 32; ks += 2)
        asm volatile("s_waitcnt lgkmcnt(%4)" : "+v"(kf[0][ks]), "+v"(kf[1][ks]), "+v"(kf[0][ks + 1]), "+v"(kf[1][ks + 1]) : "n"(2 * (D / 32 - 2 - ks)) : "memory");
}

// V^T fragments of a tile, all feature tiles: transposing LDS reads and the wait for them, through which every result passes.
template <int D>
__device__ __forceinline__ void v_fragments(unsigned at, bf16x4 (&vh)[D / 16][2]) {
#pragma unroll
    for (int dt = 0; dt < D / 16; dt++) {
        asm volatile("ds_read_b64_tr_b16 %0, %1 offset:0" : "=v"(vh[dt][0]) : "v"(at ^ (dt * 32u)));
        asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2" : "=v"(vh[dt][1]) : "v"(at ^ (dt * 32u)), "i"(16 * D * 2));
    }
#pragma unroll
    for (int dt = 0; dt < D / 16; dt += 4)
        asm volatile("s_waitcnt lgkmcnt(%8)"
                     : "+v"(vh[dt][0]), "+v"(vh[dt][1]), "+v"(vh[dt + 1][0]), "+v"(vh[dt + 1][1]), "+v"(vh[dt + 2][0]), "+v"(vh[dt + 2][1]), "+v"(vh[dt + 3][0]), "+v"(vh[dt + 3][1])
                     : "n"(2 * (D / 16 - 4 - dt)) : "memory");
}

// The piece-th piece of up to 64 sequences: all pieces of part_keys keys, then what is left of every sequence, the longest quarters first: the short ones fill the end of a launch of several rounds
// (24 caches of 7200 to 8000 keys, 8 heads of 128: 153 us in the order of the sequences, 145 so; launches of one round lose 0.4 us and take that order).  Lane s
// holds sequence s.  Fills in the sequence's rows and the part (-1: there are fewer pieces).
__device__ __forceinline__ void piece_in_order(const PackedAttnArgs& a, int piece, PackedUnit& u) {
    const int lane = threadIdx.x % 64;
    const PackedUnit lanes = packed_lanes(a);
    const int full = packed_div(lanes.n_k, a.by_piece), rest = lanes.n_k - full * a.part_keys;
    int end = full;              // full pieces up to and with this sequence
#pragma unroll
    for (int i = 1; i < 64; i <<= 1) {
        const int below = __shfl_up(end, i, 64);
        end += lane >= i ? below : 0;
    }
    const int all = __builtin_amdgcn_readlane(end, 63);
    int s, part;
    if (piece < all) {
        s = __popcll(__ballot(end <= piece));
        part = piece - __builtin_amdgcn_readlane(end - full, s);
    } else {
        const int left = piece - all;
        u.part = -1;
        if (left >= a.sequences) return;
        const int size = lane < a.sequences ? (int)((unsigned)rest * 4u / (unsigned)a.part_keys) : -1;      // (rest < 2^30)
        int before = 0, rank = 0;
#pragma unroll
        for (int c = 3; c >= 0; c--) {
            const unsigned long long these = __ballot(size == c);
            const int rank_here = before + __builtin_amdgcn_mbcnt_hi((unsigned)(these >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)these, 0u));
            rank = size == c ? rank_here : rank;
            before += __popcll(these);
        }
        s = __builtin_ctzll(__ballot(size >= 0 && rank == left));
        part = __builtin_amdgcn_readlane(rest > 0 || lanes.n_k == 0 ? full : -1, s);
    }
    packed_take(lanes, s, u);
    u.part = part;
}

template <int D, bool PRE>
__global__ __launch_bounds__(256, D == 64 ? 4 : 2) void packed_attention_few_kernel(PackedAttnArgs a) {
    constexpr int ROWB = D * 2, TILE_BYTES = BKV * ROWB, SLOTS = ROWB / 16, CHUNK_ROWS = 1024 / ROWB, CHUNKS = TILE_BYTES / 1024;
    constexpr int KS = D / 32, DT = D / 16;
    __shared__ __attribute__((aligned(2 * TILE_BYTES))) unsigned char smem[WAVES][2][TILE_BYTES];    // a wave's keys and values; later its 16 x D results
    __shared__ float part_ml[WAVES][2][BQ];
    PackedUnit u = {};
    // XCD x serves the key heads = x mod gcd(8, k_heads), see packed_unit()
    const unsigned id = packed_group_id();
    const int xcd = (int)(id % 8), of_head = packed_div((int)(id / 8), a.by_heads), piece = of_head * a.xcd_share + (xcd >> a.xcd_shift);
    if (piece >= a.pieces) return;
    u.head = (xcd & (a.xcd_heads - 1)) + a.xcd_heads * ((int)(id / 8) - of_head * (a.k_heads >> a.xcd_shift));
    if (a.rests_last) {
        piece_in_order(a, piece, u);
    } else {
        u.part = piece - packed_find<true>(a, piece, u, [&](int k0) { return packed_div(k0, a.by_piece); });
    }
    const int rows = u.n_q * a.group, parts = rows <= BQ ? packed_div(u.n_k + a.part_keys - 1, a.by_piece) : 1;
    if (rows == 0 || u.part < 0 || u.part >= max(parts, 1)) return;
    const int lane = threadIdx.x % 64, l16 = lane % 16, q4 = lane / 16;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);

    const char* kp = static_cast<const char*>(a.k) + (size_t)u.k0 * a.k_token + (size_t)u.head * a.k_head;
    const char* vp = static_cast<const char*>(a.v) + (size_t)u.k0 * a.v_token + (size_t)u.head * a.v_head;
    // slot s of row r of a tile holds feature vector s ^ swz(r); rows behind the last key are copies of it
    const int r0 = lane / SLOTS, slot = (lane % SLOTS) ^ swz<D>(r0);
    auto issue = [&](const char* p, size_t token, int t, unsigned char* dst0) {
        const int left = u.n_k - t * BKV, stride = (int)token;
        const __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc((void*)(p + (size_t)t * BKV * token), 0, (min(left, BKV) - 1) * stride + ROWB, 0x00020000);
#pragma unroll
        for (int c = 0; c < CHUNKS; c++) {
            const int r = min(r0 + c * CHUNK_ROWS, left - 1), off = r * stride + (slot ^ swz<D>(c * CHUNK_ROWS)) * 16;
            unsigned char* dst = dst0 + c * 1024;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (lptr_t)dst, 16, off, 0, 0, 0);
        }
    };

    const int kq = (q4 >> 1) | ((q4 & 1) << 1);      // which 8 of a step's 32 features the lane holds (lanes i and i + 32 take neighbouring slots)
    const int v_key = 4 * q4 + l16 / 4;
    const unsigned lds0 = (unsigned)(size_t)(lptr_t)&smem[wave][0][0];
    const float c = PRE ? 1.f : a.scale * 1.4426950408889634f;
    // (more than 16 rows only where a sequence has more queries than the caller said: then the part is all of the keys, block by block)
    for (u.row0 = 0; u.row0 < rows; u.row0 += BQ) {
        u.rows = min(rows - u.row0, BQ);
        if (u.row0 > 0) __syncthreads();       // everyone is done with the last block's results
        const int row = u.row0 + min(l16, u.rows - 1), tok = packed_div(row, a.by_group), last = packed_last_key(a, u, tok);
        bf16x8 qf[KS];
        {
            const char* qp = static_cast<const char*>(a.q) + (size_t)(u.q0 + tok) * a.q_token + (size_t)(u.head * a.group + row - tok * a.group) * a.q_head;
#pragma unroll
            for (int ks = 0; ks < KS; ks++) qf[ks] = *reinterpret_cast<const bf16x8*>(qp + ks * 64 + kq * 16);
        }
        const int block_min = packed_last_key(a, u, packed_div(u.row0, a.by_group)), block_max = packed_last_key(a, u, packed_div(u.row0 + u.rows - 1, a.by_group));
        const int part_tiles = a.part_keys / BKV, nt = (block_max + BKV) / BKV;
        const int t_begin = parts > 1 ? min(u.part * part_tiles, nt) : 0, t_end = parts > 1 ? min(t_begin + part_tiles, nt) : nt;

        float m_run = -__builtin_inff(), l_run = 0.f;        // l: over the lane's own keys
        f32x4 o[DT];
#pragma unroll
        for (int dt = 0; dt < DT; dt++) o[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
        const unsigned kb = lds0 + l16 * ROWB + ((kq ^ swz<D>(l16)) * 16);
        const unsigned vb = lds0 + TILE_BYTES + v_key * ROWB + (((l16 % 4) / 2) ^ swz<D>(v_key)) * 16 + (l16 % 2) * 8;

        int t = t_begin + wave;
        if (t < t_end) {
            issue(kp, a.k_token, t, smem[wave][0]);
            issue(vp, a.v_token, t, smem[wave][1]);
        }
        for (; t < t_end; t += WAVES) {
            const bool more = t + WAVES < t_end;
            bf16x8 kf[2][KS];        // [key tile][32-feature step]
            memory_wait<CHUNKS>();   // the keys have landed; the values may be on their way
            k_fragments<D>(kb, kf);
            if (more) issue(kp, a.k_token, t + WAVES, smem[wave][0]);
            f32x4 s[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};      // keys 16 kt + 4 q4 + i of row l16
#pragma unroll
            for (int ks = 0; ks < KS; ks++)
#pragma unroll
                for (int kt = 0; kt < 2; kt++) s[kt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[kt][ks], qf[ks], s[kt], 0, 0, 0);
            const bool masked = t * BKV + BKV - 1 > block_min;
            if (masked) {
                const int seen = last - t * BKV - 4 * q4;
#pragma unroll
                for (int kt = 0; kt < 2; kt++)
#pragma unroll
                    for (int i = 0; i < 4; i++)
                        if (kt * 16 + i > seen) s[kt][i] = -__builtin_inff();
            }
            // the reference only advances when a score exceeds it by more than 2^RESCALE_LOG2; it is the same for the four lanes of a row
            float mx = fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])), fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3])));
            if (__any((mx - m_run) * c > RESCALE_LOG2)) {
                mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
                mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
                const bool grow = (mx - m_run) * c > RESCALE_LOG2;
                const float corr = grow ? __builtin_amdgcn_exp2f((m_run - mx) * c) : 1.f;
                m_run = grow ? mx : m_run;
                l_run *= corr;
#pragma unroll
                for (int dt = 0; dt < DT; dt++) o[dt] *= corr;
            }
            const float mc = m_run == -__builtin_inff() ? 0.f : m_run * c;
            bf16x8 pb;
#pragma unroll
            for (int kt = 0; kt < 2; kt++)
#pragma unroll
                for (int i = 0; i < 4; i++) pb[4 * kt + i] = (bf16_t)__builtin_amdgcn_exp2f(fmaf(s[kt][i], c, -mc));
            const bf16x2 ones = {(bf16_t)1.0f, (bf16_t)1.0f};
#pragma unroll
            for (int j = 0; j < 8; j += 2) {
                const bf16x2 pr = {pb[j], pb[j + 1]};
                l_run = __builtin_amdgcn_fdot2_f32_bf16(pr, ones, l_run, false);
            }
            if (more) memory_wait<CHUNKS>();       // the values have landed; the next keys may be on their way
            else memory_wait<0>();
            bf16x4 vh[DT][2];
            v_fragments<D>(vb, vh);
            bool odd = false;
            if (masked) {
                unsigned any = 0;
#pragma unroll
                for (int dt = 0; dt < DT; dt++)
#pragma unroll
                    for (int j = 0; j < 2; j++) {
                        const u32x2 w = __builtin_bit_cast(u32x2, vh[dt][j]);
                        any |= odd_bits_bf16(w[0]) | odd_bits_bf16(w[1]);
                    }
                odd = __any(any != 0);
                if (odd) {
#pragma unroll
                    for (int dt = 0; dt < DT; dt++) {
                        keep_finite(vh[dt][0]);
                        keep_finite(vh[dt][1]);
                    }
                }
            }
            if (odd) {               // a hidden key's infinity or NaN reaches no row, a seen one's those that see it
#pragma unroll 1
                for (int key = 0; key < BKV; key++) {
                    const unsigned seen = t * BKV + key <= last ? ~0u : 0u;
#pragma unroll
                    for (int dt = 0; dt < DT; dt++)
                        o[dt] += only_odd(*(const u32x2 __attribute__((address_space(3)))*)(lds0 + TILE_BYTES + key * ROWB + (((2 * dt + q4 / 2) ^ swz<D>(key)) * 16) + (q4 % 2) * 8), seen);
                }
                lds_done();
            }
            if (more) issue(vp, a.v_token, t + WAVES, smem[wave][1]);
#pragma unroll
            for (int dt = 0; dt < DT; dt++)
                o[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(bf16x8{vh[dt][0][0], vh[dt][0][1], vh[dt][0][2], vh[dt][0][3], vh[dt][1][0], vh[dt][1][1], vh[dt][1][2], vh[dt][1][3]}, pb, o[dt], 0, 0, 0);
        }

        // join of the waves, in order
        l_run += __shfl_xor(l_run, 16, 64);
        l_run += __shfl_xor(l_run, 32, 64);
        float* mine = reinterpret_cast<float*>(&smem[wave][0][0]);       // [16 rows][D]
        if (q4 == 0) {
            part_ml[wave][0][l16] = m_run;
            part_ml[wave][1][l16] = l_run;
        }
#pragma unroll
        for (int dt = 0; dt < DT; dt++) *reinterpret_cast<f32x4*>(mine + l16 * D + 16 * dt + 4 * q4) = o[dt];
        __syncthreads();
        for (int i = threadIdx.x; i < u.rows * (D / 4); i += 256) {
            const int r = i / (D / 4), f = i % (D / 4) * 4;
            float m_all = -__builtin_inff();
#pragma unroll
            for (int p = 0; p < WAVES; p++)
                if (part_ml[p][1][r] != 0.f) m_all = fmaxf(m_all, part_ml[p][0][r]);
            float l = 0.f;
            f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int p = 0; p < WAVES; p++) {
                const float mp = part_ml[p][0][r], lp = part_ml[p][1][r];
                if (lp == 0.f) continue;
                const float w = mp == m_all ? 1.f : __builtin_amdgcn_exp2f((mp - m_all) * c);
                l = fmaf(lp, w, l);
                const f32x4 y = *reinterpret_cast<const f32x4*>(reinterpret_cast<const float*>(&smem[p][0][0]) + r * D + f);
#pragma unroll
                for (int e = 0; e < 4; e++) x[e] = fmaf(y[e], w, x[e]);
            }
            const int rr = u.row0 + r, tk = packed_div(rr, a.by_group), head = u.head * a.group + (rr - tk * a.group);
            if (parts > 1) {
                const size_t place = (size_t)(packed_div(u.k0, a.by_piece) + u.sequence + u.part), at = (place * a.k_heads + u.head) * BQ + r;     // (the piece's number)
                if (f == 0) *reinterpret_cast<f32x2*>(a.part + packed_piece_rows(a.pieces, a.k_heads) * D + at * 2) = f32x2{m_all, l};
                *reinterpret_cast<f32x4*>(a.part + at * D + f) = x;
            } else {
                const float inv = l == 0.f ? 0.f : 1.0f / l;
                *reinterpret_cast<bf16x4*>(static_cast<char*>(a.o) + (size_t)(u.q0 + tk) * a.o_token + (size_t)head * a.o_head + 2 * f) =
                    bf16x4{(bf16_t)(x[0] * inv), (bf16_t)(x[1] * inv), (bf16_t)(x[2] * inv), (bf16_t)(x[3] * inv)};
            }
        }
    }
}

// Joins the pieces of a sequence that has several: with references m_p, normalisers l_p and accumulators o_p a row is sum_p o_p w_p / sum_p l_p w_p, w_p =
// 2^((m_p - M) c), M = max m_p over the pieces that the row sees.  A workgroup per row: thread (g, f) sums features 4 f .. 4 f + 3 of the pieces g, g + G, ...,
// the G sums are added in order.  Bound by latency, so up to 64 pieces all loads are requested before the first weight is known.
template <int D>
__global__ __launch_bounds__(256) void packed_join_kernel(PackedAttnArgs a, float c) {
    constexpr int F = D / 4, G = 256 / F, U = 64 / G;
    __shared__ f32x4 sums[G][F];
    __shared__ float weight[64];
    const PackedUnit u = packed_unit<1>(a, packed_group_id());
    if (u.rows == 0 || u.n_q * a.group > BQ) return;
    const int parts = packed_div(u.n_k + a.part_keys - 1, a.by_piece);
    if (parts <= 1) return;              // (written already)
    const int tid = threadIdx.x, f = tid % F, g = tid / F;
    const int row = u.row0, tok = packed_div(row, a.by_group), head = u.head * a.group + (row - tok * a.group);
    const size_t at = ((size_t)(packed_div(u.k0, a.by_piece) + u.sequence) * a.k_heads + u.head) * BQ + row, step = (size_t)a.k_heads * BQ;
    const f32x2* ml = reinterpret_cast<const f32x2*>(a.part + packed_piece_rows(a.pieces, a.k_heads) * D) + at;
    const float* o = a.part + at * D + 4 * f;
    f32x4 x = {0.f, 0.f, 0.f, 0.f};
    float m_all = -__builtin_inff(), l_all = 0.f;       // of the rounds so far, the same in all threads
    for (int p0 = 0; p0 < parts; p0 += 64) {
        f32x4 v[U];
#pragma unroll
        for (int j = 0; j < U; j++) v[j] = *reinterpret_cast<const f32x4*>(o + min(p0 + g + j * G, parts - 1) * step * D);
        const int mine = p0 + tid % 64;
        f32x2 e = ml[min(mine, parts - 1) * step];
        const bool any = mine < parts && e[1] != 0.f;
        const float m_new = fmaxf(m_all, wave_max(any ? e[0] : -__builtin_inff()));
        const float w = !any ? 0.f : e[0] == m_new ? 1.f : __builtin_amdgcn_exp2f((e[0] - m_new) * c);
        const float old = m_all == m_new ? 1.f : __builtin_amdgcn_exp2f((m_all - m_new) * c);
        l_all = l_all * old + wave_sum(any ? e[1] * w : 0.f);
        m_all = m_new;
        if (p0 > 0) __syncthreads();
        if (tid < 64) weight[tid] = w;
        __syncthreads();
        x *= old;
#pragma unroll
        for (int j = 0; j < U; j++) {
            if (p0 + g + j * G >= parts) continue;
            const float wj = weight[g + j * G];
#pragma unroll
            for (int i = 0; i < 4; i++) x[i] = fmaf(v[j][i], wj, x[i]);
        }
    }
    sums[g][f] = x;
    __syncthreads();
    if (g > 0) return;
#pragma unroll
    for (int j = 1; j < G; j++) x += sums[j][f];
    x *= l_all == 0.f ? 0.f : 1.0f / l_all;
    *reinterpret_cast<bf16x4*>(static_cast<char*>(a.o) + (size_t)(u.q0 + tok) * a.o_token + (size_t)head * a.o_head + 8 * f) = bf16x4{(bf16_t)x[0], (bf16_t)x[1], (bf16_t)x[2], (bf16_t)x[3]};
}

template <int D, bool PRE>
int launch(PackedAttnArgs& a, hipStream_t st) {
    const size_t total = 8 * (size_t)(a.k_heads / a.xcd_heads) * ((a.pieces + a.xcd_share - 1) / a.xcd_share);
    a.by_heads = packed_divisor((unsigned)(a.k_heads / a.xcd_heads));
    {
        HybTraceScope trace("packed_attention_few", "byte", 4.0 * D * ((double)a.total_q * a.q_heads + (double)a.total_k * a.k_heads), st);
        hipLaunchKernelGGL((packed_attention_few_kernel<D, PRE>), packed_grid_of(total), dim3(256), 0, st, a);
    }
    const int rc = hyb_check_launch("packed_attention_few");
    if (rc || a.pieces <= a.sequences) return rc;       // no sequence can have two pieces
    HybTraceScope trace("packed_attention_join", "byte", 4.0 * D * (double)a.pieces * a.q_heads, st);
    const dim3 grid = packed_grid(a);
    hipLaunchKernelGGL((packed_join_kernel<D>), grid, dim3(256), 0, st, a, PRE ? 1.f : a.scale * 1.4426950408889634f);
    return hyb_check_launch("packed_attention_join");
}

}  // namespace

int hyb_launch_packed_attention_few(PackedAttnArgs& a, int head_dim, hipStream_t st) {
    if (head_dim == 64) return a.prescaled ? launch<64, true>(a, st) : launch<64, false>(a, st);
    return a.prescaled ? launch<128, true>(a, st) : launch<128, false>(a, st);
}
