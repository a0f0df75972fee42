// Attention over packed batches for gfx950, bf16 operands, head_dim 64 or 128: a streaming softmax over key tiles, scores never stored.
//
// A workgroup of 4 waves owns 128 rows (queries x heads of a group, see packed_attention.h) of one (sequence, key head), each wave 32 of
// them (two tiles of 16).  Keys and values come 64 (head_dim 128: 32) at a time through double-buffered LDS tiles of 8 KB by 16-byte direct-to-LDS copies, rows unpadded
// with their 16-byte slots XOR-swizzled.  Both contractions run on v_mfma_f32_16x16x32_bf16 in transposed form, S^T = K Q^T and
// O^T += V^T P^T: lane (l16 = lane % 16, q4 = lane / 16) of an accumulator tile holds column l16 and rows 4 q4 .. 4 q4 + 3, so all scores of a
// lane belong to ONE row per 16-row tile, row sums are per-lane scalars plus two exchanges at the end, and the exponentiated scores of key tiles
// 2 s and 2 s + 1, rounded to bf16, are the B operand of the second contraction as they lie (the order of a contraction's index does not
// matter as long as both operands agree: k = 4 q4 + i of key tile 2 s, then of 2 s + 1).
//
// Softmax in fp32, base 2.  A workgroup first sums 2^(c score) without a reference maximum (c = scale x log2 e; 1 for queries that carry it);
// that is the softmax as long as every row's sum lies in [2^-32, 2^64] and the sums over values are finite.  If a row's are not, the workgroup starts over with a running maximum.
// (Products of a probability and a value below 2^-149 are lost: with a sum of 2^-32 a result is off by up to 2^-118 a key, with one of 2^-64 by 2^-86; and probabilities below 2^-126, which
// is 2^-94 of such a sum.)
// Probabilities are rounded to bf16 for the second contraction, whose instruction takes both operands in one type (in fp32 it has a ninth of the rate), and the normaliser is the sum of the
// rounded ones, so that a mean of equal values is that value.  This rounding is all that tells the results from rounded exact ones: 1.1e-3 to 1.6e-3 relative L2 before the results' own
// rounding to bf16 (1.6e-3), 1.9e-3 to 2.3e-3 with it.
//
// Masks: the last key that a row sees is one number per row (causal, or the end of the sequence); only tiles in which a wave's rows differ from
// "all of the tile" compare against it.  A probability of 0 does not keep an infinity or NaN of a hidden key's value out of an MFMA.  The first attempt lets them in; if a
// result is not finite, the workgroup starts over in the same way as for sums out of range, and the second attempt searches every tile that not all rows see, zeroes such
// values in the fragments and adds them to the rows that do see them.  (The search in the first attempt takes 3 to 9 % of launches over short sequences.)
//
// Bound by what the matrix cores sustain beside the softmax (16717 tokens, 24 heads of 64: 1180 TFLOP/s; 8192 tokens, 32 / 8 heads of 128: 1300, causal 1255) and, for short sequences, by the 7 us
// that a workgroup takes before and after its key loop (24 prompts of 33 to 4000: 2 to find its unit, 2 for the first tile, 3 for the result, 24 for the keys; 880 TFLOP/s): 4 workgroups a CU
// at head_dim 64, 3 at 128.  (64 keys a tile at head_dim 128 take 200 registers, 2 workgroups a CU: 2 % slower on
// 8192 tokens, 8 % on prompts of 33 to 4000, 14 % on prompts of 300.  Workgroups that walk through several units, the next one's first tile under way, from a queue filled by a
// kernel before: as fast at head_dim 128, 20 % slower at 64.)
#include "packed_attention.h"

#include <type_traits>

namespace {

constexpr int BQ = kPackedRowsMfma;
constexpr float RESCALE_LOG2 = 8.0f;

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef void __attribute__((address_space(3)))* lptr_t;

template <int D> __device__ __forceinline__ int swz(int r) {
    // 128-byte rows: see attention_mfma.hip.  256-byte rows cover all banks: 16 rows (8 for the transposing reads, which take 32 bytes of a row) go to different slots.
    return D == 64 ? (r & 6) | ((r >> 3) & 1) : ((r & 7) << 1) | ((r >> 3) & 1);
}

__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}

// Transposing LDS reads of the V^T fragments of 32 output features (two 16-feature tiles, two 32-key steps of two reads each).  Written as asm so that they can be issued
// ahead of their use: a wait that the compiler places before such a read through its builtin also waits for the next tile's copies.  Every result goes
// through lds_wait(), which stands between these reads and their use and keeps the registers in use until they are written.  (That nothing, a spill or a copy, touches the registers before is
// looked up in the compiler's listing by the build.)
template <int D, int PS>
__device__ __forceinline__ void v_reads(unsigned at, bf16x4 (&vh)[2][PS][2]) {
    constexpr int ROWB = D * 2;
#pragma unroll
    for (int dd = 0; dd < 2; dd++)
#pragma unroll
        for (int ks = 0; ks < PS; ks++)
#pragma unroll
            for (int half = 0; half < 2; half++)
                asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2" : "=v"(vh[dd][ks][half]) : "v"(dd ? at ^ 32u : at), "i"((ks * 32 + half * 16) * ROWB));
}
// Waits until at most YOUNGER LDS reads are outstanding; reads complete in order.
template <int YOUNGER>
__device__ __forceinline__ void lds_wait(bf16x4 (&vh)[2][2][2]) {
    asm volatile("s_waitcnt lgkmcnt(%8)"
                 : "+v"(vh[0][0][0]), "+v"(vh[0][0][1]), "+v"(vh[0][1][0]), "+v"(vh[0][1][1]), "+v"(vh[1][0][0]), "+v"(vh[1][0][1]), "+v"(vh[1][1][0]), "+v"(vh[1][1][1])
                 : "n"(YOUNGER));
}
template <int YOUNGER>
__device__ __forceinline__ void lds_wait(bf16x4 (&vh)[2][1][2]) {
    asm volatile("s_waitcnt lgkmcnt(%4)" : "+v"(vh[0][0][0]), "+v"(vh[0][0][1]), "+v"(vh[1][0][0]), "+v"(vh[1][0][1]) : "n"(YOUNGER));
}

// The same for a K fragment: requested, and awaited with at most YOUNGER reads outstanding.
template <int OFFSET>
__device__ __forceinline__ void k_read(unsigned at, bf16x8& f) { asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(f) : "v"(at), "i"(OFFSET)); }
template <int YOUNGER>
__device__ __forceinline__ void k_wait(bf16x8& f) { asm volatile("s_waitcnt lgkmcnt(%1)" : "+v"(f) : "n"(YOUNGER)); }

// f(0), f(1), ... f(N - 1) with the index as a type
template <int N, int I = 0, typename F>
__device__ __forceinline__ void unrolled(F f) {
    if constexpr (I < N) {
        f(std::integral_constant<int, I>{});
        unrolled<N, I + 1>(f);
    }
}

// Everything that makes these values stands before, everything that uses them behind this place.
template <typename V, int N>
__device__ __forceinline__ void keep_order(V (&x)[N][2]) {
#pragma unroll
    for (int i = 0; i < N; i++) asm volatile("" : "+v"(x[i][0]), "+v"(x[i][1]));
}

// Stands between MFMAs and inline asm that takes their results: a vector instruction may come 8 wait states after a 16x16x32 MFMA, which the compiler sees to for its own instructions but
// not for those in asm.
__device__ __forceinline__ void mfma_wait(f32x4 (&x)[4][2]) {
    asm volatile("s_nop 7" : "+v"(x[0][0]), "+v"(x[0][1]), "+v"(x[1][0]), "+v"(x[1][1]), "+v"(x[2][0]), "+v"(x[2][1]), "+v"(x[3][0]), "+v"(x[3][1]));
}
__device__ __forceinline__ void mfma_wait(f32x4 (&x)[2][2]) { asm volatile("s_nop 7" : "+v"(x[0][0]), "+v"(x[0][1]), "+v"(x[1][0]), "+v"(x[1][1])); }

// The lane's index from an instruction the compiler cannot trace back: what rare paths and the epilogue derive from it is not kept in registers over the key loop.
__device__ __forceinline__ int lane_again() {
    int lane = __builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u));
    asm volatile("" : "+v"(lane));
    return lane;
}

template <int D, bool PRE>
__global__ __launch_bounds__(256, D == 64 ? 4 : 3) void packed_attention_kernel(PackedAttnArgs a) {
    constexpr int BKV = packed_tile_keys(D), KT = BKV / 16, PS = BKV / 32;      // keys of a tile; 16-key tiles; 32-key steps of the second contraction
    constexpr int ROWB = D * 2, TILE_BYTES = BKV * ROWB, SLOTS = ROWB / 16;
    constexpr int CHUNK_ROWS = 1024 / ROWB, CHUNKS = BKV / CHUNK_ROWS / 4;      // rows of a 1 KB copy; copies per wave, operand and tile
    constexpr int KS = D / 32, DT = D / 16, VG = D / 32;
    constexpr unsigned OTHER = 2 * TILE_BYTES;                                  // XOR to the other buffer
    // [buffer][K tile | V tile]
    __shared__ __attribute__((aligned(4 * TILE_BYTES))) unsigned char smem[2][2 * TILE_BYTES];
    __shared__ int row_last[BQ];         // last key that each row sees (read in masked tiles only)
    __shared__ int wave_flags[4];

    __builtin_amdgcn_s_setprio(3);           // before the tiles, beside waves that have been at 1 in theirs (finding the unit, 24 sequences: 2.8 us without, 2.1 so)
    const PackedUnit u = packed_unit<BQ, true>(a, packed_group_id());
    if (u.rows == 0) return;
    const int lane = threadIdx.x % 64;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int l16 = lane % 16, q4 = lane / 16;
    const int kq = (q4 >> 1) | ((q4 & 1) << 1);      // which 8 of a step's 32 features the lane holds (lanes i and i + 32 take neighbouring slots)

    // the lane's rows, one per 16-row tile (rows behind the block's last are copies of it, never stored)
    bf16x8 qf[2][KS];
#pragma unroll
    for (int qt = 0; qt < 2; qt++) {
        const int row = u.row0 + min(wave * 32 + qt * 16 + l16, u.rows - 1);
        const int t = packed_div(row, a.by_group), g = row - t * a.group;
        if (q4 == 0) row_last[wave * 32 + qt * 16 + l16] = packed_last_key(a, u, t);
        const char* qp = static_cast<const char*>(a.q) + (size_t)(u.q0 + t) * a.q_token + (size_t)(u.head * a.group + g) * a.q_head;
#pragma unroll
        for (int ks = 0; ks < KS; ks++) qf[qt][ks] = *reinterpret_cast<const bf16x8*>(qp + ks * 64 + kq * 16);
    }
    // the wave's rows see at least the keys 0 .. wave_min and at most 0 .. wave_max, the block's rows at most 0 .. block_max
    const bool active = wave * 32 < u.rows;
    const int wave_min = packed_last_key(a, u, packed_div(u.row0 + min(wave * 32, u.rows - 1), a.by_group));
    const int wave_max = active ? packed_last_key(a, u, packed_div(u.row0 + min(wave * 32 + 31, u.rows - 1), a.by_group)) : -1;
    const int block_max = packed_last_key(a, u, packed_div(u.row0 + u.rows - 1, a.by_group));

    const int nt = (block_max + BKV) / BKV, part_tiles = packed_part_tiles(a, nt, BKV);        // (block_max == -1: no tile)
    const int t_begin = min(u.part * part_tiles, nt), t_end = min(t_begin + part_tiles, nt);
    // Tiles t_begin .. plain_end - 1 are seen whole by all rows and followed by a whole tile of BKV keys: a loop of its own, which holds no masks in registers.
    const int block_min = packed_last_key(a, u, packed_div(u.row0, a.by_group));
    const int plain_end = min(min((block_min + 1) / BKV, u.n_k / BKV - 1), t_end - 1);

    // Tile copy: lane i of a 1 KB chunk fills slot i % SLOTS of row i / SLOTS with feature vector slot ^ swz(row) (the swizzle is the same for a wave's
    // chunks).  The tile's first row is in the resource (64-bit), so an offset never exceeds a tile.  Only the ragged last tile has its rows clamped.
    const char* kp = static_cast<const char*>(a.k) + (size_t)u.k0 * a.k_token + (size_t)u.head * a.k_head;
    const char* vp = static_cast<const char*>(a.v) + (size_t)u.k0 * a.v_token + (size_t)u.head * a.v_head;
    const int k_token = (int)a.k_token, v_token = (int)a.v_token;
    const int r0 = wave * CHUNK_ROWS + lane / SLOTS, slot_off = ((lane % SLOTS) ^ swz<D>(r0)) * 16;
    const int k_off = r0 * k_token + slot_off, v_off = r0 * v_token + slot_off;
    auto issue = [&](int t, int buf, auto whole_tag) {     // whole: the tile has BKV keys
        const int left = u.n_k - t * BKV;
        const __amdgpu_buffer_rsrc_t k_rsrc = __builtin_amdgcn_make_buffer_rsrc((void*)(kp + (size_t)t * BKV * a.k_token), 0, (min(left, BKV) - 1) * k_token + ROWB, 0x00020000);
        const __amdgpu_buffer_rsrc_t v_rsrc = __builtin_amdgcn_make_buffer_rsrc((void*)(vp + (size_t)t * BKV * a.v_token), 0, (min(left, BKV) - 1) * v_token + ROWB, 0x00020000);
        unsigned char* dst = smem[buf] + wave * 1024;
        if (decltype(whole_tag)::value || left >= BKV) {
#pragma unroll
            for (int c = 0; c < CHUNKS; c++) {
                __builtin_amdgcn_raw_ptr_buffer_load_lds(k_rsrc, (lptr_t)(dst + c * 4096), 16, k_off, c * 4 * CHUNK_ROWS * k_token, 0, 0);
                __builtin_amdgcn_raw_ptr_buffer_load_lds(v_rsrc, (lptr_t)(dst + c * 4096 + TILE_BYTES), 16, v_off, c * 4 * CHUNK_ROWS * v_token, 0, 0);
            }
        } else {
            const int ln = lane_again(), first = wave * CHUNK_ROWS + ln / SLOTS, so = ((ln % SLOTS) ^ swz<D>(first)) * 16;
#pragma unroll
            for (int c = 0; c < CHUNKS; c++) {
                const int row = min(first + c * 4 * CHUNK_ROWS, left - 1);
                __builtin_amdgcn_raw_ptr_buffer_load_lds(k_rsrc, (lptr_t)(dst + c * 4096), 16, row * k_token + so, 0, 0, 0);
                __builtin_amdgcn_raw_ptr_buffer_load_lds(v_rsrc, (lptr_t)(dst + c * 4096 + TILE_BYTES), 16, row * v_token + so, 0, 0, 0);
            }
        }
    };

    const float c = PRE ? 1.f : a.scale * 1.4426950408889634f;
    float m_run[2], l_run[2];
    f32x4 o[DT][2];      // [16-feature tile][row tile]: features 16 dt + 4 q4 .. + 3 of row 16 qt + l16
    auto clear = [&](float m) {
        m_run[0] = m_run[1] = m;
        l_run[0] = l_run[1] = 0.f;
#pragma unroll
        for (int dt = 0; dt < DT; dt++)
#pragma unroll
            for (int qt = 0; qt < 2; qt++) o[dt][qt] = f32x4{0.f, 0.f, 0.f, 0.f};
    };

    // LDS addresses of the fragments, one for K and one for V^T, in the buffer of the current tile; everything else is a constant XOR or offset
    const unsigned lds0 = (unsigned)(size_t)(lptr_t)&smem[0][0];
    const int v_key = 4 * q4 + l16 / 4;                                                     // transposing reads: 4 keys x 16 features per 16 lanes
    unsigned kb = lds0 + l16 * ROWB + ((kq ^ swz<D>(l16)) * 16);                            // + 64 ks by XOR, + 16 kt rows
    unsigned vb = lds0 + TILE_BYTES + v_key * ROWB + (((l16 % 4) / 2) ^ swz<D>(v_key)) * 16 + (l16 % 2) * 8;   // + 32 dt by XOR, + 16 keys

    // PLAIN: all of the block's rows see all of the tile, and the next tile is whole
    auto tile = [&](int t, int buf, auto direct_tag, auto plain_tag) {
        constexpr bool DIRECT = decltype(direct_tag)::value, PLAIN = decltype(plain_tag)::value;
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // this wave's part of tile t has landed
        __builtin_amdgcn_s_barrier();                      // everyone's has; and the other buffer is free again
        if (PLAIN || t + 1 < t_end) issue(t + 1, buf ^ 1, plain_tag);
        if (PLAIN ? !active : t * BKV > wave_max) return;  // none of the wave's rows sees this tile
        const bool masked = !PLAIN && t * BKV + BKV - 1 > wave_min;

        // S^T = K Q^T; the K fragments (step j / KT, key tile j % KT) flow through a ring of four reads that run ahead of the MFMAs
        bf16x8 ring[4];
        __builtin_amdgcn_s_setprio(1);
        auto k_frag = [&](auto j) { k_read<(j.value % KT) * 16 * ROWB>(kb ^ ((j.value / KT) * 64u), ring[j.value & 3]); };
        unrolled<4>(k_frag);
        f32x4 s[KT][2];   // [key tile][row tile]: keys 16 kt + 4 q4 .. + 3 of row 16 qt + l16
#pragma unroll
        for (int kt = 0; kt < KT; kt++)
#pragma unroll
            for (int qt = 0; qt < 2; qt++) s[kt][qt] = f32x4{0.f, 0.f, 0.f, 0.f};
        unrolled<KT * KS>([&](auto j) {
            constexpr int J = j.value;
            k_wait<(KT * KS - 1 - J < 3 ? KT * KS - 1 - J : 3)>(ring[J & 3]);
#pragma unroll
            for (int qt = 0; qt < 2; qt++) s[J % KT][qt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ring[J & 3], qf[qt][J / KT], s[J % KT][qt], 0, 0, 0);
            if constexpr (J + 4 < KT * KS) k_frag(std::integral_constant<int, J + 4>{});
        });

        bf16x4 vh[2][2][PS][2];   // [two groups of 32 features in flight][16-feature tile][32-key step][read]
        bool odd = false;        // infinities or NaN among the values of a tile that not all rows see (looked for in the second attempt only)
        if (masked) {
            const int ln = lane_again();
#pragma unroll
            for (int qt = 0; qt < 2; qt++) {
                const int seen = row_last[wave * 32 + qt * 16 + ln % 16] - t * BKV - 4 * (ln / 16);     // keys 16 kt + i > seen are hidden
#pragma unroll
                for (int kt = 0; kt < KT; kt++)
#pragma unroll
                    for (int i = 0; i < 4; i++)
                        if (kt * 16 + i > seen) s[kt][qt][i] = -__builtin_inff();
            }
            if constexpr (!DIRECT) {
                unsigned any = 0;
#pragma unroll 1
                for (int j = 0; j < TILE_BYTES / 1024; j++) {
                    const u32x4 x = *(const u32x4 __attribute__((address_space(3)))*)(lds0 + (buf ? OTHER : 0u) + TILE_BYTES + j * 1024 + ln * 16);
#pragma unroll
                    for (int e = 0; e < 4; e++) any |= odd_bits_bf16(x[e]);
                }
                odd = __any(any != 0);
            }
        }
        if constexpr (DIRECT) v_reads<D, PS>(vb, vh[0]);       // (the form with row maxima holds more values meanwhile and requests them after them)
        // the exponentiated scores of key tiles 2 ks, 2 ks + 1, rounded to bf16, are the B operand of 32-key step ks
        if constexpr (DIRECT && !PRE) {
#pragma unroll
            for (int kt = 0; kt < KT; kt++)
#pragma unroll
                for (int qt = 0; qt < 2; qt++) s[kt][qt] *= c;
            keep_order(s);
        }
        __builtin_amdgcn_s_setprio(0);     // a wave yields during its exponentials, so that they do not hold up another wave's MFMAs
        bf16x8 pb[PS][2];   // [32-key step][row tile]
        if constexpr (DIRECT) {
#pragma unroll
            for (int kt = 0; kt < KT; kt++)
#pragma unroll
                for (int qt = 0; qt < 2; qt++)
#pragma unroll
                    for (int i = 0; i < 4; i++) s[kt][qt][i] = __builtin_amdgcn_exp2f(s[kt][qt][i]);
            keep_order(s);
            __builtin_amdgcn_s_setprio(1);
#pragma unroll
            for (int kt = 0; kt < KT; kt++)
#pragma unroll
                for (int qt = 0; qt < 2; qt++)
#pragma unroll
                    for (int i = 0; i < 4; i++) pb[kt >> 1][qt][4 * (kt & 1) + i] = (bf16_t)s[kt][qt][i];
        } else {
            mfma_wait(s);
            float mx[2];
#pragma unroll
            for (int qt = 0; qt < 2; qt++) {
                float m0 = s[0][qt][0];
#pragma unroll
                for (int kt = 0; kt < KT; kt++) m0 = max3(max3(s[kt][qt][0], s[kt][qt][1], m0), s[kt][qt][2], s[kt][qt][3]);
                m0 = max3(m0, __shfl_xor(m0, 16, 64), m0);
                mx[qt] = max3(m0, __shfl_xor(m0, 32, 64), m0);
            }
            const bool grow0 = (mx[0] - m_run[0]) * c > RESCALE_LOG2, grow1 = (mx[1] - m_run[1]) * c > RESCALE_LOG2;   // (only hidden keys so far: -inf - -inf, false)
            if (__any(grow0 || grow1)) {
#pragma unroll
                for (int qt = 0; qt < 2; qt++) {
                    const bool grow = qt ? grow1 : grow0;
                    const float m_new = grow ? mx[qt] : m_run[qt];
                    const float corr = grow ? __builtin_amdgcn_exp2f((m_run[qt] - m_new) * c) : 1.f;
                    m_run[qt] = m_new;
                    l_run[qt] *= corr;
#pragma unroll
                    for (int dt = 0; dt < DT; dt++) o[dt][qt] *= corr;
                }
            }
#pragma unroll
            for (int qt = 0; qt < 2; qt++) {
                const float mc = m_run[qt] == -__builtin_inff() ? 0.f : m_run[qt] * c;
#pragma unroll
                for (int kt = 0; kt < KT; kt++)
#pragma unroll
                    for (int i = 0; i < 4; i++) pb[kt >> 1][qt][4 * (kt & 1) + i] = (bf16_t)__builtin_amdgcn_exp2f(fmaf(s[kt][qt][i], c, -mc));
            }
            keep_order(pb);
            __builtin_amdgcn_s_setprio(1);
            v_reads<D, PS>(vb, vh[0]);
        }

        // O^T += V^T P^T, 32 features at a time, the next 32 on their way
#pragma unroll
        for (int g = 0; g < VG; g++) {
            if (g + 1 < VG) {
                v_reads<D, PS>(vb ^ ((g + 1) * 64u), vh[(g + 1) & 1]);
                lds_wait<4 * PS>(vh[g & 1]);
            } else {
                lds_wait<0>(vh[g & 1]);
            }
            if (!DIRECT && odd) {
#pragma unroll
                for (int dd = 0; dd < 2; dd++)
#pragma unroll
                    for (int ks = 0; ks < PS; ks++) {
                        keep_finite(vh[g & 1][dd][ks][0]);
                        keep_finite(vh[g & 1][dd][ks][1]);
                    }
            }
#pragma unroll
            for (int dd = 0; dd < 2; dd++)
#pragma unroll
                for (int ks = 0; ks < PS; ks++) {
                    const bf16x4 lo = vh[g & 1][dd][ks][0], hi = vh[g & 1][dd][ks][1];
                    const bf16x8 vf = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
#pragma unroll
                    for (int qt = 0; qt < 2; qt++) o[2 * g + dd][qt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pb[ks][qt], o[2 * g + dd][qt], 0, 0, 0);
                }
            if (g == 0) {        // the normaliser, from the rounded probabilities, beside the MFMAs
                const bf16x2 ones = {(bf16_t)1.0f, (bf16_t)1.0f};
#pragma unroll
                for (int ks = 0; ks < PS; ks++)
#pragma unroll
                    for (int qt = 0; qt < 2; qt++)
#pragma unroll
                        for (int j = 0; j < 8; j += 2) {
                            const bf16x2 pr = {pb[ks][qt][j], pb[ks][qt][j + 1]};
                            l_run[qt] = __builtin_amdgcn_fdot2_f32_bf16(pr, ones, l_run[qt], false);
                        }
            }
        }
        if (!DIRECT && odd) {
            const int ln = lane_again();
#pragma unroll 1
            for (int key = 0; key < BKV; key++) {
                unsigned seen[2];
#pragma unroll
                for (int qt = 0; qt < 2; qt++) seen[qt] = t * BKV + key <= row_last[wave * 32 + qt * 16 + ln % 16] ? ~0u : 0u;
#pragma unroll
                for (int dt = 0; dt < DT; dt++) {
                    const u32x2 x = *(const u32x2 __attribute__((address_space(3)))*)(lds0 + (buf ? OTHER : 0u) + TILE_BYTES + key * ROWB + (((2 * dt + ln / 32) ^ swz<D>(key)) * 16) + (ln / 16 % 2) * 8);
#pragma unroll
                    for (int qt = 0; qt < 2; qt++) o[dt][qt] += only_odd(x, seen[qt]);
                }
            }
        }
    };
    auto row_total = [&](float x) {
        x += __shfl_xor(x, 16, 64);
        return x + __shfl_xor(x, 32, 64);
    };
    auto key_loop = [&](auto direct_tag) {
        if (t_begin < t_end) issue(t_begin, 0, std::false_type{});
        int t = t_begin, buf = 0;
        if constexpr (decltype(direct_tag)::value) {
            for (; t < plain_end; t++, buf ^= 1) {
                tile(t, buf, direct_tag, std::true_type{});
                kb ^= OTHER;
                vb ^= OTHER;
            }
        }
        for (; t < t_end; t++, buf ^= 1) {
            tile(t, buf, direct_tag, std::false_type{});
            kb ^= OTHER;
            vb ^= OTHER;
        }
        if ((t_end - t_begin) & 1) {     // back to the first buffer
            kb ^= OTHER;
            vb ^= OTHER;
        }
    };
    clear(0.f);
    key_loop(std::true_type{});
    {
        bool out_of_range = false;
#pragma unroll
        for (int qt = 0; qt < 2; qt++) {
            const float l = row_total(l_run[qt]);
            // (a row that sees none of these keys has no sum to judge)
            if (active && t_begin < t_end && row_last[wave * 32 + qt * 16 + lane_again() % 16] >= t_begin * BKV) out_of_range |= !(l > 0x1p-32f && l < 0x1p+64f);       // also true for NaN
        }
        // an infinity or NaN in a row's result may come from a value that the row does not see (0 x it in an MFMA); 0 x the results finds them
        f32x4 zero = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int dt = 0; dt < DT; dt++)
#pragma unroll
            for (int qt = 0; qt < 2; qt++)
#pragma unroll
                for (int i = 0; i < 4; i++) zero[i] = fmaf(o[dt][qt][i], 0.f, zero[i]);
        out_of_range |= !(zero[0] + zero[1] + zero[2] + zero[3] == 0.f);
        const int wave_bad = __any(out_of_range) ? 1 : 0;
        if (lane == 0) wave_flags[wave] = wave_bad;
        __syncthreads();                                     // ... and every wave is done with the tile buffers, in which the wave's 32 rows of the result are turned
        const bool again = (wave_flags[0] | wave_flags[1] | wave_flags[2] | wave_flags[3]) != 0;
        if (again) {
            clear(-__builtin_inff());
            key_loop(std::false_type{});
            __syncthreads();
        }
    }

    const int le = lane_again(), l16e = le % 16, q4e = le / 16;
    // results leave through LDS, whole rows with 16 bytes a lane (straight from the accumulators, 8 bytes a lane in 32-byte pieces: 1 to 2 % slower at head_dim 128, the same at 64)
    unsigned char* out = &smem[0][0] + wave * 32 * ROWB;
#pragma unroll
    for (int qt = 0; qt < 2; qt++) {
        const float l = row_total(l_run[qt]);
        const int row = u.row0 + wave * 32 + qt * 16 + l16e;
        const int tok = packed_div(row, a.by_group), head = u.head * a.group + (row - tok * a.group);
        if (a.parts > 1) {
            if (wave * 32 + qt * 16 + l16e >= u.rows) continue;
            const size_t at = ((size_t)(u.q0 + tok) * a.q_heads + head) * a.parts + u.part;
            // references are stored in base 2.  What the first attempt summed (reference 0) leaves with a power of two taken out, its sum in [1/2, 1): up to 2^64 of it times a value
            // may be just finite here and not in the merge of several parts.  (With a running maximum the sum is at most 2^8 a key.)
            const int e = m_run[qt] == 0.f ? __builtin_amdgcn_frexp_expf(l) : 0;         // (l = 0: 0)
            const float out_of = __builtin_amdgcn_ldexpf(1.f, -e);
            if (q4e == 0) *reinterpret_cast<f32x2*>(a.part + (size_t)a.total_q * a.q_heads * a.parts * D + at * 2) = f32x2{l == 0.f ? -__builtin_inff() : fmaf(m_run[qt], c, (float)e), l * out_of};
            if (l != 0.f) {                                  // (nothing to merge otherwise)
#pragma unroll
                for (int dt = 0; dt < DT; dt++) *reinterpret_cast<f32x4*>(a.part + at * D + dt * 16 + 4 * q4e) = o[dt][qt] * out_of;
            }
            continue;
        }
        const float inv = l == 0.f ? 0.f : 1.0f / l;         // no key with a score above minus infinity: zeros
        const int r = qt * 16 + l16e;
#pragma unroll
        for (int dt = 0; dt < DT; dt++)
            *reinterpret_cast<bf16x4*>(out + r * ROWB + (((2 * dt + q4e / 2) ^ (r % SLOTS)) * 16) + (q4e % 2) * 8) =
                bf16x4{(bf16_t)(o[dt][qt][0] * inv), (bf16_t)(o[dt][qt][1] * inv), (bf16_t)(o[dt][qt][2] * inv), (bf16_t)(o[dt][qt][3] * inv)};
    }
    if (a.parts > 1) return;
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int j = 0; j < 32 / CHUNK_ROWS; j++) {
        const int r = j * CHUNK_ROWS + le / SLOTS, row0 = wave * 32 + r;
        if (row0 >= u.rows) continue;
        const int row = u.row0 + row0, tok = packed_div(row, a.by_group), head = u.head * a.group + (row - tok * a.group);
        *reinterpret_cast<bf16x8*>(static_cast<char*>(a.o) + (size_t)(u.q0 + tok) * a.o_token + (size_t)head * a.o_head + (le % SLOTS) * 16) =
            *reinterpret_cast<const bf16x8*>(out + r * ROWB + (((le % SLOTS) ^ (r % SLOTS)) * 16));
    }
}

}  // namespace

int hyb_launch_packed_attention_mfma(PackedAttnArgs& a, int head_dim, hipStream_t st) {
    const dim3 grid = packed_grid(a);
    HybTraceScope trace("packed_attention_mfma", "byte", 4.0 * head_dim * ((double)a.total_q * a.q_heads + (double)a.total_k * a.k_heads), st);
    if (head_dim == 64) {
        if (a.prescaled) hipLaunchKernelGGL((packed_attention_kernel<64, true>), grid, dim3(256), 0, st, a);
        else hipLaunchKernelGGL((packed_attention_kernel<64, false>), grid, dim3(256), 0, st, a);
    } else {
        if (a.prescaled) hipLaunchKernelGGL((packed_attention_kernel<128, true>), grid, dim3(256), 0, st, a);
        else hipLaunchKernelGGL((packed_attention_kernel<128, false>), grid, dim3(256), 0, st, a);
    }
    return hyb_check_launch("packed_attention_mfma");
}
