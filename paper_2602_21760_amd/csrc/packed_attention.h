// Internal interface of the attention over packed batches: o = softmax(q k^T * scale) v per sequence and head, keys grouped.
//
// The queries of the q_heads / k_heads heads that share a key head are rows of one matrix: row r of (sequence, key head) is query
// r / group of head key_head * group + r % group.  A tile of rows then reads each key once for all of its heads, and a single new token
// still fills as many rows as it has heads in a group.
#pragma once
#include "common.h"

// n / d for 0 <= n < 2^32 by a multiplication and shifts (l = ceil(log2 d), m = floor(2^32 (2^l - d) / d) + 1: the quotient is exact).
struct PackedDivisor { unsigned m, shift1, shift2; };
inline PackedDivisor packed_divisor(unsigned d) {
    unsigned l = 0;
    while (l < 32 && ((unsigned long long)1 << l) < d) l++;
    return {(unsigned)((((unsigned long long)1 << l) - d) * ((unsigned long long)1 << 32) / d) + 1, l < 1 ? l : 1, l > 1 ? l - 1 : 0};
}
__device__ __forceinline__ int packed_div(int n, PackedDivisor d) {
    const unsigned t = __umulhi(d.m, (unsigned)n);
    return (int)((t + (((unsigned)n - t) >> d.shift1)) >> d.shift2);
}

struct PackedAttnArgs {
    const void *q, *k, *v;
    void* o;
    const int *offsets_q, *offsets_k;
    int sequences, total_q, total_k;
    int q_heads, k_heads, group;
    PackedDivisor by_group;
    float scale;                                  // > 0; PRE kernels do not use it
    int causal, prescaled;
    size_t q_token, q_head, k_token, k_head, v_token, v_head, o_token, o_head;   // strides in bytes
    int rows;                                     // rows of a block (few-rows kernel: not used)
    int blocks;                                   // row blocks of all sequences, an upper bound (see packed_find)
    int parts;                                    // the keys of a block are cut into up to `parts` parts (see packed_part_tiles); 1: not cut
    int pieces, part_keys;                        // few-rows kernel: pieces of part_keys keys of all sequences, an upper bound; 0 otherwise
    PackedDivisor by_piece;                       // part_keys
    int rests_last;                               // few-rows kernel: pieces that are not full come last (see piece_in_order)
    float* part;                                  // scratch (see below)
    int xcd_heads, xcd_shift, xcd_share;          // gcd(8, k_heads), its logarithm, 8 / gcd
    int per_head;                                 // units of a key head on each of its XCDs (this and the divisors: filled in by packed_grid)
    PackedDivisor by_heads, by_parts;             // heads of an XCD, parts
};

// Scratch of cut keys.  Blocks of rows that are cut (all but the few-rows kernel): for each (row of q, head) `parts` unnormalised accumulators of head_dim values, then for each `parts` pairs (reference in base 2, sum).
__host__ __device__ inline size_t packed_part_floats(int total_q, int q_heads, int parts, int head_dim) {
    return (size_t)total_q * q_heads * parts * (head_dim + 2);
}

// The few-rows kernel numbers pieces of part_keys keys: for each (piece, key head) 16 rows of head_dim values, then for each 16 pairs.
__host__ __device__ inline size_t packed_piece_rows(int pieces, int k_heads) { return (size_t)pieces * k_heads * 16; }

int hyb_launch_packed_attention_mfma(PackedAttnArgs& a, int head_dim, hipStream_t st);
int hyb_launch_packed_attention_few(PackedAttnArgs& a, int head_dim, hipStream_t st);
int hyb_launch_packed_attention_f32(PackedAttnArgs& a, int head_dim, hipStream_t st);

constexpr int kPackedRowsMfma = 128;                                                 // rows of a block: bf16
constexpr int kPackedRowsFew = 16;                                                   // bf16, few rows per sequence
constexpr int kPackedMaxParts = 64;
constexpr int kPackedPartKeys = 256;                                                 // least keys of a part
constexpr int packed_tile_keys(int head_dim) { return head_dim == 64 ? 64 : 32; }    // keys of its LDS tiles

// Most blocks of `rows` rows that any offsets can ask for.
inline long long packed_blocks(const PackedAttnArgs& a, int rows) { return (long long)a.total_q * a.group / rows + a.sequences; }

// Workgroups of a launch.  A grid dimension holds less than 2^32 threads: what goes beyond 2^23 workgroups goes into the second one.
inline dim3 packed_grid_of(size_t total) {
    const size_t x = total < ((size_t)1 << 23) ? total : (size_t)1 << 23;
    return dim3((unsigned)x, (unsigned)((total + x - 1) / x));
}
// Grid of a launch over a.blocks row blocks of every key head in a.parts parts; fills in the divisors by which the kernel finds its unit.
inline dim3 packed_grid(PackedAttnArgs& a) {
    const unsigned per_head = (unsigned)((a.blocks + a.xcd_share - 1) / a.xcd_share) * (unsigned)a.parts;
    a.by_heads = packed_divisor((unsigned)(a.k_heads / a.xcd_heads));
    a.by_parts = packed_divisor((unsigned)a.parts);
    a.per_head = (int)per_head;
    return packed_grid_of(8 * (size_t)(a.k_heads / a.xcd_heads) * per_head);
}
__device__ __forceinline__ unsigned packed_group_id() { return blockIdx.y * gridDim.x + blockIdx.x; }

// Rows of a sequence after the offsets are brought into 0 .. total.
__device__ __forceinline__ int packed_offset(const int* offsets, int s, int total) { return min(max(offsets[s], 0), total); }

// What a workgroup works on; rows == 0: nothing.
struct PackedUnit {
    int head, part;              // key head, part of the keys
    int row0, rows;              // first row of the block in its sequence, rows of the block (<= ROWS)
    int q0, k0;                  // first row of the sequence in q / o and in k / v
    int n_q, n_k;
    int sequence;
};
__device__ __forceinline__ void packed_rows_of(const PackedAttnArgs& a, int s, PackedUnit& u) {
    u.q0 = packed_offset(a.offsets_q, s, a.total_q);
    u.k0 = packed_offset(a.offsets_k, s, a.total_k);
    u.n_q = max(packed_offset(a.offsets_q, s + 1, a.total_q) - u.q0, 0);
    u.n_k = max(packed_offset(a.offsets_k, s + 1, a.total_k) - u.k0, 0);
}

// Up to 64 sequences: lane s holds sequence s (lanes without one: no rows), so that one trip to memory finds a unit.
__device__ __forceinline__ PackedUnit packed_lanes(const PackedAttnArgs& a) {
    PackedUnit mine = {};
    const int lane = threadIdx.x % 64;
    if (lane < a.sequences) packed_rows_of(a, lane, mine);
    return mine;
}
__device__ __forceinline__ void packed_take(const PackedUnit& lanes, int s, PackedUnit& u) {
    u.sequence = s;
    u.q0 = __builtin_amdgcn_readlane(lanes.q0, s);
    u.k0 = __builtin_amdgcn_readlane(lanes.k0, s);
    u.n_q = __builtin_amdgcn_readlane(lanes.n_q, s);
    u.n_k = __builtin_amdgcn_readlane(lanes.n_k, s);
}

// Pieces of sequences are numbered without a table: with `per` pieces' worth of rows (a block of query rows, a part of the keys) sequence s begins at number
// floor(first row / per) + s, which leaves every sequence at least as many numbers as it has pieces, and at least one (floor(x + n) - floor(x) + 1 >=
// ceil(n)); numbers left over have no rows.  The sequence of a number is the last one that begins at or before it, found by all lanes of the wave at
// once, 64 candidates a step.
// KEYS: pieces are of the keys, otherwise of the rows of queries; number: floor(first row / per).  Fills in the sequence's rows and returns the number of its first piece.
template <bool KEYS, typename N>
__device__ __forceinline__ int packed_find(const PackedAttnArgs& a, int piece, PackedUnit& u, N number) {
    const int lane = threadIdx.x % 64;
    if (a.sequences <= 64) {
        const PackedUnit lanes = packed_lanes(a);
        const int first = number(KEYS ? lanes.k0 : lanes.q0) + lane;
        const int s = max(__popcll(__ballot(lane < a.sequences && first <= piece)) - 1, 0);
        packed_take(lanes, s, u);
        return __builtin_amdgcn_readlane(first, s);
    }
    const int* offsets = KEYS ? a.offsets_k : a.offsets_q;
    const int total = KEYS ? a.total_k : a.total_q;
    int lo = 0, len = a.sequences;
    while (len > 1) {
        const int step = (len + 63) / 64, s = min(lo + lane * step, a.sequences - 1);
        const int count = __popcll(__ballot(lane * step < len && number(packed_offset(offsets, s, total)) + s <= piece));
        const int at = count > 0 ? count - 1 : 0;
        lo += at * step;
        len = min(step, len - at * step);
    }
    u.sequence = __builtin_amdgcn_readfirstlane(lo);
    packed_rows_of(a, u.sequence, u);
    return number(KEYS ? u.k0 : u.q0) + u.sequence;
}

// The rank-th block when sequences come in the order of decreasing numbers of keys (up to 64 of them) and a sequence's late blocks first, which are the long ones
// with a causal mask: a launch takes several rounds of workgroups of very different lengths and ends when the last one does.  Lane s holds sequence s and counts the
// blocks before its own.  Fills in the sequence's rows; returns the block's index in its sequence (-1: there are fewer).  (The order of single blocks by their number of
// keys, by bisection, takes three times the instructions and no less time; a table of it made by a kernel before this one neither.)
template <int ROWS>
__device__ __forceinline__ int packed_ranked_block(const PackedAttnArgs& a, int rank, PackedUnit& u) {
    const int lane = threadIdx.x % 64;
    const PackedUnit lanes = packed_lanes(a);
    const int blocks = (int)(((unsigned)(lanes.n_q * a.group) + ROWS - 1) / ROWS);
    const int key = min(lanes.n_k, (1 << 24) - 1) * 64 + 63 - lane;       // all different
    int before = 0;
    for (int s0 = 0; s0 < a.sequences; s0 += 8)
#pragma unroll
        for (int s = s0; s < s0 + 8; s++) before += __builtin_amdgcn_readlane(key, s) > key ? __builtin_amdgcn_readlane(blocks, s) : 0;     // (lanes without a sequence have no blocks)
    const unsigned long long here = __ballot(rank >= before && rank - before < blocks);
    if (here == 0) return -1;
    const int s = __builtin_ctzll(here);
    packed_take(lanes, s, u);
    return __builtin_amdgcn_readlane(blocks - 1 - (rank - before), s);
}

// Unit number `id` of a launch with packed_grid(a), most of them with rows.
template <int ROWS, bool LONG_FIRST = false>
__device__ __forceinline__ PackedUnit packed_unit(const PackedAttnArgs& a, unsigned id) {
    PackedUnit u = {};
    // XCD x (workgroups go round to the 8 XCDs) serves key heads = x mod gcd(8, k_heads), and where XCDs share a head every 8 / gcd-th block of it: the keys of a
    // head stay in as few L2s as possible, and every XCD gets blocks of all lengths.  A block's heads come one after the other, so that the order of lengths is that of the launch
    // (one sequence of 4096, causal, 24 heads of 64: 64 us; head after head 78.  Keys that no longer fit an L2 together cost nothing: 16717 tokens, the same heads, 1417 us either way).
    const int xcd = (int)(id % 8), hx = xcd & (a.xcd_heads - 1), sx = xcd >> a.xcd_shift;
    int j = (int)(id / 8);
    const int of_head = packed_div(j, a.by_heads);
    if (of_head >= a.per_head) return u;
    u.head = hx + a.xcd_heads * (j - of_head * (a.k_heads >> a.xcd_shift));
    j = of_head;
    const int b = packed_div(j, a.by_parts);
    u.part = j - b * a.parts;
    int block = b * a.xcd_share + sx;
    if (block >= a.blocks) return u;
    int first = 0;
    if (LONG_FIRST && a.sequences > 1 && a.sequences <= 64) {
        block = packed_ranked_block<ROWS>(a, block, u);
        if (block < 0) return u;
    } else {
        block = a.blocks - 1 - block;        // late blocks first: with a causal mask they are the long ones
        first = packed_find<false>(a, block, u, [&](int q0) { return (int)((long long)q0 * a.group / ROWS); });
        if (first > block) return u;
    }
    const long long all = (long long)u.n_q * a.group, row0 = (long long)(block - first) * ROWS;
    u.rows = (int)max(min(all - row0, (long long)ROWS), 0ll);
    u.row0 = (int)row0;           // (meaningful when rows > 0: below total_q * group, which the launcher keeps below 2^31)
    return u;
}

// Tiles of a part of a block that sees nt tiles of `tile` keys: even shares, which need no knowledge of the longest sequence on the host.
__device__ __forceinline__ int packed_part_tiles(const PackedAttnArgs& a, int nt, int tile) {
    return a.parts == 1 ? nt : max((nt + a.parts - 1) / a.parts, kPackedPartKeys / tile);
}

// Last key that query t of a sequence sees (-1: none).
__device__ __forceinline__ int packed_last_key(const PackedAttnArgs& a, const PackedUnit& u, int t) {
    return a.causal ? max(min(t + u.n_k - u.n_q, u.n_k - 1), -1) : u.n_k - 1;
}

// Infinities and NaN (exponent bits all ones), found and blanked without comparisons, which would need a scalar register pair per value: the exponent field
// plus its lowest bit carries into the sign's place.  bf16: two values per word.
__device__ __forceinline__ unsigned odd_bits_bf16(unsigned x) { return ((x & 0x7f807f80u) + 0x00800080u) & 0x80008000u; }
__device__ __forceinline__ unsigned odd_mask_bf16(unsigned x) {    // all ones in the places of such values
    const unsigned h = odd_bits_bf16(x);
    return (h << 1) - (h >> 15);
}
__device__ __forceinline__ unsigned odd_bits_f32(unsigned x) { return ((x & 0x7f800000u) + 0x00800000u) & 0x80000000u; }
__device__ __forceinline__ unsigned odd_mask_f32(unsigned x) { return (unsigned)((int)odd_bits_f32(x) >> 31); }

__device__ __forceinline__ void keep_finite(bf16x4& x) {
    u32x2 w = __builtin_bit_cast(u32x2, x);
    w[0] &= ~odd_mask_bf16(w[0]);
    w[1] &= ~odd_mask_bf16(w[1]);
    x = __builtin_bit_cast(bf16x4, w);
}
// The infinities and NaN among four values where `seen` (0 or all ones) says so, zeros elsewhere.
__device__ __forceinline__ f32x4 only_odd(u32x2 w, unsigned seen) {
    const unsigned a = w[0] & odd_mask_bf16(w[0]) & seen, b = w[1] & odd_mask_bf16(w[1]) & seen;
    return f32x4{__uint_as_float(a << 16), __uint_as_float(a & 0xffff0000u), __uint_as_float(b << 16), __uint_as_float(b & 0xffff0000u)};
}
