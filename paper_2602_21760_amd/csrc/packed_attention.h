// Internal interface of the attention over packed batches: o = softmax(q k^T * scale) v per sequence and head, keys grouped.
//
// The queries of the q_heads / k_heads heads that share a key head are rows of one matrix: row r of (sequence, key head) is query
// r / group of head key_head * group + r % group.  A tile of rows then reads each key once for all of its heads, and a single new token
// still fills as many rows as it has heads in a group.
#pragma once
#include "common.h"

struct PackedAttnArgs {
    const void *q, *k, *v;
    void* o;
    const int *offsets_q, *offsets_k;
    int sequences, total_q, total_k;
    int q_heads, k_heads, group;
    float scale;                                  // > 0; PRE kernels do not use it
    int causal, prescaled;
    size_t q_token, q_head, k_token, k_head, v_token, v_head, o_token, o_head;   // strides in bytes
    int blocks;                                   // row blocks of all sequences, an upper bound (see find_block)
    int parts, part_keys;                         // keys are cut into `parts` of part_keys keys (the last part takes what is left); 1: not cut
    float* part;                                  // parts > 1: PartRows
    int xcd_heads, xcd_share;                     // gcd(8, k_heads), 8 / gcd
};

// Scratch of cut keys: for each (row of q, head) `parts` unnormalised accumulators of head_dim values, then for each `parts` pairs (reference, sum).
__host__ __device__ inline size_t packed_part_floats(int total_q, int q_heads, int parts, int head_dim) {
    return (size_t)total_q * q_heads * parts * (head_dim + 2);
}

int hyb_launch_packed_attention_mfma(const PackedAttnArgs& a, int head_dim, hipStream_t st);
int hyb_launch_packed_attention_f32(const PackedAttnArgs& a, int head_dim, hipStream_t st);

constexpr int kPackedRowsMfma = 128;                                                 // rows of a block: bf16
constexpr int packed_rows_f32(int head_dim) { return head_dim == 64 ? 32 : 16; }     // fp32

// Most blocks of `rows` rows that any offsets can ask for.
inline long long packed_blocks(const PackedAttnArgs& a, int rows) { return (long long)a.total_q * a.group / rows + a.sequences; }

// Workgroups of a launch.  A grid dimension holds less than 2^32 threads: what goes beyond 2^23 workgroups goes into the second one.
inline dim3 packed_grid(const PackedAttnArgs& a) {
    const size_t per_head = (size_t)((a.blocks + a.xcd_share - 1) / a.xcd_share) * a.parts;
    const size_t total = 8 * (size_t)(a.k_heads / a.xcd_heads) * per_head, x = total < ((size_t)1 << 23) ? total : (size_t)1 << 23;
    return dim3((unsigned)x, (unsigned)((total + x - 1) / x));
}

// Rows of a sequence after the offsets are brought into 0 .. total.
__device__ __forceinline__ int packed_offset(const int* offsets, int s, int total) { return min(max(offsets[s], 0), total); }

// Blocks are numbered without a table: sequence s begins at block floor(first row / ROWS) + s, which leaves every sequence at least as
// many numbers as it has blocks of ROWS rows (floor(x + n) - floor(x) + 1 >= ceil(n)); the numbers left over have no rows.  The sequence of a
// number is the last one that begins at or before it, found by all lanes of the wave at once, 64 candidates a step.
template <int ROWS>
__device__ __forceinline__ int packed_sequence_of(const PackedAttnArgs& a, int block) {
    const int lane = threadIdx.x % 64;
    int lo = 0, len = a.sequences;
    while (len > 1) {
        const int step = (len + 63) / 64, s = lo + lane * step;
        const bool begins = lane * step < len &&
                            (int)((long long)packed_offset(a.offsets_q, min(s, a.sequences - 1), a.total_q) * a.group / ROWS) + s <= block;
        const int count = __popcll(__ballot(begins));
        const int at = count > 0 ? count - 1 : 0;
        lo += at * step;
        len = min(step, len - at * step);
    }
    return __builtin_amdgcn_readfirstlane(lo);
}

// What a workgroup works on; rows == 0: nothing.
struct PackedUnit {
    int head, part;              // key head, part of the keys
    int row0, rows;              // first row of the block in its sequence, rows of the block (<= ROWS)
    int q0, k0;                  // first row of the sequence in q / o and in k / v
    int n_q, n_k;
};
template <int ROWS>
__device__ __forceinline__ PackedUnit packed_unit(const PackedAttnArgs& a) {
    PackedUnit u = {};
    // XCD x (workgroups go round to the 8 XCDs) serves key heads = x mod gcd(8, k_heads), and where XCDs share a head every 8 / gcd-th block of it: the keys of a
    // head stay in as few L2s as possible, and every XCD gets blocks of all lengths.  Late blocks first: with a causal mask they are the long ones.
    const unsigned id = blockIdx.y * gridDim.x + blockIdx.x;
    const int xcd = (int)(id % 8), hx = xcd % a.xcd_heads, sx = xcd / a.xcd_heads;
    unsigned j = id / 8;
    const unsigned per_head = (unsigned)((a.blocks + a.xcd_share - 1) / a.xcd_share) * (unsigned)a.parts;
    u.head = hx + a.xcd_heads * (int)(j / per_head);
    if (u.head >= a.k_heads) return u;
    j %= per_head;
    u.part = (int)(j % (unsigned)a.parts);
    const int block = a.blocks - 1 - ((int)(j / (unsigned)a.parts) * a.xcd_share + sx);
    if (block < 0) return u;
    const int s = packed_sequence_of<ROWS>(a, block);
    const int q0 = packed_offset(a.offsets_q, s, a.total_q), k0 = packed_offset(a.offsets_k, s, a.total_k);
    const long long first = (long long)q0 * a.group / ROWS + s;
    if (first > block) return u;
    u.q0 = q0; u.k0 = k0;
    u.n_q = packed_offset(a.offsets_q, s + 1, a.total_q) - q0;
    u.n_k = max(packed_offset(a.offsets_k, s + 1, a.total_k) - k0, 0);
    const long long all = (long long)max(u.n_q, 0) * a.group, row0 = (block - first) * ROWS;
    u.rows = (int)max(min(all - row0, (long long)ROWS), 0ll);
    u.row0 = (int)row0;           // (meaningful when rows > 0: below total_q * group, which the launcher keeps below 2^31)
    return u;
}

// Last key that query t of a sequence sees (-1: none).
__device__ __forceinline__ int packed_last_key(const PackedAttnArgs& a, const PackedUnit& u, int t) {
    return a.causal ? max(min(t + u.n_k - u.n_q, u.n_k - 1), -1) : u.n_k - 1;
}
