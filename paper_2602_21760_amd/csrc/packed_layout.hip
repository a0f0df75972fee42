// Layout of a packed batch: offsets of the requests, and request index and (time, height, width) position of every token.
//
// Bound by what it writes, 16 bytes a row (4000 requests, 18 million rows: 5.3 TB/s); small batches by launch latency (8 requests, 20 000 rows: 4.2 us on the GPU; 256, 1.2 million: 8.5).  Lengths are summed with an addition that
// saturates at the capacity (associative, and exact for everything below it), so a prefix sum needs no 64-bit numbers.
#include "common.h"

namespace {

constexpr int kThreads = 256;
constexpr int kRowsPerThread = 4;       // 16 bytes of request indices and 48 bytes of positions: four full stores
constexpr int kInOne = 2048;            // requests whose prefix sum every workgroup makes for itself (8 KB of LDS)

__device__ __forceinline__ unsigned add_capped(unsigned a, unsigned b, unsigned cap) {   // a, b <= cap < 2^31
    return min(a + b, cap);
}

__device__ __forceinline__ unsigned tokens_of(int4 s, unsigned cap) {
    const unsigned long long f = max(s.x, 0), h = max(s.y, 0), w = max(s.z, 0), t = max(s.w, 0);
    const unsigned long long fh = min(f * h, (unsigned long long)1 << 31);       // < 2^62 before, and the next product < 2^62 again
    return (unsigned)min(fh * w + t, (unsigned long long)cap);
}

// Exclusive prefix sum of one value per thread; *total gets the sum.  wave_sums: LDS, kThreads / 64 values.
__device__ __forceinline__ unsigned block_scan(unsigned x, unsigned cap, unsigned* wave_sums, unsigned* total) {
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    unsigned inc = x;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const unsigned below = __shfl_up(inc, o, 64);
        if (lane >= o) inc = add_capped(inc, below, cap);
    }
    if (lane == 63) wave_sums[wave] = inc;
    __syncthreads();
    unsigned before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kThreads / 64; w++) {
        if (w < wave) before = add_capped(before, wave_sums[w], cap);
        all = add_capped(all, wave_sums[w], cap);
    }
    __syncthreads();
    *total = all;
    unsigned excl = __shfl_up(inc, 1, 64);
    if (lane == 0) excl = 0;
    return add_capped(before, excl, cap);
}

// offsets[0 .. requests] by one workgroup, eight requests per thread at a time: 2048 requests per scan (4000 requests, 18 million rows, both kernels: 54.1 us,
// one request per thread 59.6).
__global__ __launch_bounds__(kThreads) void packed_offsets_kernel(const int4* shapes, int requests, unsigned cap, int* offsets) {
    __shared__ unsigned wave_sums[kThreads / 64];
    constexpr int kEach = 8;
    unsigned carry = 0;
    for (int s0 = 0; s0 < requests; s0 += kThreads * kEach) {
        const int first = s0 + threadIdx.x * kEach;
        unsigned before[kEach], mine = 0, all;       // tokens before each of the thread's requests
#pragma unroll
        for (int i = 0; i < kEach; i++) {
            before[i] = mine;
            mine = add_capped(mine, first + i < requests ? tokens_of(shapes[first + i], cap) : 0u, cap);
        }
        const unsigned start = add_capped(carry, block_scan(mine, cap, wave_sums, &all), cap);
#pragma unroll
        for (int i = 0; i < kEach; i++)
            if (first + i < requests) offsets[first + i] = (int)add_capped(start, before[i], cap);
        carry = add_capped(carry, all, cap);
    }
    if (threadIdx.x == 0) offsets[requests] = (int)carry;
}

struct Place { int request, t, y, x; };
__device__ __forceinline__ Place place_of(int s, int4 sh, unsigned i, bool text_after) {
    const unsigned f = max(sh.x, 0), h = max(sh.y, 0), w = max(sh.z, 0);
    const unsigned long long hw = (unsigned long long)h * w;
    // (an image of 2^32 tokens or more holds every row that fits; its row index still fits 32 bits)
    const bool image = hw > 0xffffffffull ? f > 0 : (unsigned long long)f * hw > i;
    if (image) {
        const unsigned plane = hw > 0xffffffffull ? 0u : i / (unsigned)hw, in = hw > 0xffffffffull ? i : i - plane * (unsigned)hw;
        return {s, (int)plane, (int)(in / w), (int)(in % w)};
    }
    const unsigned j = i - f * (unsigned)hw;
    const int p = text_after ? (int)(max(f, max(h, w)) + j) : 0;
    return {s, p, p, p};
}

// Four rows per thread.  SCAN: every workgroup sums the lengths in LDS itself (requests <= kInOne), the first writes the offsets too: one launch;
// otherwise the offsets are there.
template <bool SCAN>
__global__ __launch_bounds__(kThreads) void packed_rows_kernel(const int4* shapes, int requests, unsigned cap, int text_after, int chunks, int* offsets, int* request, int* positions) {
    __shared__ unsigned own[SCAN ? kInOne + 1 : 1];
    __shared__ int4 stage[kThreads / 64][192];
    const unsigned lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    __shared__ unsigned wave_sums[kThreads / 64];
    if constexpr (SCAN) {
        unsigned carry = 0;
        for (int s0 = 0; s0 < requests; s0 += kThreads) {
            const int s = s0 + threadIdx.x;
            unsigned all;
            const unsigned before = block_scan(s < requests ? tokens_of(shapes[s], cap) : 0u, cap, wave_sums, &all);
            if (s < requests) own[s] = add_capped(carry, before, cap);
            carry = add_capped(carry, all, cap);
        }
        if (threadIdx.x == 0) own[requests] = carry;
        __syncthreads();
        if (blockIdx.x == 0)
            for (int s = threadIdx.x; s <= requests; s += kThreads) offsets[s] = (int)own[s];
    }
    auto first_row = [&](int s) { return SCAN ? own[s] : (unsigned)offsets[s]; };
    const unsigned rows = first_row(requests);
    for (int chunk = 0; chunk < chunks; chunk++) {
        const unsigned r0 = (((unsigned)blockIdx.x * chunks + chunk) * kThreads + threadIdx.x) * kRowsPerThread;
        const unsigned wave0 = r0 - lane * kRowsPerThread;       // (the wave's first row)
        if (r0 >= rows) return;
        int s = 0;                                  // the last request that begins at or before r0: it is not empty, first_row(s) <= r0 < first_row(s + 1)
        for (int len = requests; len > 1;) {
            const int half = len / 2;
            if (first_row(s + half) <= r0) { s += half; len -= half; }
            else len = half;
        }
        int4 sh = shapes[s];
        unsigned begin = first_row(s), end = first_row(s + 1);
        int req[kRowsPerThread], pos[kRowsPerThread][3];
        const unsigned i0 = r0 - begin;
        const Place p = place_of(s, sh, i0, text_after != 0);
        // four rows of one image (almost all threads): counting on from the first; otherwise row by row
        const unsigned long long image = (unsigned long long)((unsigned)max(sh.y, 0) * (unsigned long long)max(sh.z, 0)) * (unsigned)max(sh.x, 0);
        if (r0 + kRowsPerThread <= end && i0 + kRowsPerThread <= image) {
            int t = p.t, y = p.y, x = p.x;
#pragma unroll
            for (int i = 0; i < kRowsPerThread; i++) {
                req[i] = s; pos[i][0] = t; pos[i][1] = y; pos[i][2] = x;
                x++;
                const int line = x == sh.z;
                x = line ? 0 : x;
                y += line;
                const int frame = y == sh.y;
                y = frame ? 0 : y;
                t += frame;
            }
        } else {
            const int count = (int)min(rows - r0, (unsigned)kRowsPerThread);
#pragma unroll
            for (int i = 0; i < kRowsPerThread; i++) {
                if (i >= count) { req[i] = -1; pos[i][0] = pos[i][1] = pos[i][2] = 0; continue; }
                while (r0 + i >= end) {             // (ends: r0 + i < rows = the end of the last request)
                    s++;
                    begin = end;
                    end = first_row(s + 1);
                    sh = shapes[s];
                }
                const Place p = place_of(s, sh, r0 + i - begin, text_after != 0);
                req[i] = p.request; pos[i][0] = p.t; pos[i][1] = p.y; pos[i][2] = p.x;
            }
        }
        if (wave0 + 64 * kRowsPerThread <= rows) {
            if (request) *reinterpret_cast<int4*>(request + r0) = make_int4(req[0], req[1], req[2], req[3]);
            if (positions) {     // through LDS, so that a store of the wave writes 1 KB in a row and not every third 16 bytes of 3 KB
                stage[wave][3 * lane] = make_int4(pos[0][0], pos[0][1], pos[0][2], pos[1][0]);
                stage[wave][3 * lane + 1] = make_int4(pos[1][1], pos[1][2], pos[2][0], pos[2][1]);
                stage[wave][3 * lane + 2] = make_int4(pos[2][2], pos[3][0], pos[3][1], pos[3][2]);
                __builtin_amdgcn_wave_barrier();
                int4* dst = reinterpret_cast<int4*>(positions + (size_t)wave0 * 3);
#pragma unroll
                for (int i = 0; i < 3; i++) dst[64 * i + lane] = stage[wave][64 * i + lane];
                __builtin_amdgcn_wave_barrier();
            }
        } else {
#pragma unroll
            for (int i = 0; i < kRowsPerThread; i++) {
                if (req[i] < 0) continue;
                if (request) request[r0 + i] = req[i];
                if (positions)
                    for (int a = 0; a < 3; a++) positions[(size_t)(r0 + i) * 3 + a] = pos[i][a];
            }
        }
    }
}

}  // namespace

extern "C" int hyb_packed_layout(const int* shapes, int requests, int capacity, int text_after, int* offsets, int* request, int* positions, void* stream) {
    HYB_REQUIRE(requests >= 0 && capacity >= 0, HYB_ERR_SHAPE, "hyb_packed_layout: negative size");
    HYB_CHECK_PTR(offsets); HYB_CHECK_ALIGN(offsets);
    if (requests > 0) HYB_CHECK_PTR(shapes);
    HYB_CHECK_ALIGN(shapes); HYB_CHECK_ALIGN(request); HYB_CHECK_ALIGN(positions);
    const hipStream_t st = (hipStream_t)stream;
    const int4* sh = reinterpret_cast<const int4*>(shapes);
    const unsigned cap = (unsigned)capacity;
    const bool rows = requests > 0 && capacity > 0 && (request || positions);
    // chunks of 1024 rows; workgroups take several in a row where there are more than the chip holds, so that the sums are made less often
    const size_t all = ((size_t)capacity + kThreads * kRowsPerThread - 1) / (kThreads * kRowsPerThread), most = (size_t)hyb_cu_count() * 4;
    const int chunks = requests <= kInOne ? (int)((all + most - 1) / most) : (all > 0), groups = chunks ? (int)((all + chunks - 1) / chunks) : 0;
    if (rows && requests <= kInOne) {
        HybTraceScope trace("packed_layout", "byte", 16.0 * requests + 16.0 * capacity, st);
        hipLaunchKernelGGL(packed_rows_kernel<true>, dim3(groups), dim3(kThreads), 0, st, sh, requests, cap, text_after, chunks, offsets, request, positions);
        return hyb_check_launch("packed_layout");
    }
    {
        HybTraceScope trace("packed_offsets", "byte", 20.0 * requests, st);
        hipLaunchKernelGGL(packed_offsets_kernel, dim3(1), dim3(kThreads), 0, st, sh, requests, cap, offsets);
    }
    const int rc = hyb_check_launch("packed_offsets");
    if (rc != HYB_OK || !rows) return rc;
    HybTraceScope trace("packed_layout", "byte", 16.0 * capacity, st);
    hipLaunchKernelGGL(packed_rows_kernel<false>, dim3(groups), dim3(kThreads), 0, st, sh, requests, cap, text_after, chunks, offsets, request, positions);
    return hyb_check_launch("packed_layout");
}
