// Routed pairs sorted by expert into groups of rows (ft_expert_sort): a stable counting sort.
//
// A pair's row is the start of its expert's group plus the number of pairs of that expert before it.  Within
// a wave that number comes from the lanes that hold the same expert (one ballot per bit of the id), across
// the waves of a workgroup from their counts in LDS, across workgroups from a table of counts.  No atomic decides a
// place, so equal calls give equal tables.
//
// Up to kSortPairs pairs: one launch of one workgroup.  More: counts per workgroup, and the placing, in which every
// workgroup sums up the counts before its own and forms the groups' starts for itself; past kSortOwnSums workgroups a
// launch between the two turns the counts into sums.  Bound: launches and round trips: 32 pairs 4.5 us, 2048 7.4, 65536 11.7,
// 786432 17.0.  One wave per expert that clears the rows behind its pairs, in place of clearing all of them ahead of the
// counts: 7.2 us for 32 pairs of 256 experts.
#include "ftmoe_device.h"
#include "ftmoe_internal.h"

namespace ftmoe {

constexpr int kSortThreads = 512, kSortWaves = kSortThreads / 64, kSortSteps = kSortPairs / kSortThreads;

// local expert of pair p; n where it has none here
__device__ __forceinline__ int sort_key(const SortArgs &a, int p) {
    const uint32_t e = static_cast<uint32_t>(a.ids[p]) - static_cast<uint32_t>(a.first);
    const bool in = e < static_cast<uint32_t>(a.n) && (!a.mask || a.mask[p / a.k]);
    return in ? static_cast<int>(e) : a.n;
}

// rows without a pair are what the placing leaves of this
__device__ __forceinline__ void sort_clear(const SortArgs &a) {
    for (int r = blockIdx.x * kSortThreads + threadIdx.x; r < a.rows; r += gridDim.x * kSortThreads) a.row_pair[r] = -1;
}

__global__ __launch_bounds__(kSortThreads) void sort_count(SortArgs a) {
    extern __shared__ int hist[];   // [n + 1]
    const int p0 = blockIdx.x * a.chunk, p1 = min(p0 + a.chunk, a.pairs);
    for (int e = threadIdx.x; e <= a.n; e += kSortThreads) hist[e] = 0;
    sort_clear(a);
    __syncthreads();
    for (int sub = p0; sub < p1; sub += kSortPairs) {
        int key[kSortSteps];
#pragma unroll
        for (int i = 0; i < kSortSteps; ++i) {
            const int p = sub + i * kSortThreads + threadIdx.x;
            key[i] = p < p1 ? sort_key(a, p) : a.n;
        }
#pragma unroll
        for (int i = 0; i < kSortSteps; ++i) atomicAdd(&hist[key[i]], 1);
    }
    __syncthreads();
    for (int e = threadIdx.x; e < a.n; e += kSortThreads) a.table[static_cast<size_t>(blockIdx.x) * a.n + e] = hist[e];
}

// one wave per expert: its counts become the counts before each workgroup
__global__ __launch_bounds__(64) void sort_prefix(SortArgs a) {
    int32_t *col = a.table + blockIdx.x;
    const int per = (a.blocks + 63) / 64, b0 = min(static_cast<int>(threadIdx.x) * per, a.blocks), b1 = min(b0 + per, a.blocks);
    uint32_t sum = 0;
    for (int b = b0; b < b1; ++b) sum += col[static_cast<size_t>(b) * a.n];
    const uint32_t upto = wave_incl_scan_u32(sum);
    uint32_t before = upto - sum;
    for (int b = b0; b < b1; ++b) {
        const uint32_t v = col[static_cast<size_t>(b) * a.n];
        col[static_cast<size_t>(b) * a.n] = static_cast<int32_t>(before);
        before += v;
    }
    if (threadIdx.x == 63) a.totals[blockIdx.x] = static_cast<int32_t>(upto);
}

__global__ __launch_bounds__(kSortThreads) void sort_place(SortArgs a, int nbits) {
    extern __shared__ int lds[];
    int *hist = lds;                          // [waves][n]: pairs of a wave, then the row of its first one
    int *off = hist + kSortWaves * a.n;       // [n + 1] groups' starts
    int *end = off + a.n + 1;                 // [n] one past the last row with a pair
    int *run = end + a.n;                     // [n] totals, then the next row to fill
    int *lead = run + a.n;                    // [n] pairs in the workgroups before this one
    const int t = threadIdx.x, wave = t / 64, lane = lane_id();
    const bool whole = a.blocks == 1;
    if (whole) sort_clear(a);
    const int p0 = blockIdx.x * a.chunk, p1 = min(p0 + a.chunk, a.pairs);
    bool first = true;
    for (int sub = p0; first || sub < p1; sub += kSortPairs) {
        for (int i = t; i < kSortWaves * a.n; i += kSortThreads) hist[i] = 0;
        __syncthreads();
        // a wave's pairs are consecutive, so that its counts come in the order of the pairs
        const int each = (min(p1 - sub, kSortPairs) + kSortThreads - 1) / kSortThreads;   // steps of 64 pairs
        int key[kSortSteps], rank[kSortSteps];
#pragma unroll
        for (int i = 0; i < kSortSteps; ++i) {
            const int p = sub + (wave * each + i) * 64 + lane;
            key[i] = i < each && p < p1 ? sort_key(a, p) : a.n;
        }
#pragma unroll
        for (int i = 0; i < kSortSteps; ++i) {
            const bool in = key[i] < a.n;
            if (i >= each || !__ballot(in)) continue;
            const uint64_t same = match_lanes(key[i], nbits, __ballot(in)), lower = same & lanemask_lt();
            int *h = hist + wave * a.n + (in ? key[i] : 0);
            const int had = in ? *h : 0;
            rank[i] = had + __popcll(lower);
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            if (in && lower == 0) *h = had + __popcll(same);
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        }
        __syncthreads();
        if (first) {
            for (int e = t; e < a.n; e += kSortThreads) {
                int sum = 0, mine = 0;
                if (whole) {
#pragma unroll
                    for (int w = 0; w < kSortWaves; ++w) sum += hist[w * a.n + e];
                } else if (a.blocks > kSortOwnSums) {
                    sum = a.totals[e];
                    mine = a.table[static_cast<size_t>(blockIdx.x) * a.n + e];
                } else {
#pragma unroll 8
                    for (int b = 0; b < a.blocks; ++b) {
                        const int v = a.table[static_cast<size_t>(b) * a.n + e];
                        sum += v;
                        mine += b < static_cast<int>(blockIdx.x) ? v : 0;
                    }
                }
                run[e] = sum;
                lead[e] = mine;
            }
            __syncthreads();
            if (wave == 0) {
                const int per = (a.n + 63) / 64, e0 = min(lane * per, a.n), e1 = min(e0 + per, a.n);
                // groups may pass 32 bits only together: rows are counted up to the capacity
                uint32_t sum = 0, lost = 0;
                const uint32_t cap = a.rows;
                auto padded = [&](int e) { return min((static_cast<uint32_t>(run[e]) + a.align - 1) / a.align * a.align, cap); };
                for (int e = e0; e < e1; ++e) sum = min(sum + padded(e), cap);
                uint32_t before = wave_incl_scan_u32(sum) - sum;   // at most 64 capacities of 2^20
                for (int e = e0; e < e1; ++e) {
                    const uint32_t o = min(before, cap), c = min(static_cast<uint32_t>(run[e]), cap - o);
                    off[e] = static_cast<int>(o);
                    end[e] = static_cast<int>(o + c);
                    lost += run[e] - c;
                    before = min(before + padded(e), cap);
                }
                const uint32_t all = wave_incl_scan_u32(sum), drops = wave_incl_scan_u32(lost);
                if (lane == 63) {
                    off[a.n] = static_cast<int>(min(all, cap));
                    if (blockIdx.x == 0) *a.dropped = static_cast<int32_t>(drops);
                }
            }
            __syncthreads();
            for (int e = t; e < a.n; e += kSortThreads) {
                run[e] = off[e] + lead[e];
                if (blockIdx.x == 0) a.count[e] = end[e] - off[e];
            }
            if (blockIdx.x == 0)
                for (int e = t; e <= a.n; e += kSortThreads) a.off[e] = off[e];
            first = false;
        }
        __syncthreads();
        for (int e = t; e < a.n; e += kSortThreads) {
            int at = run[e];
            for (int w = 0; w < kSortWaves; ++w) {
                const int v = hist[w * a.n + e];
                hist[w * a.n + e] = at;
                at += v;
            }
            run[e] = at;
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kSortSteps; ++i) {
            const int p = sub + (wave * each + i) * 64 + lane;
            if (i >= each || p >= p1) continue;
            int row = -1;
            if (key[i] < a.n) {
                row = hist[wave * a.n + key[i]] + rank[i];
                if (row < end[key[i]]) a.row_pair[row] = p;
                else row = -1;
            }
            a.pair_row[p] = row;
        }
        __syncthreads();
    }
}

hipError_t launch_sort(const SortArgs &a, hipStream_t s) {
    if (a.blocks > 1) {
        hipLaunchKernelGGL(sort_count, dim3(a.blocks), dim3(kSortThreads), (a.n + 1) * 4, s, a);
        if (a.blocks > kSortOwnSums) hipLaunchKernelGGL(sort_prefix, dim3(a.n), dim3(64), 0, s, a);
    }
    int nbits = 1;
    while ((1 << nbits) < a.n) ++nbits;   // of the keys that have an expert here
    const unsigned lds = ((kSortWaves + 4) * a.n + 1) * 4;
    hipLaunchKernelGGL(sort_place, dim3(a.blocks), dim3(kSortThreads), lds, s, a, nbits);
    return hipGetLastError();
}

}  // namespace ftmoe
