// Products over groups of rows, one weight per group (ft_expert_linear, ft_expert_weight_grad): the tiles of
// product_tile.h, each of which lies in one group.  The groups' sizes are known on the device only: the grid covers
// the most tiles that the rows can make, a workgroup finds its tile from the groups' starts, and those without one end.
//
// ft_expert_linear: A is expert e's weight, B the rows of group e.  ft_expert_weight_grad: A and B are the column
// forms of x and dy, whose blocks of 128 tokens lie in one group each, and the reduction runs over the group's.
#include "product_tile.h"

#include <algorithm>
#include <cmath>

namespace ftmoe {

// Group e as the tables have it, held inside the rows whatever they say.
__device__ __forceinline__ int group_start(const GroupArgs &g, int e) {
    return min(max(g.off[e], 0), g.rows) & -g.align;
}

struct GroupTile {
    int e, row, real, end;   // expert, first row, one past its last row with a pair and past its last row
};

// Tile t of BB rows, in the order of the experts.  Every wave finds it for itself: 64 lanes hold up to 16 experts each.
template <int BB>
__device__ __forceinline__ void group_scan(const GroupArgs &g, uint32_t &before, uint32_t &upto, int &per) {
    per = (g.n + 63) / 64;
    const int e0 = min(lane_id() * per, g.n), e1 = min(e0 + per, g.n);
    uint32_t sum = 0;
    int o = group_start(g, e0);
#pragma unroll 4
    for (int e = e0; e < e1; ++e) {
        const int next = group_start(g, e + 1);
        sum += static_cast<uint32_t>(max(next - o, 0) + BB - 1) / BB;
        o = next;
    }
    upto = wave_incl_scan_u32(sum);
    before = upto - sum;
}
template <int BB>
__device__ __forceinline__ GroupTile group_tile(const GroupArgs &g, uint32_t t, uint32_t before, uint32_t upto, int per) {
    GroupTile r;
    const int lane = __ffsll(static_cast<unsigned long long>(__ballot(t >= before && t < upto))) - 1;   // t is below the total
    uint32_t rest = t - readlane_u32(before, lane);
    r.e = lane * per;
    for (;; ++r.e) {
        r.row = group_start(g, r.e);
        r.end = group_start(g, r.e + 1);
        const uint32_t tiles = static_cast<uint32_t>(max(r.end - r.row, 0) + BB - 1) / BB;
        if (rest < tiles) break;
        rest -= tiles;
    }
    r.real = r.row + min(max(g.count[r.e], 0), max(r.end - r.row, 0));
    r.row += static_cast<int>(rest) * BB;
    r.end = min(r.end, r.row + BB);
    return r;
}

// zeros in rows [b0, b1) and columns [a0, a1) of an output of M columns (a0, a1 and M multiples of 16)
template <int OUT>
__device__ __forceinline__ void zero_tile(void *out, int M, int a0, int a1, int b0, int b1) {
    constexpr int kEach = OUT == 0 ? 8 : 4;
    const int width = (a1 - a0) / kEach;
    for (int i = threadIdx.x; i < (b1 - b0) * width; i += blockDim.x) {
        const int b = b0 + i / width, a = a0 + i % width * kEach;
        *reinterpret_cast<u32x4_t *>(static_cast<uint8_t *>(out) + (static_cast<size_t>(b) * M + a) * (OUT == 0 ? 2 : 4)) = u32x4_t{};
    }
}

__device__ __forceinline__ ProductArgs of_expert(ProductArgs p, const GroupArgs &g, const GroupTile &t) {
    p.a += t.e * g.a_stride;
    p.as = static_cast<const float *>(p.as) + t.e * g.as_stride;
    p.R = t.real;
    return p;
}

// Tiles of eight waves take a CU each.  Where the last round of them would fill no more than half of the card, its tiles are
// halved along A and fill twice as many CUs for 0.6 to 0.7 of the time (256 x 256: 16 of 1024 x 4096, 264 tiles, 109 -> 94 us; 8 of
// 2048 x 7168, 352 tiles, 179 -> 155; 32 of 4096 x 7168, 2112 tiles, 936 -> 893; 256 x 128: 16 of 2048 x 2048, 320 tiles, 46 -> 42).
constexpr int kCus = 256;

template <int WA, int WB, int GA, int GB, bool WIDE, int OUT>
__global__ __launch_bounds__(64 * GA * GB, 2) void expert_tiled(ProductArgs p, GroupArgs g, int na) {
    constexpr int BA = 16 * WA * GA, BB = 16 * WB * GB;
    constexpr bool kHalves = GA * GB == 8;
    uint32_t before, upto;
    int per, ta, tb;
    group_scan<BB>(g, before, upto, per);
    const int nb = readlane_u32(upto, 63), tiles = na * nb, last = tiles % kCus;
    const int whole = kHalves && last <= kCus / 2 ? tiles - last : tiles, rest = 2 * (tiles - whole);
    int block = blockIdx.x, half = 0;
    if (block >= whole + rest) return;
    const bool split = block >= whole;
    if (split) {
        block = xcd_remap(block - whole, rest);
        half = block % 2;
        block = whole + block / 2;
    } else {
        block = xcd_remap(block, whole);
    }
    tile_at(block, na, nb, ta, tb);
    const GroupTile t = group_tile<BB>(g, tb, before, upto, per);
    const int a0 = ta * BA + half * (BA / 2);
    if (a0 >= p.M) return;   // the second half of a tile of fewer features
    if (t.row >= t.real) {
        zero_tile<OUT>(p.out, p.M, a0, min(a0 + (split ? BA / 2 : BA), p.M), t.row, t.end);
        return;
    }
    __shared__ __attribute__((aligned(1024))) uint8_t lds[lds_tile_bytes<WA, WB, GA, GB>];
    // the last rows of a group in a tile of half as many (10400 rows in 32 groups, 4096 x 2048: 130 -> 124 us;
    // 32768 tokens, 32 of 4096 x 7168: 1 %)
    if constexpr (BB == 256) {
        if (t.end - t.row <= 128) {
            if (split) lds_tile<4, 2, 2, 4, 0, WIDE, OUT, true, true>(lds, of_expert(p, g, t), a0, t.row, 0, p.Kp / 128, t.end);
            else lds_tile<4, 4, 4, 2, 0, WIDE, OUT, true, true>(lds, of_expert(p, g, t), a0, t.row, 0, p.Kp / 128, t.end);
            return;
        }
    }
    if constexpr (kHalves) {
        if (split) {
            lds_tile<WA / 2, WB, GA, GB, 0, WIDE, OUT, true, (BB >= 128)>(lds, of_expert(p, g, t), a0, t.row, 0, p.Kp / 128, t.end);
            return;
        }
    }
    lds_tile<WA, WB, GA, GB, 0, WIDE, OUT, true, (BB >= 128)>(lds, of_expert(p, g, t), a0, t.row, 0, p.Kp / 128, t.end);
}

template <int RA, int TB, int W, bool WIDE, int OUT>
__global__ __launch_bounds__(64 * W) void expert_direct(ProductArgs p, GroupArgs g) {
    constexpr int BA = 16 * RA, BB = 16 * TB;
    uint32_t before, upto;
    int per;
    group_scan<BB>(g, before, upto, per);
    const uint32_t tb = blockIdx.y, ta = blockIdx.x;
    if (tb >= readlane_u32(upto, 63)) return;
    const GroupTile t = group_tile<BB>(g, tb, before, upto, per);
    if (t.row >= t.real) {
        zero_tile<OUT>(p.out, p.M, ta * BA, min(static_cast<int>(ta + 1) * BA, p.M), t.row, t.end);
        return;
    }
    direct_tile<RA, TB, W, 0, 0, WIDE, OUT, true>(of_expert(p, g, t), ta * BA, t.row, 0, p.Kp / 128, t.end);
}

// Groups of few rows lie a few hundred bytes wide in each row of the column forms.  Read as their tiles come, memory serves every
// row's piece by itself: 128 experts of 1536 x 2048, 1500 tokens, float32: 442 us, 305 where the forms are in the cache already.
// So the experts are taken in runs of kAheadExperts, and in front of a run's tiles some workgroups read the next run's
// columns, a kilobyte and more of every row, into the cache that the XCDs share (through LDS, where nobody reads them): 358 us.
// Runs of 16 and 32 gave 358 and 367 (4096 x 7168, 64 experts here: 1076, 1120 and 1196 for 8, 16 and 32); 4 leave XCDs
// without patches.  32 workgroups that read ahead and 64 or 128: alike.
constexpr int kAheadExperts = 8, kAheadBlocks = 32;
__device__ __forceinline__ void columns_ahead(const ProductArgs &p, const GroupArgs &g, int e0, int index, uint8_t *lds) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), waves = blockDim.x / 64;
    if (e0 >= g.n) return;
    const int first = group_start(g, e0), bytes = group_start(g, min(e0 + kAheadExperts, g.n)) - first;   // a multiple of 128
    if (bytes <= 0) return;
    const uint32_t to = lds_address(lds) + wave * 1024;
    for (int row = index * waves + wave; row < p.M + p.R; row += kAheadBlocks * waves) {
        const uint8_t *from = (row < p.M ? p.a + static_cast<size_t>(row) * p.Kp : p.b + static_cast<size_t>(row - p.M) * p.Kp) + first;
        for (int at = 0; at < bytes; at += 1024) dma16(from, min(at + 16 * lane_id(), bytes - 16), to);
    }
    wait_vmcnt<0>();
}

// Patches of up to 4 B tiles by all A tiles go over the XCDs in turn: groups of unlike sizes then keep all of them busy.  An
// expert's patches are alike: 6 B tiles as 4 and 2 in place of 3 and 3 give some XCDs twice the work of others (64
// experts of 1408 x 2048, mean 96 and 512 rows: 125 and 209 us, 105 and 173).
__host__ __device__ __forceinline__ int grad_bands(int nb) { return (nb + 3) / 4; }

template <int WA, int WB, int GA, int GB, bool WIDE, int OUT, bool AHEAD>
__global__ __launch_bounds__(64 * GA * GB, 2) void expert_grad(ProductArgs p, GroupArgs g, int na, int nb) {
    constexpr int BA = 16 * WA * GA, BB = 16 * WB * GB;
    __shared__ __attribute__((aligned(1024))) uint8_t lds[lds_tile_bytes<WA, WB, GA, GB>];   // 1 KB a wave at least
    const int bands = grad_bands(nb), wide = (nb + bands - 1) / bands;
    int block = blockIdx.x, e0 = 0, experts = g.n;
    if constexpr (AHEAD) {
        const int tiles = (kAheadExperts * bands + 7) / 8 * 8 * wide * na, run = block / (kAheadBlocks + tiles);
        block -= run * (kAheadBlocks + tiles);
        e0 = run * kAheadExperts;
        experts = min(kAheadExperts, g.n - e0);
        if (block < kAheadBlocks) {
            columns_ahead(p, g, e0 + kAheadExperts, block, lds);
            return;
        }
        block -= kAheadBlocks;
    }
    const int i = block / 8, turn = i / (wide * na), at = i - turn * (wide * na);
    const int patch = turn * 8 + block % 8, of = patch / bands, band = patch - of * bands, bw = min(wide, nb - band * wide);
    if (of >= experts || at >= bw * na) return;
    const int e = e0 + of, ta = at / bw, tb = band * wide + at % bw;
    int o = 0, blocks = 0;   // without tables there are no rows
    if (g.off) {
        o = group_start(g, e);
        blocks = (min(max(g.count[e], 0), max(group_start(g, e + 1) - o, 0)) + 127) / 128;
    }
    p.out = static_cast<uint8_t *>(p.out) + static_cast<size_t>(e) * p.R * p.M * (OUT == 0 ? 2 : 4);
    if (blocks == 0) {
        if constexpr (OUT != 2) zero_tile<OUT>(p.out, p.M, ta * BA, min((ta + 1) * BA, p.M), tb * BB, min((tb + 1) * BB, p.R));
        return;
    }
    lds_tile<WA, WB, GA, GB, 1, WIDE, OUT, false, true>(lds, p, ta * BA, tb * BB, o / 128, o / 128 + blocks, 0);
}

// Most tiles of bb rows that the groups can make: each is a multiple of align rows, and their sum is within the rows.
static long most_tiles(const GroupArgs &g, long pairs, int bb) {
    const long rows = std::min<long>(g.rows, (pairs + std::min<long>(g.n, pairs) * (g.align - 1)) / g.align * g.align);
    if (bb <= g.align) return rows / bb;
    const long groups = std::min<long>(std::min<long>(g.n, pairs), rows / g.align);
    return (rows + groups * (bb - g.align)) / bb;
}

template <int WA, int WB, int GA, int GB, bool WIDE, int OUT>
static void tiled(const ProductArgs &p, const GroupArgs &g, long pairs, hipStream_t s) {
    const int na = (p.M + 16 * WA * GA - 1) / (16 * WA * GA);
    const long nb = most_tiles(g, pairs, 16 * WB * GB);
    hipLaunchKernelGGL((expert_tiled<WA, WB, GA, GB, WIDE, OUT>), dim3(na * nb + (GA * GB == 8 ? kCus / 2 : 0)), dim3(64 * GA * GB), 0, s, p, g, na);
}
template <int RA, int TB, int W, bool WIDE, int OUT>
static void direct(const ProductArgs &p, const GroupArgs &g, long pairs, hipStream_t s) {
    const int na = (p.M + 16 * RA - 1) / (16 * RA);
    const long nb = most_tiles(g, pairs, 16 * TB);
    hipLaunchKernelGGL((expert_direct<RA, TB, W, WIDE, OUT>), dim3(na, nb), dim3(64 * W), 0, s, p, g);
}

// Which kernel, by the rows that a group holds on average.  In order: direct 32 x 16; through LDS 128 x 64, 128 x 128,
// 256 x 128, 256 x 256 (us):
//   128 experts of 1536 x 2048, bf16    mean 1: 43.8 46.5 47.9 - 70.6;  4: 69.4 75.7 79.9 - 110;  8: 84.9 82.3 85.8 - 113;
//                                       32: 169 89.7 93.6 - 140;  64: 333 126 109 104 132;  128: - 153 125 121 138
//   64 of 1536 x 2048, bf16             192: - - 80.7 78.0 88.0;  256: - - 95.3 91.6 91.3;  320: - - 110 109 104;  384: - - 126 121 110
//   32 of 4096 x 2048, bf16             192: - - 104 102 103;  256: - - 120 121 110;  384: - - 169 166 144;  1024: - - 370 354 310
//   32 of 2048 x 7168, bf16             192: - - 175 158 169;  256: - - 203 190 195;  320: - - 235 212 212;  512: - - 339 313 275
//   128 of 1536 x 2048, float32         mean 1: 45.1 52.1 63.2;  4: 73.5 84.7 103;  16: 112 97.8 117;  64: 336 151 142 151
// Where the tiles of 128 x 128 fill the card no more than twice, or are odd in number along the features, the larger ones lose:
// 8 of 576 x 4096, mean 1024: 34.1 50.9 49.6; 16 of 400 x 1040, mean 64: 10.8 13.5 18.8.  Direct tiles of 16 x 16, 16 x 32,
// 32 x 32 and 64 x 16, of 4 and 8 waves, and 64 x 64 and 128 x 256 through LDS were never more than 2 % better.
template <bool WIDE, int OUT>
static hipError_t product(const ProductArgs &p, const GroupArgs &g, long pairs, float mean, hipStream_t s) {
    const int a128 = (p.M + 127) / 128;
    const float small = static_cast<float>(a128) * g.n * std::ceil(mean / 128);                                   // tiles of 128 x 128
    const float largest = static_cast<float>((p.M + 255) / 256) * g.n * std::ceil(mean / 256);   // of 256 x 256
    if (mean <= 6) {
        direct<2, 1, 4, WIDE, OUT>(p, g, pairs, s);
    } else if (mean <= 48) {
        tiled<4, 2, 2, 2, WIDE, OUT>(p, g, pairs, s);
    } else if constexpr (WIDE) {
        tiled<4, 4, 2, 2, WIDE, OUT>(p, g, pairs, s);
    } else {
        if (mean >= 256 && largest >= 192) tiled<8, 4, 2, 4, WIDE, OUT>(p, g, pairs, s);
        else if (a128 % 2 == 0 && small >= 512) tiled<4, 4, 4, 2, WIDE, OUT>(p, g, pairs, s);
        else tiled<4, 4, 2, 2, WIDE, OUT>(p, g, pairs, s);
    }
    return hipGetLastError();
}

hipError_t launch_expert_product(const ProductArgs &p, const GroupArgs &g, long pairs, float mean, int out, hipStream_t s) {
    return out == 0 ? product<false, 0>(p, g, pairs, mean, s) : product<true, 1>(p, g, pairs, mean, s);
}

template <int WA, int WB, int GA, int GB, bool WIDE, int OUT>
static void grad(const ProductArgs &p, const GroupArgs &g, bool ahead, hipStream_t s) {
    const int na = (p.M + 16 * WA * GA - 1) / (16 * WA * GA), nb = (p.R + 16 * WB * GB - 1) / (16 * WB * GB), bands = grad_bands(nb);
    const int wide = (nb + bands - 1) / bands;
    auto tiles = [&](int experts) { return (experts * bands + 7) / 8 * 8 * wide * na; };
    if (ahead) {
        const int runs = (g.n + kAheadExperts - 1) / kAheadExperts;
        hipLaunchKernelGGL((expert_grad<WA, WB, GA, GB, WIDE, OUT, true>), dim3(runs * (kAheadBlocks + tiles(kAheadExperts))), dim3(64 * GA * GB), 0, s, p, g, na, nb);
    } else {
        hipLaunchKernelGGL((expert_grad<WA, WB, GA, GB, WIDE, OUT, false>), dim3(tiles(g.n)), dim3(64 * GA * GB), 0, s, p, g, na, nb);
    }
}

// bf16: 256 x 256 where three rounds of the CUs are full or one nearly is, as one such tile of 1 to 64 steps reads half of
// what four of 128 x 128 do (64 experts of 2048 x 1536, mean 16, 96, 512 and 1024 rows: 99 111 178 258 us, 128 x 128:
// 118 131 202 294).  Fewer tiles leave CUs without work in the last round (64 of 512 x 768, mean 512 and 1024: 45 and
// 76 us, 128 x 128: 43 and 62; 16 of 1024 x 1024, mean 1024: 49 and 42), and so do results that cover
// less than 3/4 of their tiles (128 of 128 x 2048, mean 12, 96 and 384: 36 45 81 us, 128 x 128: 31 38 70; of 384 x 2048: 66 77 124
// and 69 77 117; of 640 x 2048, 5/6: 94 114 189 and 115 130 192).  float32 results, whose operands are widened in registers:
// 128 x 128 was best of 128 x 64, 256 x 64, 128 x 256 and 256 x 128 (128 of 1536 x 2048, mean 94: 417 us, the last two 432 and 467).
// Reading ahead gains up to some 512 rows a group (32 of 4096 x 7168, mean 48, 256, 512 and 1024: 635 657 827 1151 us without,
// 545 572 761 1144 with it) and from two runs of experts on (8 to 15 experts: alike, or slower).
hipError_t launch_expert_weight_grad(const ProductArgs &p, const GroupArgs &g, float mean, int out, hipStream_t s) {
    const bool ahead = g.off && g.n >= 2 * kAheadExperts && mean <= 1024;
    const float largest = static_cast<float>((p.M + 255) / 256) * ((p.R + 255) / 256) * g.n;   // tiles of 256 x 256
    const bool full = (largest >= 768 || (largest > 128 && largest <= 224)) && static_cast<float>(p.M) * p.R * g.n >= 0.75f * 65536 * largest;
    if (out == 0 && full) grad<8, 4, 2, 4, false, 0>(p, g, ahead, s);
    else if (out == 0) grad<4, 4, 2, 2, false, 0>(p, g, ahead, s);
    else if (out == 1) grad<4, 4, 2, 2, true, 1>(p, g, ahead, s);
    else grad<4, 4, 2, 2, true, 2>(p, g, ahead, s);
    return hipGetLastError();
}

}  // namespace ftmoe
