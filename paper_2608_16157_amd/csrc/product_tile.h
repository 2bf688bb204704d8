// Kernels of the 8-bit products (linear.hip, expert_products.hip); internal.
//
//   out[b][a] = sum_kb sA(a, kb) sB(b, kb) sum_{k in block kb} A[a][k] B[b][k]
//
// with e4m3fn codes A [M][Kp], B [R][Kp] and one scale per block of 128 along the reduction.
//
// Arithmetic.  bf16 results come from the fp8 matrix instructions, which take the e8m0 scales in their
// scale operands.  Measured with single products at chosen places: the instruction aligns the products of each group
// of 8 consecutive codes to the largest exponent among them (the sum of the operands' exponents; a subnormal code
// has that of 2^-6) and keeps what lies at or above 2^-13 of it; groups and blocks are then added in float32, and the
// accumulator takes no part in the alignment.  So a sum is off by up to 7 * 2^-13 of each group's largest product
// (8.4e-4 of the sum of magnitudes reached), eight times that where it comes from a subnormal code (6.3e-3 reached),
// which is not bounded by the result where terms cancel.  Over a whole matrix it is 1.5e-5 to 1.8e-5 of the
// result's norm for normally distributed operands and up to 6e-5 where magnitudes span 2^8 and more, without growth
// with the length; bf16's rounding is 1.7e-3 by that measure.  float32 results, whose readers expect
// more, widen the codes to bf16 with their power-of-two scale, which is exact (but 2^128, which bf16 cannot
// hold), and use the bf16 instructions, whose products and sums are exact to float32's rounding (1e-7 measured), at
// half the rate.  A float32 weight scale multiplies the finished float32 sum of its block in either case.
#pragma once

#include "act_codes.h"
#include "ftmoe_internal.h"
#include "gemm_tile.h"

#include <type_traits>

namespace ftmoe {

__device__ __forceinline__ i32x8_vec_t codes32(const uint8_t *p) {
    const uint4 lo = reinterpret_cast<const uint4 *>(p)[0], hi = reinterpret_cast<const uint4 *>(p)[4];
    return i32x8_vec_t{static_cast<int>(lo.x), static_cast<int>(lo.y), static_cast<int>(lo.z), static_cast<int>(lo.w),
                       static_cast<int>(hi.x), static_cast<int>(hi.y), static_cast<int>(hi.z), static_cast<int>(hi.w)};
}

// 16 x 16 products over one block of 128, scaled by e8m0, added to z (WIDE: the arithmetic of float32 results)
template <bool WIDE>
__device__ __forceinline__ floatx4_t block_product(i32x8_vec_t a, int sa, i32x8_vec_t b, int sb, floatx4_t z) {
    if constexpr (WIDE) {
#pragma unroll
        for (int q = 0; q < 4; ++q)
            z = __builtin_amdgcn_mfma_f32_16x16x32_bf16(act_bf16x8(a[2 * q], a[2 * q + 1], act_scale_operand(sa)),
                                                        act_bf16x8(b[2 * q], b[2 * q + 1], act_scale_operand(sb)), z, 0, 0, 0);
        return z;
    } else {
        return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, z, 0, 0, 0, sa, 0, sb);
    }
}

// four consecutive results: 0 bf16 (rounded once, to nearest even), 1 float32, 2 added to the float32 there
template <int OUT>
__device__ __forceinline__ void store4(void *out, size_t at, floatx4_t v) {
    if constexpr (OUT == 0) {
        *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(out) + at) =
            uint2{f32_to_bf16_any(v[0]) | f32_to_bf16_any(v[1]) << 16, f32_to_bf16_any(v[2]) | f32_to_bf16_any(v[3]) << 16};
    } else {
        floatx4_t *o = reinterpret_cast<floatx4_t *>(static_cast<float *>(out) + at);
        *o = OUT == 2 ? *o + v : v;
    }
}

// The reduction may be split over the grid's third dimension: each part sums its blocks into float32 rows of
// its own in the workspace (p.part), which product_join adds in order.
__device__ __forceinline__ void split_range(const ProductArgs &p, int nkb, int &kb0, int &kb1) {
    kb0 = static_cast<int>(static_cast<long>(nkb) * blockIdx.z / gridDim.z);
    kb1 = static_cast<int>(static_cast<long>(nkb) * (blockIdx.z + 1) / gridDim.z);
}
__device__ __forceinline__ void *split_out(const ProductArgs &p) {
    return p.part ? p.part + static_cast<size_t>(blockIdx.z) * p.R * p.M : p.out;
}

// Direct kernel: operands from global memory to registers, the reduction split over the waves of a
// workgroup and joined in LDS in a fixed order.  A wave holds 16 RA rows of A and 16 TB rows of B; lane
// (r = lane % 16, g = lane / 16) 32 codes of row r of a block, [16 g, 16 g + 16) and the same 64 further on.
// BX: 0 B is codes; 1 B is bf16, 2 float32: then every workgroup first brings the few rows into 8 bits in LDS
// (the same in all of them: cheaper than a launch for up to kDirectTokens rows, kDirectBytes of codes).  ASC: 0 float32 block scales, 1 e8m0.
// WIDE: the arithmetic of float32 results.  OUT: see store4.
// Bound: one read of the weight, and at these times the launch and the chain of load, product and join:
// 1 x 4096 x 7168 with its quantiser 7.7 us, 3.8 TB/s; 32 x 7168 x 2048 7.2 us.  Two more blocks requested ahead
// by every wave were no faster, in a loop that waits on memory in other places too: as compiled, the second B
// operand is requested after the first has been used, and a block's float32 scale where it is applied.
// Tile at rows a0 of A and b0 of B, blocks [kb0, kb1).  GROUPED: the rows from p.R up to `end` are stored as zeros.
template <int RA, int TB, int W, int ASC, int BX, bool WIDE, int OUT, bool GROUPED>
__device__ __forceinline__ void direct_tile(ProductArgs p, int a0, int b0, int kb0, int kb1, int end) {
    constexpr int kTile = RA * TB * 256;
    static_assert(BX == 0 || TB == 1, "quantised rows fit one operand");
    __shared__ float red[W / 2][kTile];
    extern __shared__ __attribute__((aligned(16))) uint8_t s_codes[];   // the rows' codes and behind them their scales
    uint8_t *s_scales = s_codes + static_cast<size_t>(p.R) * p.Kp;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = lane_id();
    const int r = lane & 15, g = lane >> 4;
    const int nkb = p.Kp / 128;
    floatx4_t acc[RA][TB];
#pragma unroll
    for (int i = 0; i < RA; ++i)
#pragma unroll
        for (int j = 0; j < TB; ++j) acc[i][j] = floatx4_t{};
    const uint8_t *ap[RA];
#pragma unroll
    for (int i = 0; i < RA; ++i) ap[i] = p.a + static_cast<size_t>(min(a0 + 16 * i + r, p.M - 1)) * p.Kp + 16 * g;
    int brow[TB];
#pragma unroll
    for (int j = 0; j < TB; ++j) brow[j] = min(b0 + 16 * j + r, p.R - 1);
    i32x8_vec_t ahead[RA];   // the weight's next block, where the rows are quantised here
    auto request = [&](int kb) {
#pragma unroll
        for (int i = 0; i < RA; ++i) ahead[i] = codes32(ap[i] + static_cast<size_t>(kb) * 128);
    };
    if constexpr (BX != 0) {
        // One lane row of 16 lanes per row and block, 8 values a lane, three blocks on the way at a time.  The weight's
        // first block is requested behind the first of them, which must not wait for it: loads return in order.
        // (1 x 7168 x 2048: 5.7 -> 5.2 us; two and four blocks of the weight ahead 5.5 and 7.1.)
        using XT = std::conditional_t<BX == 1, uint16_t, float>;
        constexpr int kOnWay = 3, kLaneRows = 4 * W;
        const int sub = threadIdx.x % 16, n = p.R * nkb;
        float v[kOnWay][8];
        auto load = [&](int first) {
#pragma unroll
            for (int q = 0; q < kOnWay; ++q) {
                const int i = min(first + q * kLaneRows, n - 1), row = i / nkb, k = (i - row * nkb) * 128 + 8 * sub;
                load8(static_cast<const XT *>(p.x) + static_cast<size_t>(row) * p.K + min(k, p.K - 8), v[q]);
            }
        };
        int first = threadIdx.x / 16;
        load(first);
        __builtin_amdgcn_sched_barrier(0);
        request(min(kb0 + wave, kb1 - 1));
        __builtin_amdgcn_sched_barrier(0);
        while (first < n) {
#pragma unroll
            for (int q = 0; q < kOnWay; ++q) {
                const int i = first + q * kLaneRows;
                if (i >= n) break;
                quiet(v[q]);
                if (i % nkb * 128 + 8 * sub >= p.K)   // K is a multiple of 16
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[q][e] = 0.0f;
                const int byte = act_scale_byte(block_mag16(v[q]));
                const float sc = act_scale_operand(byte);
                *reinterpret_cast<uint2 *>(s_codes + i * 128 + 8 * sub) =
                    uint2{act_codes4(v[q][0], v[q][1], v[q][2], v[q][3], sc), act_codes4(v[q][4], v[q][5], v[q][6], v[q][7], sc)};
                if (sub == 0) s_scales[i] = static_cast<uint8_t>(byte);
            }
            first += kOnWay * kLaneRows;
            if (first < n) load(first);
        }
        __syncthreads();
    }
    for (int kb = kb0 + wave; kb < kb1; kb += W) {
        i32x8_vec_t a[RA], b[TB];
        int sb[TB];
#pragma unroll
        for (int i = 0; i < RA; ++i) a[i] = BX ? ahead[i] : codes32(ap[i] + static_cast<size_t>(kb) * 128);
        if (BX && kb + W < kb1) request(kb + W);
#pragma unroll
        for (int j = 0; j < TB; ++j) {
            if constexpr (BX == 0) {
                b[j] = codes32(p.b + static_cast<size_t>(brow[j]) * p.Kp + static_cast<size_t>(kb) * 128 + 16 * g);
                sb[j] = p.bs[static_cast<size_t>(kb) * p.bsr + brow[j]];
            } else {
                b[j] = codes32(s_codes + (brow[j] * nkb + kb) * 128 + 16 * g);
                sb[j] = s_scales[brow[j] * nkb + kb];
            }
        }
#pragma unroll
        for (int i = 0; i < RA; ++i) {
            float sw = 1.0f;
            int sa = 127;
            if constexpr (ASC == 0) sw = static_cast<const float *>(p.as)[static_cast<size_t>(min(a0 + 16 * i, p.M - 1) / 128) * nkb + kb];
            else sa = static_cast<const uint8_t *>(p.as)[static_cast<size_t>(kb) * p.asr + min(a0 + 16 * i + r, p.M - 1)];
#pragma unroll
            for (int j = 0; j < TB; ++j) {
                const floatx4_t z = block_product<WIDE>(a[i], sa, b[j], sb[j], ASC == 0 ? floatx4_t{} : acc[i][j]);
                // a weight block with scale 0 adds nothing, whatever its codes and the rows hold
                if constexpr (ASC == 0)
#pragma unroll
                    for (int q = 0; q < 4; ++q) acc[i][j][q] = fmaf(sw, sw == 0.0f ? 0.0f : z[q], acc[i][j][q]);
                else acc[i][j] = z;
            }
        }
    }
    // join the waves: W/2 give their sums to the others, until one holds the tile
#pragma unroll
    for (int s = W / 2; s >= 1; s /= 2) {
        if (wave >= s && wave < 2 * s)
#pragma unroll
            for (int i = 0; i < RA; ++i)
#pragma unroll
                for (int j = 0; j < TB; ++j)
                    *reinterpret_cast<floatx4_t *>(&red[wave - s][((i * TB + j) * 64 + lane) * 4]) = acc[i][j];
        __syncthreads();
        if (wave < s)
#pragma unroll
            for (int i = 0; i < RA; ++i)
#pragma unroll
                for (int j = 0; j < TB; ++j)
                    acc[i][j] += *reinterpret_cast<const floatx4_t *>(&red[wave][((i * TB + j) * 64 + lane) * 4]);
        __syncthreads();
    }
    if (wave) return;
    // element q of a 16 x 16 tile in lane (r, g): row 4 g + q of A, row r of B
#pragma unroll
    for (int j = 0; j < TB; ++j) {
        const int b = b0 + 16 * j + r;
        if (b >= (GROUPED ? end : p.R)) continue;
#pragma unroll
        for (int i = 0; i < RA; ++i) {
            const int a = a0 + 16 * i + 4 * g;
            if (GROUPED && b >= p.R) acc[i][j] = floatx4_t{};
            if (a < p.M) store4<OUT>(split_out(p), static_cast<size_t>(b) * p.M + a, acc[i][j]);   // M is a multiple of 16
        }
    }
}

template <int RA, int TB, int W, int ASC, int BX, bool WIDE, int OUT>
__global__ __launch_bounds__(64 * W) void product_direct(ProductArgs p) {
    int kb0, kb1;
    split_range(p, p.Kp / 128, kb0, kb1);
    direct_tile<RA, TB, W, ASC, BX, WIDE, OUT, false>(p, blockIdx.x * 16 * RA, blockIdx.y * 16 * TB, kb0, kb1, 0);
}

// One 16 x 16 tile at (a0, b0) by one wave from global memory, without the weight blocks of scale 0.
template <bool WIDE, int OUT, bool GROUPED>
__device__ __forceinline__ void again(const ProductArgs &p, int a0, int b0, int k0, int k1, int end) {
    const int lane = lane_id(), r = lane & 15, g = lane >> 4, nkb = p.Kp / 128;
    if (a0 >= p.M) return;   // M is a multiple of 16
    const int row = min(b0 + r, p.R - 1);
    const uint8_t *pa = p.a + static_cast<size_t>(a0 + r) * p.Kp + 16 * g, *pb = p.b + static_cast<size_t>(row) * p.Kp + 16 * g;
    const float *scale = static_cast<const float *>(p.as) + static_cast<size_t>(a0 / 128) * nkb;
    floatx4_t acc{};
#pragma unroll 1
    for (int kb = k0; kb < k1; ++kb) {
        const float f = scale[kb];
        if (f == 0.0f) continue;
        const size_t at = static_cast<size_t>(kb) * 128;
        const floatx4_t z = block_product<WIDE>(codes32(pa + at), 127, codes32(pb + at), p.bs[kb * static_cast<size_t>(p.bsr) + row], floatx4_t{});
#pragma unroll
        for (int q = 0; q < 4; ++q) acc[q] = fmaf(f, z[q], acc[q]);
    }
    if (GROUPED && b0 + r >= p.R) acc = floatx4_t{};
    if (b0 + r < (GROUPED ? end : p.R)) store4<OUT>(split_out(p), static_cast<size_t>(b0 + r) * p.M + a0 + 4 * g, acc);
}

// Tiled kernel: a workgroup of GA x GB waves owns a tile of 16 WA GA rows of A by 16 WB GB rows of B, each
// wave 16 WA x 16 WB of it.  Blocks (128 codes of every row of both operands, and their e8m0 bytes) go from
// global memory straight into LDS; 16-byte chunks lie XOR-swizzled by their row, so that the operand
// reads of 16 consecutive rows meet no bank twice.  A wave keeps the block's B operands in registers and
// walks the A operands, one per step: each step reads the next A operand while the matrix instructions of
// the current one run, and the float32 scale of the sums before is applied between them.
//
// B's place in LDS is free as soon as the block's operands are in registers, A's half by half, so B lies in
// a ring of two blocks and A in one of five half blocks, and everything is requested about two blocks
// before it is read.  The two hand-offs of a block, in the last step of each half: wait for what the next
// step reads (requests return in order, so the younger ones may stay in flight) and for this wave's own
// LDS reads, barrier, and request into the freed places between the step's matrix instructions.
//
// What bounds it, at 8192 x 4096 x 7168 (201 us, 2390 TFLOP/s; the library's largest fp8 product, without
// block scales, reaches 3110, and 2800 at this size): the matrix units are busy 0.65 of the time inside the
// loop, at a clock of 1.85 to 2.0 GHz, where power holds it (2.4 when it does not).  What takes the rest, timed by
// leaving it out: issuing the requests 30 us, the barriers 15, the float32 scale of every sum 20; waiting for
// data 2 and its way through L2 (81 % hits, two patches of tiles compared) nothing.  32 x 32 instructions,
// behind which the scale hides whole, draw more power: 206 us at the same busy share and a lower clock.
// Tile at rows a0 of A and b0 of B, blocks [k0, k1), k1 > k0.  GROUPED: the rows from p.R up to `end` are stored as zeros.
// STREAM: the results' stores do not stay in the caches.
// lds: lds_tile_bytes, aligned to 1024.
template <int WA, int WB, int GA, int GB>
constexpr int lds_tile_bytes = 5 * 8 * WA * GA * 128 + 2 * 16 * WB * GB * 128 + 4 * 512;

template <int WA, int WB, int GA, int GB, int ASC, bool WIDE, int OUT, bool GROUPED, bool STREAM>
__device__ __forceinline__ void lds_tile(uint8_t *lds, ProductArgs p, int a0, int b0, int k0, int k1, int end) {
    constexpr bool kWide = WIDE;
    constexpr int NW = GA * GB, BA = 16 * WA * GA, BB = 16 * WB * GB, HS = WA / 2;   // HS steps per half
    constexpr int kHalf = BA / 2 * 128, kAHalves = 5, kBBlock = BB * 128;
    constexpr int kB = kAHalves * kHalf, kS = kB + 2 * kBBlock;     // LDS: A halves, B blocks, 4 blocks' scales
    constexpr int AH = BA / 2 / 8 / NW, BI = BB / 8 / NW;           // 1 KB requests per wave
    constexpr int kInFlight = 3 * AH + BI + 1;                      // younger than what a hand-off waits for
    static_assert(AH * 16 * NW == BA && BI * 8 * NW == BB && BA <= 256 && BB <= 256 && WA % 2 == 0 && kS + 4 * 512 == lds_tile_bytes<WA, WB, GA, GB>, "tile");
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = lane_id();
    const int r = lane & 15, g = lane >> 4, wa = wave % GA, wb = wave / GA;
    const int nkb = k1 - k0;   // blocks k0 .. k0 + nkb - 1 of the Kp / 128

    // requests: lane i of one fills 16 bytes of row i / 8 of its 8 rows, the chunk that belongs at place
    // i % 8.  Half H of an A block holds the rows of the steps [H HS, (H + 1) HS), 16 HS of each GA.
    const uint8_t *abase = p.a + static_cast<size_t>(a0) * p.Kp + static_cast<size_t>(k0) * 128;
    const uint8_t *bbase = p.b + static_cast<size_t>(b0) * p.Kp + static_cast<size_t>(k0) * 128;
    uint32_t aoff[2][AH], boff[BI];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < AH; ++i) {
            const int at = (wave * AH + i) * 8 + lane / 8;   // row of the half
            const int row = at / (16 * HS) * (16 * WA) + h * 16 * HS + at % (16 * HS);
            aoff[h][i] = static_cast<uint32_t>(min(row, p.M - 1 - a0)) * p.Kp + (swz<128>(at, lane % 8) << 4);
        }
#pragma unroll
    for (int i = 0; i < BI; ++i) {
        const int row = (wave * BI + i) * 8 + lane / 8;
        boff[i] = static_cast<uint32_t>(min(row, p.R - 1 - b0)) * p.Kp + (swz<128>(row, lane % 8) << 4);
    }
    // scales of a block: B's e8m0 bytes, and, asked for by the odd waves, A's, or the float32 scales of the
    // tile's one or two weight blocks (32 copies each: every lane of a request brings one word).  Every
    // wave asks, the same words to the same place: a branch here would split the loop's body, which the
    // compiler then reorders.
    const bool sa_wave = wave & 1;
    const size_t srow = sa_wave ? (ASC ? p.asr : 4) : p.bsr;
    const uint8_t *sbase = (sa_wave ? static_cast<const uint8_t *>(p.as) : p.bs) + k0 * srow;
    const int sdst = sa_wave ? 256 : 0;
    const uint32_t soff = !sa_wave ? min(b0 + 4 * lane, p.bsr - 4)
                          : ASC    ? min(a0 + 4 * lane, p.asr - 4)
                                   : static_cast<uint32_t>(min(a0 / 128 + lane / 32, (p.M - 1) / 128)) * (p.Kp / 128) * 4;
    const uint32_t l0 = lds_address(lds);
    // the first requests repeat the last block where there are fewer
    auto request_a = [&](auto half, auto i, int kb, int slot) {
        constexpr int H = decltype(half)::value, I = decltype(i)::value;
        dma16(abase + static_cast<size_t>(min(kb, nkb - 1)) * 128, aoff[H][I], l0 + slot + (wave * AH + I) * 1024);
    };
    auto request_b = [&](auto i, int kb) {
        constexpr int I = decltype(i)::value;
        const int k = min(kb, nkb - 1);
        if constexpr (I < BI) dma16(bbase + static_cast<size_t>(k) * 128, boff[I], l0 + kB + (kb & 1) * kBBlock + (wave * BI + I) * 1024);
        else dma4(sbase + static_cast<size_t>(k) * srow, soff, l0 + kS + (kb & 3) * 512 + sdst);
    };
    // operand reads: chunks g and g + 4 of row r of a 16-row tile (which codes of the block a lane holds is free
    // as long as A and B agree).  Chunks 2 g and 2 g + 1 would meet banks twice: 123 against 221 B/clk.
    const int chunk = swz<128>(r, g) << 4, other = (chunk ^ 64) - chunk;
    const uint8_t *la = lds + (wa * HS * 16 + r) * 128 + chunk, *lb = lds + kB + (wb * WB * 16 + r) * 128 + chunk;
    const uint8_t *lbs = lds + kS + wb * WB * 16 + r, *las = lds + kS + 256 + wa * WA * 16 + r;
    auto operand = [&](const uint8_t *q) {
        const u32x4_t lo = *reinterpret_cast<const u32x4_t *>(q), hi = *reinterpret_cast<const u32x4_t *>(q + other);
        return i32x8_vec_t{static_cast<int>(lo[0]), static_cast<int>(lo[1]), static_cast<int>(lo[2]), static_cast<int>(lo[3]),
                           static_cast<int>(hi[0]), static_cast<int>(hi[1]), static_cast<int>(hi[2]), static_cast<int>(hi[3])};
    };
    const uint8_t *lws = lds + kS + 256 + wa * WA * 16 / 128 * 128;
    auto weight_scale = [&](int slot) { return ASC ? 1.0f : *reinterpret_cast<const float *>(lws + slot); };

    constexpr int kLag = WB;   // sums in flight between a matrix instruction and its scale
    floatx4_t acc[WA][WB], z[kLag];
#pragma unroll
    for (int i = 0; i < WA; ++i)
#pragma unroll
        for (int j = 0; j < WB; ++j) acc[i][j] = floatx4_t{};
#pragma unroll
    for (int j = 0; j < kLag; ++j) z[j] = floatx4_t{};
    i32x8_vec_t a, b[WB];
    int sa = 127, sb[WB];
    bf16x8_t bwide[kWide ? WB : 1][4];

    auto all_a = [&](auto half, int kb, int slot) { static_for<0, AH>([&](auto i) { request_a(half, i, kb, slot); }); };
    auto all_b = [&](int kb) { static_for<0, BI + 1>([&](auto i) { request_b(i, kb); }); };
    all_a(ic<0>{}, 0, 0);
    all_b(0);
    all_a(ic<1>{}, 0, kHalf);
    all_a(ic<0>{}, 1, 2 * kHalf);
    all_b(1);
    all_a(ic<1>{}, 1, 3 * kHalf);
    all_a(ic<0>{}, 2, 4 * kHalf);
    wait_vmcnt<4 * AH + BI + 1>();
    stage_barrier();
    a = operand(la);
    if (ASC) sa = las[0];
#pragma unroll
    for (int j = 0; j < WB; ++j) {
        b[j] = operand(lb + j * 2048);
        sb[j] = lbs[16 * j];
    }
    float sw = weight_scale(0), swz_old = 0.0f;   // weight scale of this block, and of the sums in z
    uint32_t least = 1;                           // 0 once a weight scale was 0
    int s0 = 0;                                   // A slot of the block's first half
    auto after = [&](int slot) { return slot + kHalf == kAHalves * kHalf ? 0 : slot + kHalf; };
    // one block; `more`: there are blocks to request
    auto block = [&](int kb, auto more) {
        constexpr bool kMore = decltype(more)::value;
        const int s1 = after(s0), s2 = after(s1), bn = ((kb + 1) & 1) * kBBlock, sn = ((kb + 1) & 3) * 512;
        float sw_next = sw;
        if constexpr (kWide)
#pragma unroll
            for (int j = 0; j < WB; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q) bwide[j][q] = act_bf16x8(b[j][2 * q], b[j][2 * q + 1], act_scale_operand(sb[j]));
        static_for<0, WA>([&](auto ii) {
            constexpr int I = decltype(ii)::value, P = (I + WA - 1) % WA, N = (I + 1) % WA;
            constexpr bool kMid = I == HS - 1, kLast = I == WA - 1;
            constexpr bool kHandOff = kMid || kLast;
            i32x8_vec_t an;
            int san = 127;
            auto hand_off = [&] {
                wait_vmcnt<kMore ? kInFlight : 0>();
                wait_lgkmcnt0();
                stage_barrier();
            };
            auto read_next = [&] {
                an = operand(la + (kLast ? s2 : N < HS ? s0 : s1) + N % HS * 2048);
                if constexpr (kLast) sw_next = weight_scale(sn);
                if (ASC) san = las[kLast ? sn : (kb & 3) * 512 + N * 16];
            };
            // the requests into the places that a hand-off freed, spread over the steps up to the next one:
            // behind matrix instruction J of this step
            auto requests = [&](auto jj) {
                constexpr int J = decltype(jj)::value, M = BI + 1 + AH;
                if constexpr (kMore) static_for<0, M>([&](auto i) {
                    constexpr int Q = decltype(i)::value;
                    if constexpr (Q * HS * WB / M == (I - (HS - 1)) * WB + J) {
                        if constexpr (Q <= BI) request_b(i, kb + 2);
                        else request_a(ic<1>{}, ic<Q - BI - 1>{}, kb + 2, s0);
                    }
                });
                if constexpr (kMore && kLast)
                    static_for<0, AH>([&](auto i) {
                        if constexpr (decltype(i)::value * WB / AH == J) request_a(ic<0>{}, i, kb + 3, s1);
                    });
            };
            if constexpr (kWide) {
                if constexpr (kHandOff) hand_off();
                static_for<0, WB>(requests);
            }
            if constexpr (kWide || !kHandOff) read_next();
            if constexpr (kWide) {
                floatx4_t zn[WB];
#pragma unroll
                for (int j = 0; j < WB; ++j) zn[j] = ASC ? acc[I][j] : floatx4_t{};
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const bf16x8_t aw = act_bf16x8(a[2 * q], a[2 * q + 1], act_scale_operand(sa));
#pragma unroll
                    for (int j = 0; j < WB; ++j) zn[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(aw, bwide[j][q], zn[j], 0, 0, 0);
                }
                if constexpr (kLast) {
#pragma unroll
                    for (int j = 0; j < WB; ++j) {
                        b[j] = operand(lb + bn + j * 2048);
                        sb[j] = lbs[sn + 16 * j];
                    }
                }
#pragma unroll
                for (int j = 0; j < WB; ++j) {
                    if constexpr (ASC) {
                        acc[I][j] = zn[j];
                    } else {
#pragma unroll
                        for (int q = 0; q < 4; ++q) acc[P][j][q] = fmaf(I == 0 ? swz_old : sw, z[j][q], acc[P][j][q]);
                        z[j] = zn[j];
                    }
                }
            } else {
                // in program order: one matrix instruction, the scale of the sums kLag instructions back, and
                // in the last step the next block's operand into the registers the instruction has just
                // read.  A hand-off comes behind the step's first instruction, which covers it.
                __builtin_amdgcn_sched_barrier(0);
                static_for<0, WB>([&](auto jj) {
                    constexpr int J = decltype(jj)::value;
                    if constexpr (ASC) {
                        acc[I][J] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b[J], acc[I][J], 0, 0, 0, sa, 0, sb[J]);
                    } else {
                        constexpr int T = I * WB + J, F = (T + WA * WB - kLag) % (WA * WB);
                        const float f = T < kLag ? swz_old : sw;
#pragma unroll
                        for (int q = 0; q < 4; ++q)
                            acc[F / WB][F % WB][q] = fmaf(f, z[F % kLag][q], acc[F / WB][F % WB][q]);
                        z[T % kLag] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b[J], floatx4_t{}, 0, 0, 0, sa, 0, sb[J]);
                    }
                    if constexpr (kHandOff && J == 0) {
                        __builtin_amdgcn_sched_barrier(0);
                        hand_off();
                        read_next();
                    }
                    requests(jj);
                    if constexpr (kLast) {
                        b[J] = operand(lb + bn + J * 2048);
                        sb[J] = lbs[sn + 16 * J];
                    }
                    __builtin_amdgcn_sched_barrier(0);
                });
            }
            a = an;
            sa = san;
        });
        if (!ASC) least = min(least, __float_as_uint(sw) << 1);
        swz_old = sw;
        sw = sw_next;
        s0 = s2;
    };
    int kb = 0;
    for (; kb < nkb - 2; ++kb) block(kb, ic<1>{});
    for (; kb < nkb; ++kb) block(kb, ic<0>{});
    wait_vmcnt<0>();
    if constexpr (!ASC)
#pragma unroll
        for (int j = 0; j < WB; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q) acc[WA - 1][j][q] = fmaf(swz_old, z[j][q], acc[WA - 1][j][q]);
    // Through LDS, 16 rows of B at a time and each wave by itself, so that whole lines leave: as the sums lie in
    // the registers, a store would write 32 bytes of each of 16 rows (8192 x 4096 results: 28 us for K = 128 against 21).
    constexpr int kSize = OUT == 0 ? 2 : 4, kRow = 16 * WA * kSize, kPitch = kRow + 16, kLanes = kRow / 16;
    static_assert(16 * kPitch * NW <= kS + 4 * 512, "epilogue");
    stage_barrier();   // every wave has read its last operands, and its requests have landed
    // A weight block with scale 0 adds nothing, whatever its codes and the rows that meet them hold.  Where those are
    // finite its product was 0 already; where a sum is NaN the wave forms its sums again without such blocks, in the
    // same order, straight from global memory.  (In the loop it would take a branch around a block, whose two sides
    // spill, or an instruction more for every sum.)
    if constexpr (!ASC) {
        static_assert(128 % (16 * WA) == 0, "a wave's rows of A lie in one weight block");
        bool nan = false;
        if (__builtin_expect(__builtin_amdgcn_readfirstlane(least) == 0, 0))
#pragma unroll
            for (int i = 0; i < WA; ++i)
#pragma unroll
                for (int j = 0; j < WB; ++j)
#pragma unroll
                    for (int q = 0; q < 4; ++q) nan |= acc[i][j][q] != acc[i][j][q];
        if (__builtin_expect(__ballot(nan) != 0, 0)) {
#pragma unroll 1
            for (int t = 0; t < WA * WB; ++t)
                again<WIDE, OUT, GROUPED>(p, a0 + (wa * WA + t / WB) * 16, b0 + (wb * WB + t % WB) * 16, k0, k1, end);
            return;
        }
    }
    uint8_t *mine = lds + wave * 16 * kPitch;
#pragma unroll
    for (int j = 0; j < WB; ++j) {
#pragma unroll
        for (int i = 0; i < WA; ++i) {
            uint8_t *at = mine + r * kPitch + (16 * i + 4 * g) * kSize;
            if constexpr (OUT == 0 && (GROUPED || STREAM))
                *reinterpret_cast<uint2 *>(at) = uint2{bf16_pair(acc[i][j][0], acc[i][j][1]), bf16_pair(acc[i][j][2], acc[i][j][3])};
            else if constexpr (OUT == 0)
                *reinterpret_cast<uint2 *>(at) = uint2{f32_to_bf16_any(acc[i][j][0]) | f32_to_bf16_any(acc[i][j][1]) << 16,
                                                       f32_to_bf16_any(acc[i][j][2]) | f32_to_bf16_any(acc[i][j][3]) << 16};
            else *reinterpret_cast<floatx4_t *>(at) = acc[i][j];
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");   // a wave's own LDS operations execute in order
        const int ai = a0 + wa * WA * 16 + lane % kLanes * (16 / kSize);   // M is a multiple of 16
#pragma unroll
        for (int q = 0; q < 16; q += 64 / kLanes) {
            const int row = q + lane / kLanes, bi = b0 + (wb * WB + j) * 16 + row;
            u32x4_t v = *reinterpret_cast<const u32x4_t *>(mine + row * kPitch + lane % kLanes * 16);
            if (GROUPED && bi >= p.R) v = u32x4_t{};
            if (bi < (GROUPED ? end : p.R) && ai < p.M) {
                u32x4_t *o = reinterpret_cast<u32x4_t *>(static_cast<uint8_t *>(split_out(p)) + (static_cast<size_t>(bi) * p.M + ai) * kSize);
                if constexpr (OUT == 2) *reinterpret_cast<floatx4_t *>(o) += __builtin_bit_cast(floatx4_t, v);
                else if constexpr (STREAM) __builtin_nontemporal_store(v, o);
                else *o = v;
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
}

// Tile L of na x nb: tiles that run at the same time on one XCD form a patch of kBand B tiles by some A tiles.
__device__ __forceinline__ void tile_at(int L, int na, int nb, int &ta, int &tb) {
    constexpr int kBand = 4;
    const int band = L / (kBand * na), rem = L - band * (kBand * na);
    const int bw = min(kBand, nb - band * kBand);
    ta = rem / bw;
    tb = band * kBand + rem % bw;
}

template <int WA, int WB, int GA, int GB, int ASC, bool WIDE, int OUT>
__global__ __launch_bounds__(64 * GA * GB, 2) void product_tiled(ProductArgs p, int na, int nb) {
    int ta, tb, k0, k1;
    tile_at(xcd_remap(blockIdx.x, na * nb), na, nb, ta, tb);
    split_range(p, p.Kp / 128, k0, k1);
    __shared__ __attribute__((aligned(1024))) uint8_t lds[lds_tile_bytes<WA, WB, GA, GB>];
    lds_tile<WA, WB, GA, GB, ASC, WIDE, OUT, false, false>(lds, p, ta * 16 * WA * GA, tb * 16 * WB * GB, k0, k1, 0);
}

}  // namespace ftmoe
