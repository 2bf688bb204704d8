// Dense product over 8-bit operands, one scale per block of 128 along the reduction:
//
//   out[b][a] = sum_kb sA(a, kb) sB(b, kb) sum_{k in block kb} A[a][k] B[b][k]
//
// with e4m3fn codes A [M][Kp], B [R][Kp].  ft_linear: A is the weight (float32 scale per 128 x 128 block)
// and B the activations (e8m0 scale per row and block), out = y [T][N].  ft_linear_weight_grad: A is the
// column form of x, B that of dy (e8m0 scales both), the reduction runs over the tokens, out = dW [N][K].
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
#include "act_codes.h"
#include "ftmoe_internal.h"
#include "gemm_tile.h"

#include <algorithm>
#include <cmath>
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

// Bound: the parts' bytes, mostly still in the caches: with its launch 1.9 us and 5.4 TB/s over write and read.
template <int OUT>
__global__ __launch_bounds__(256) void product_join(ProductArgs p, int parts) {
    const size_t n = static_cast<size_t>(p.R) * p.M, i = (static_cast<size_t>(blockIdx.x) * 256 + threadIdx.x) * 4;
    if (i >= n) return;
    floatx4_t v = *reinterpret_cast<const floatx4_t *>(p.part + i);
    for (int z = 1; z < parts; z += 4) {   // four parts on the way at a time; behind the last one it again, unused
        floatx4_t part[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) part[q] = *reinterpret_cast<const floatx4_t *>(p.part + min(z + q, parts - 1) * n + i);
#pragma unroll
        for (int q = 0; q < 4; ++q)
            if (z + q < parts) v += part[q];
    }
    store4<OUT>(p.out, i, v);
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
template <int RA, int TB, int W, int ASC, int BX, bool WIDE, int OUT>
__global__ __launch_bounds__(64 * W) void product_direct(ProductArgs p) {
    constexpr int kTile = RA * TB * 256;
    static_assert(BX == 0 || TB == 1, "quantised rows fit one operand");
    __shared__ float red[W / 2][kTile];
    extern __shared__ __attribute__((aligned(16))) uint8_t s_codes[];   // the rows' codes and behind them their scales
    uint8_t *s_scales = s_codes + static_cast<size_t>(p.R) * p.Kp;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = lane_id();
    const int r = lane & 15, g = lane >> 4;
    const int a0 = blockIdx.x * 16 * RA, b0 = blockIdx.y * 16 * TB;
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
    int kb0, kb1;
    split_range(p, nkb, kb0, kb1);
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
        if (b >= p.R) continue;
#pragma unroll
        for (int i = 0; i < RA; ++i) {
            const int a = a0 + 16 * i + 4 * g;
            if (a < p.M) store4<OUT>(split_out(p), static_cast<size_t>(b) * p.M + a, acc[i][j]);   // M is a multiple of 16
        }
    }
}

// One 16 x 16 tile at (a0, b0) by one wave from global memory, without the weight blocks of scale 0.
template <bool WIDE, int OUT>
__device__ __forceinline__ void again(const ProductArgs &p, int a0, int b0, int k0, int k1) {
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
    if (b0 + r < p.R) store4<OUT>(split_out(p), static_cast<size_t>(b0 + r) * p.M + a0 + 4 * g, acc);
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
template <int WA, int WB, int GA, int GB, int ASC, bool WIDE, int OUT>
__global__ __launch_bounds__(64 * GA * GB, 2) void product_tiled(ProductArgs p, int na, int nb) {
    constexpr bool kWide = WIDE;
    constexpr int NW = GA * GB, BA = 16 * WA * GA, BB = 16 * WB * GB, HS = WA / 2;   // HS steps per half
    constexpr int kHalf = BA / 2 * 128, kAHalves = 5, kBBlock = BB * 128;
    constexpr int kB = kAHalves * kHalf, kS = kB + 2 * kBBlock;     // LDS: A halves, B blocks, 4 blocks' scales
    constexpr int AH = BA / 2 / 8 / NW, BI = BB / 8 / NW;           // 1 KB requests per wave
    constexpr int kInFlight = 3 * AH + BI + 1;                      // younger than what a hand-off waits for
    static_assert(AH * 16 * NW == BA && BI * 8 * NW == BB && BA <= 256 && BB <= 256 && WA % 2 == 0, "tile");
    __shared__ __attribute__((aligned(1024))) uint8_t lds[kS + 4 * 512];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = lane_id();
    const int r = lane & 15, g = lane >> 4, wa = wave % GA, wb = wave / GA;
    // tiles that run at the same time on one XCD form a patch of kBand B tiles by some A tiles
    constexpr int kBand = 4;
    const int L = xcd_remap(blockIdx.x, na * nb);
    const int band = L / (kBand * na), rem = L - band * (kBand * na);
    const int bw = min(kBand, nb - band * kBand);
    const int a0 = rem / bw * BA, b0 = (band * kBand + rem % bw) * BB;
    int k0, k1;
    split_range(p, p.Kp / 128, k0, k1);
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
    static_assert(16 * kPitch * NW <= sizeof(lds), "epilogue");
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
                again<WIDE, OUT>(p, a0 + (wa * WA + t / WB) * 16, b0 + (wb * WB + t % WB) * 16, k0, k1);
            return;
        }
    }
    uint8_t *mine = lds + wave * 16 * kPitch;
#pragma unroll
    for (int j = 0; j < WB; ++j) {
#pragma unroll
        for (int i = 0; i < WA; ++i) {
            uint8_t *at = mine + r * kPitch + (16 * i + 4 * g) * kSize;
            if constexpr (OUT == 0)
                *reinterpret_cast<uint2 *>(at) = uint2{f32_to_bf16_any(acc[i][j][0]) | f32_to_bf16_any(acc[i][j][1]) << 16,
                                                       f32_to_bf16_any(acc[i][j][2]) | f32_to_bf16_any(acc[i][j][3]) << 16};
            else *reinterpret_cast<floatx4_t *>(at) = acc[i][j];
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");   // a wave's own LDS operations execute in order
        const int ai = a0 + wa * WA * 16 + lane % kLanes * (16 / kSize);   // M is a multiple of 16
#pragma unroll
        for (int q = 0; q < 16; q += 64 / kLanes) {
            const int row = q + lane / kLanes, bi = b0 + (wb * WB + j) * 16 + row;
            const u32x4_t v = *reinterpret_cast<const u32x4_t *>(mine + row * kPitch + lane % kLanes * 16);
            if (bi < p.R && ai < p.M) {
                u32x4_t *o = reinterpret_cast<u32x4_t *>(static_cast<uint8_t *>(split_out(p)) + (static_cast<size_t>(bi) * p.M + ai) * kSize);
                if constexpr (OUT == 2) *reinterpret_cast<floatx4_t *>(o) += __builtin_bit_cast(floatx4_t, v);
                else *o = v;
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
}

// W^T of a block-scaled weight: codes [N][Kp] -> [K][Np], codes of the padding columns 0; one 128 x 128 block per
// workgroup through LDS, so that whole lines are read and written, and its scale.  A thread turns the codes of
// 16 rows and 4 columns, 4 x 4 at a time.  Bound: HBM; 4096 x 7168 in
// 10.9 us, 5.4 TB/s; 64 x 64 blocks and a byte at a time 15.6.
__global__ __launch_bounds__(256) void weight_transpose(const uint8_t *w, const float *s, uint8_t *wt, float *st, int N,
                                                        int K, int Np, int Kp) {
    __shared__ uint32_t tile[128][33];
    const int t = threadIdx.x, kb = blockIdx.x, nb = blockIdx.y, k0 = kb * 128, n0 = nb * 128;
    if (t == 0) st[static_cast<size_t>(kb) * (Np / 128) + nb] = s[static_cast<size_t>(nb) * (Kp / 128) + kb];
    uint4 v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {   // 16 bytes a thread of 32 rows; past the last row it again, dropped below
        const int row = min(n0 + t / 8 + 32 * i, N - 1);
        v[i] = *reinterpret_cast<const uint4 *>(w + static_cast<size_t>(row) * Kp + k0 + 16 * (t % 8));
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint32_t *to = &tile[t / 8 + 32 * i][4 * (t % 8)];
        const bool in = n0 + t / 8 + 32 * i < N;
        to[0] = in ? v[i].x : 0;
        to[1] = in ? v[i].y : 0;
        to[2] = in ? v[i].z : 0;
        to[3] = in ? v[i].w : 0;
    }
    __syncthreads();
    const int c = t % 8, k4 = t / 8;   // rows 16 c and on of W, columns 4 k4 and on
    uint32_t o[4][4];                  // [column][rows 4 q and on]
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const uint32_t a = tile[16 * c + 4 * q][k4], b = tile[16 * c + 4 * q + 1][k4], d = tile[16 * c + 4 * q + 2][k4],
                       e = tile[16 * c + 4 * q + 3][k4];
        // bytes 0 to 3 of the second operand are 0 to 3, of the first 4 to 7
        const uint32_t ab0 = __builtin_amdgcn_perm(b, a, 0x05010400u), ab1 = __builtin_amdgcn_perm(b, a, 0x07030602u);
        const uint32_t de0 = __builtin_amdgcn_perm(e, d, 0x05010400u), de1 = __builtin_amdgcn_perm(e, d, 0x07030602u);
        o[0][q] = __builtin_amdgcn_perm(de0, ab0, 0x05040100u);
        o[1][q] = __builtin_amdgcn_perm(de0, ab0, 0x07060302u);
        o[2][q] = __builtin_amdgcn_perm(de1, ab1, 0x05040100u);
        o[3][q] = __builtin_amdgcn_perm(de1, ab1, 0x07060302u);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (k0 + 4 * k4 + i < K)
            *reinterpret_cast<uint4 *>(wt + static_cast<size_t>(k0 + 4 * k4 + i) * Np + n0 + 16 * c) =
                uint4{o[i][0], o[i][1], o[i][2], o[i][3]};
}

hipError_t launch_weight_transpose(const uint8_t *w, const float *s, uint8_t *wt, float *st, int N, int K, hipStream_t stream) {
    const int Np = pad128(N), Kp = pad128(K);
    hipLaunchKernelGGL(weight_transpose, dim3(Kp / 128, Np / 128), dim3(256), 0, stream, w, s, wt, st, N, K, Np, Kp);
    return hipGetLastError();
}

template <int WA, int WB, int GA, int GB, int ASC, bool WIDE, int OUT>
static void tiled(const ProductArgs &p, int parts, hipStream_t s) {
    const int na = (p.M + 16 * WA * GA - 1) / (16 * WA * GA), nb = (p.R + 16 * WB * GB - 1) / (16 * WB * GB);
    hipLaunchKernelGGL((product_tiled<WA, WB, GA, GB, ASC, WIDE, OUT>), dim3(na * nb, 1, parts), dim3(64 * GA * GB), 0, s, p, na, nb);
}

template <int RA, int TB, int W, int ASC, int BX, bool WIDE, int OUT>
static void direct(const ProductArgs &p, int parts, hipStream_t s) {
    // only as much LDS as the rows take: more workgroups to a CU
    const unsigned lds = BX ? p.R * p.Kp / 128 * 129 : 0;
    hipLaunchKernelGGL((product_direct<RA, TB, W, ASC, BX, WIDE, OUT>),
                       dim3((p.M + 16 * RA - 1) / (16 * RA), (p.R + 16 * TB - 1) / (16 * TB), parts), dim3(64 * W), lds, s, p);
}

template <int ASC, int BX, bool WIDE, int OUT>
static void variant(const ProductArgs &p, const ProductPlan &plan, hipStream_t s) {
    if constexpr (BX != 0) {
        direct<1, 1, 8, ASC, BX, WIDE, OUT>(p, 1, s);
    } else {
        switch (plan.kernel) {
            case ProductPlan::kDirect16: direct<1, 1, 8, ASC, BX, WIDE, OUT>(p, plan.parts, s); break;
            case ProductPlan::kDirect32: direct<1, 2, 8, ASC, BX, WIDE, OUT>(p, plan.parts, s); break;
            case ProductPlan::kDirect64: direct<2, 2, 8, ASC, BX, WIDE, OUT>(p, plan.parts, s); break;
            case ProductPlan::kTile64: tiled<2, 2, 2, 2, ASC, WIDE, OUT>(p, plan.parts, s); break;
            case ProductPlan::kTile128x64: tiled<4, 2, 2, 2, ASC, WIDE, OUT>(p, plan.parts, s); break;
            case ProductPlan::kTile128: tiled<4, 4, 2, 2, ASC, WIDE, OUT>(p, plan.parts, s); break;
            case ProductPlan::kTile256:
                if constexpr (!WIDE) tiled<8, 4, 2, 4, ASC, WIDE, OUT>(p, plan.parts, s);
                break;
        }
    }
}

// Which kernel runs a product, and into how many parts its reduction is split: the least of their estimated
// times.  The estimate is a workgroup's blocks times what one takes (in microseconds, fitted to times on this
// card over ten weights, N from 512 to 8192, K from 512 to 18432, at 16 to 8192 rows, every kernel and eight splits
// of each: where the rule's choice is among those timed, 287 of 320 products, it is 0.5 % above the best of them
// in the mean, 10 % at the worst), as often as its workgroups outnumber the 256 CUs, plus the start and end of each
// round, plus the join of the parts:
//   direct kernels  the bytes of a block at 32.9 GB/s a CU (the waves of a CU share that rate), at least
//                   0.5 for every 8 blocks: a small reduction is one round trip to memory
//   tiled kernels   a block alone on its CU, and as a share of the CU's time; the second pair widened
//   join            1.9 and the parts' bytes, written and read, at 5.4 TB/s
// With M = 4096, K = 7168 (estimate / measured): 32 rows 10.6 / 12.2 (128 x 64, 8 parts), 64 x 64 in 4 parts
// 11.0 / 11.3, 16 x 32 direct 13.5 / 13.0; 256 rows 19.5 / 20.1 (128 x 64, 2 parts), 128 x 128 in 4 parts
// 20.2 / 19.6; 777 rows 32 / 34 (128 x 128), 128 x 64 39 / 37; 4096 rows 89 / 99 (256 x 256), 128 x 128 121 / 128.
ProductPlan product_plan(int M, int R, int Kp, bool wide, bool may_split) {
    struct Kind {
        ProductPlan::Kernel kernel;
        int a, b, most_rows;   // tile; rows up to which it is looked at
        float ends;            // start and end of a round
        int round;             // tiled kernels: workgroups a CU holds at once
        float alone, share, wide_alone, wide_share;
    };
    static constexpr Kind kinds[] = {{ProductPlan::kDirect16, 16, 16, 32, 2.7f},
                                     {ProductPlan::kDirect32, 16, 32, 64, 3.0f},
                                     {ProductPlan::kDirect64, 32, 32, 256, 4.0f},
                                     {ProductPlan::kTile64, 64, 64, 1 << 30, 4.5f, 4, 0.27f, 0.19f, 0.37f, 0.30f},
                                     {ProductPlan::kTile128x64, 128, 64, 1 << 30, 4.7f, 2, 0.35f, 0.31f, 0.55f, 0.53f},
                                     {ProductPlan::kTile128, 128, 128, 1 << 30, 5.4f, 2, 0.48f, 0.44f, 0.87f, 0.78f},
                                     {ProductPlan::kTile256, 256, 256, 1 << 30, 8.1f, 1, 0.97f, 1.40f}};
    const int nkb = Kp / 128;
    if (nkb == 0) return {ProductPlan::kDirect64, 1};   // no block: zeros are stored
    ProductPlan best{ProductPlan::kTile128, 1};
    float least = 1e30f;
    for (const Kind &k : kinds) {
        if (R > k.most_rows || (k.kernel == ProductPlan::kTile256 && wide)) continue;
        const float wgs = static_cast<float>((M + k.a - 1) / k.a) * static_cast<float>((R + k.b - 1) / k.b);
        for (int parts = 1; parts <= kMaxParts && parts <= nkb; ++parts) {
            if (parts > 1 && (!may_split || static_cast<size_t>(parts) * R * M * 4 > kSplitBytes)) break;
            const int blocks = (nkb + parts - 1) / parts;
            // workgroups of the fullest CU; behind the second round they even out
            const float mean = wgs * parts / 256.0f, cu = mean > 2 ? mean + 0.25f : std::ceil(mean);
            float t;
            if (k.kernel == ProductPlan::kTile256) {   // fills a CU: whole rounds, and slower the fuller the card
                const float full = std::min(mean, 1.0f);
                t = std::ceil(mean) * (blocks * (k.alone + (k.share - k.alone) * full) + k.ends + 2.5f * full);
            } else if (k.round) {
                t = blocks * (wide ? std::max(k.wide_alone, k.wide_share * cu) : std::max(k.alone, k.share * cu)) +
                    k.ends * std::ceil(cu / k.round);
            } else {
                t = std::max(cu * blocks * ((k.a + k.b) * 128) / 32900.0f, 0.5f * ((blocks + 7) / 8)) + k.ends;
            }
            if (parts > 1) t += 1.9f + static_cast<float>(parts) * R * M * 8 / 5.4e6f;
            if (t < least) {
                least = t;
                best = {k.kernel, parts};
            }
        }
    }
    return best;
}

template <int ASC, int BX, bool WIDE>
static hipError_t launch(ProductArgs p, int out, float *ws, hipStream_t s) {
    ProductPlan plan{ProductPlan::kDirect16, 1};   // the one that quantises on the way
    if (BX == 0) plan = product_plan(p.M, p.R, p.Kp, WIDE, ws != nullptr);
    if constexpr (ASC == 0 && BX == 0) {
        if (plan.parts > 1) {
            p.part = ws;
            variant<ASC, BX, WIDE, 1>(p, plan, s);
            const unsigned blocks = static_cast<unsigned>((static_cast<size_t>(p.R) * p.M / 4 + 255) / 256);
            hipLaunchKernelGGL((product_join<WIDE ? 1 : 0>), dim3(blocks), dim3(256), 0, s, p, plan.parts);
            return hipGetLastError();
        }
    }
    if constexpr (!WIDE) {
        variant<ASC, BX, WIDE, 0>(p, plan, s);
    } else if constexpr (ASC == 1) {
        if (out == 2) variant<ASC, BX, WIDE, 2>(p, plan, s);
        else variant<ASC, BX, WIDE, 1>(p, plan, s);
    } else {
        variant<ASC, BX, WIDE, 1>(p, plan, s);
    }
    return hipGetLastError();
}

hipError_t launch_product(const ProductArgs &p, bool a_e8m0, int bx, int out, float *ws, hipStream_t s) {
    if (a_e8m0) return out == 0 ? launch<1, 0, false>(p, out, ws, s) : launch<1, 0, true>(p, out, ws, s);
    if (bx == 0) return out == 0 ? launch<0, 0, false>(p, out, ws, s) : launch<0, 0, true>(p, out, ws, s);
    if (bx == 1) return out == 0 ? launch<0, 1, false>(p, out, ws, s) : launch<0, 1, true>(p, out, ws, s);
    return out == 0 ? launch<0, 2, false>(p, out, ws, s) : launch<0, 2, true>(p, out, ws, s);
}

}  // namespace ftmoe
