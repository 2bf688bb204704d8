// Dense product over 8-bit operands, one scale per block of 128 along the reduction:
//
//   out[b][a] = sum_kb sA(a, kb) sB(b, kb) sum_{k in block kb} A[a][k] B[b][k]
//
// with e4m3fn codes A [M][Kp], B [R][Kp].  ft_linear: A is the weight (float32 scale per 128 x 128 block)
// and B the activations (e8m0 scale per row and block), out = y [T][N].  ft_linear_weight_grad: A is the
// column form of x, B that of dy (e8m0 scales both), the reduction runs over the tokens, out = dW [N][K].
// The arithmetic and the kernels are in product_tile.h.
#include "product_tile.h"

#include <algorithm>
#include <cmath>

namespace ftmoe {

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
// W^T of a block-scaled weight: codes [N][Kp] -> [K][Np], codes of the padding columns 0; one 128 x 128 block per
// workgroup through LDS, so that whole lines are read and written, and its scale.  A thread turns the codes of
// 16 rows and 4 columns, 4 x 4 at a time.  Bound: HBM; 4096 x 7168 in
// 10.9 us, 5.4 TB/s; 64 x 64 blocks and a byte at a time 15.6.
__global__ __launch_bounds__(256) void weight_transpose(const uint8_t *w, const float *s, uint8_t *wt, float *st, int N,
                                                        int K, int Np, int Kp) {
    __shared__ uint32_t tile[128][33];
    const int t = threadIdx.x, kb = blockIdx.x, nb = blockIdx.y, k0 = kb * 128, n0 = nb * 128;
    // weight blockIdx.z of several
    w += static_cast<size_t>(blockIdx.z) * N * Kp;
    s += static_cast<size_t>(blockIdx.z) * (Np / 128) * (Kp / 128);
    wt += static_cast<size_t>(blockIdx.z) * K * Np;
    st += static_cast<size_t>(blockIdx.z) * (Kp / 128) * (Np / 128);
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

hipError_t launch_weight_transpose(const uint8_t *w, const float *s, uint8_t *wt, float *st, int n, int N, int K, hipStream_t stream) {
    const int Np = pad128(N), Kp = pad128(K);
    hipLaunchKernelGGL(weight_transpose, dim3(Kp / 128, Np / 128, n), dim3(256), 0, stream, w, s, wt, st, N, K, Np, Kp);
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
