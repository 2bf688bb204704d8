// Dense product over 8-bit operands, one scale per block of 128 along the reduction:
//
//   out[b][a] = sum_kb sA(a, kb) sB(b, kb) sum_{k in block kb} A[a][k] B[b][k]
//
// with e4m3fn codes A [M][Kp], B [R][Kp].  ft_linear: A is the weight (float32 scale per 128 x 128 block)
// and B the activations (e8m0 scale per row and block), out = y [T][N].  ft_linear_weight_grad: A is the
// column form of x, B that of dy (e8m0 scales both), the reduction runs over the tokens, out = dW [N][K].
//
// Arithmetic.  bf16 results come from the fp8 matrix instructions, which take the e8m0 scales in their
// scale operands.  Their sums of 128 products carry an error of about 2^-16 of the result (measured
// against 64 bits: 1.5e-5 to 1.8e-5, no bias, no growth with the length, the same for every fp8 shape of
// the unit), a hundredth of bf16's own rounding.  float32 results, whose readers expect more, widen the
// codes to bf16 with their power-of-two scale, which is exact, and use the bf16 instructions, whose
// products and sums are exact to float32's rounding (1e-7 measured), at half the rate.  A float32 weight
// scale multiplies the finished float32 sum of its block in either case.
#include "act_codes.h"
#include "ftmoe_internal.h"

#include <type_traits>

namespace ftmoe {

__device__ __forceinline__ i32x8_vec_t codes32(const uint8_t *p) {
    const uint4 lo = reinterpret_cast<const uint4 *>(p)[0], hi = reinterpret_cast<const uint4 *>(p)[1];
    return i32x8_vec_t{static_cast<int>(lo.x), static_cast<int>(lo.y), static_cast<int>(lo.z), static_cast<int>(lo.w),
                       static_cast<int>(hi.x), static_cast<int>(hi.y), static_cast<int>(hi.z), static_cast<int>(hi.w)};
}

// four consecutive results: bf16 (rounded once, to nearest even), float32, or added to the float32 there
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

// Direct kernel: operands from global memory to registers, the reduction split over the waves of a
// workgroup and joined in LDS in a fixed order.  A wave holds 16 RA rows of A and 16 TB rows of B; lane
// (r = lane % 16, g = lane / 16) the 32 codes [32 g, 32 g + 32) of row r of a block.
// BX: 0 B is codes; 1 B is bf16, 2 float32, quantised on the way.  ASC: 0 float32 block scales, 1 e8m0.
// OUT: 0 bf16, 1 float32, 2 float32 added to what is there.
template <int RA, int TB, int W, int ASC, int BX, int OUT>
__global__ __launch_bounds__(64 * W) void product_direct(ProductArgs p) {
    constexpr bool kWide = OUT != 0;
    constexpr int kTile = RA * TB * 256;
    __shared__ float red[W / 2][kTile];
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
    for (int i = 0; i < RA; ++i) ap[i] = p.a + static_cast<size_t>(min(a0 + 16 * i + r, p.M - 1)) * p.Kp + 32 * g;
    int brow[TB];
#pragma unroll
    for (int j = 0; j < TB; ++j) brow[j] = min(b0 + 16 * j + r, p.R - 1);

    for (int kb = wave; kb < nkb; kb += W) {
        i32x8_vec_t a[RA], b[TB];
        int sb[TB];
#pragma unroll
        for (int i = 0; i < RA; ++i) a[i] = codes32(ap[i] + static_cast<size_t>(kb) * 128);
#pragma unroll
        for (int j = 0; j < TB; ++j) {
            if constexpr (BX == 0) {
                b[j] = codes32(p.b + static_cast<size_t>(brow[j]) * p.Kp + static_cast<size_t>(kb) * 128 + 32 * g);
                sb[j] = p.bs[static_cast<size_t>(kb) * p.bsr + brow[j]];
            } else {
                using XT = std::conditional_t<BX == 1, uint16_t, float>;
                const XT *x = static_cast<const XT *>(p.x) + static_cast<size_t>(brow[j]) * p.K;
                float v[32];
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int k = kb * 128 + 32 * g + 8 * q;
                    if (k < p.K) load8(x + k, v + 8 * q);   // K is a multiple of 16
                    else
#pragma unroll
                        for (int e = 0; e < 8; ++e) v[8 * q + e] = 0.0f;
                }
                uint32_t m = 0;
#pragma unroll
                for (int e = 0; e < 32; ++e) m = max(m, act_mag_bits(v[e]));
                m = max(m, static_cast<uint32_t>(__shfl_xor(static_cast<int>(m), 16)));
                m = max(m, static_cast<uint32_t>(__shfl_xor(static_cast<int>(m), 32)));
                sb[j] = act_scale_byte(m);
                const float sc = act_scale_operand(sb[j]);
#pragma unroll
                for (int q = 0; q < 8; ++q) b[j][q] = static_cast<int>(act_codes4(v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3], sc));
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
                floatx4_t z = ASC == 0 ? floatx4_t{} : acc[i][j];
                if constexpr (kWide) {
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        z = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                            act_bf16x8(a[i][2 * q], a[i][2 * q + 1], act_scale_operand(sa)),
                            act_bf16x8(b[j][2 * q], b[j][2 * q + 1], act_scale_operand(sb[j])), z, 0, 0, 0);
                } else {
                    z = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a[i], b[j], z, 0, 0, 0, sa, 0, sb[j]);
                }
                if constexpr (ASC == 0)
#pragma unroll
                    for (int q = 0; q < 4; ++q) acc[i][j][q] = fmaf(sw, z[q], acc[i][j][q]);
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
            if (a < p.M) store4<OUT>(p.out, static_cast<size_t>(b) * p.M + a, acc[i][j]);   // M is a multiple of 16
        }
    }
}

// W^T of a block-scaled weight: codes [N][Kp] -> [K][Np], codes of the padding columns 0; one 64 x 64 tile
// per workgroup through LDS, and the block scales transposed by the first workgroup row.
__global__ __launch_bounds__(256) void weight_transpose(const uint8_t *w, const float *s, uint8_t *wt, float *st, int N,
                                                        int K, int Np, int Kp) {
    __shared__ uint32_t tile[64][17];
    const int t = threadIdx.x, k0 = blockIdx.x * 64, n0 = blockIdx.y * 64;
    const int nb = Np / 128, kb = Kp / 128;
    // scales: spread over the grid
    const long total = static_cast<long>(gridDim.x) * gridDim.y * 256;
    for (long i = (static_cast<long>(blockIdx.y) * gridDim.x + blockIdx.x) * 256 + t; i < static_cast<long>(nb) * kb; i += total)
        st[i] = s[(i % nb) * kb + i / nb];
    {
        const int row = t / 4, c = t % 4;   // 16 bytes a thread
        uint4 v = {0, 0, 0, 0};
        if (n0 + row < N) v = *reinterpret_cast<const uint4 *>(w + static_cast<size_t>(n0 + row) * Kp + k0 + 16 * c);
        tile[row][4 * c] = v.x;
        tile[row][4 * c + 1] = v.y;
        tile[row][4 * c + 2] = v.z;
        tile[row][4 * c + 3] = v.w;
    }
    __syncthreads();
    const int k = t / 4, c = t % 4;
    if (k0 + k < K) {
        uint32_t o[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            o[q] = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) o[q] |= ((tile[16 * c + 4 * q + e][k / 4] >> (8 * (k % 4))) & 0xFFu) << (8 * e);
        }
        *reinterpret_cast<uint4 *>(wt + static_cast<size_t>(k0 + k) * Np + n0 + 16 * c) = uint4{o[0], o[1], o[2], o[3]};
    }
}

hipError_t launch_weight_transpose(const uint8_t *w, const float *s, uint8_t *wt, float *st, int N, int K, hipStream_t stream) {
    const int Np = pad128(N), Kp = pad128(K);
    hipLaunchKernelGGL(weight_transpose, dim3(Kp / 64, Np / 64), dim3(256), 0, stream, w, s, wt, st, N, K, Np, Kp);
    return hipGetLastError();
}

template <int ASC, int BX, int OUT>
static hipError_t direct(const ProductArgs &p, hipStream_t s) {
    if (p.R <= 16) {
        hipLaunchKernelGGL((product_direct<1, 1, 8, ASC, BX, OUT>), dim3((p.M + 15) / 16, 1), dim3(512), 0, s, p);
    } else if constexpr (BX == 0) {
        hipLaunchKernelGGL((product_direct<4, 4, 4, ASC, BX, OUT>), dim3((p.M + 63) / 64, (p.R + 63) / 64), dim3(256), 0, s, p);
    }
    return hipGetLastError();
}

hipError_t launch_product(const ProductArgs &p, bool a_e8m0, int bx, int out, hipStream_t s) {
    if (a_e8m0) {
        if (out == 0) return direct<1, 0, 0>(p, s);
        if (out == 1) return direct<1, 0, 1>(p, s);
        return direct<1, 0, 2>(p, s);
    }
    if (bx == 0) return out == 0 ? direct<0, 0, 0>(p, s) : direct<0, 0, 1>(p, s);
    if (bx == 1) return out == 0 ? direct<0, 1, 0>(p, s) : direct<0, 1, 1>(p, s);
    return out == 0 ? direct<0, 2, 0>(p, s) : direct<0, 2, 1>(p, s);
}

}  // namespace ftmoe
