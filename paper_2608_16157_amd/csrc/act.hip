// Activations and gradients in 8 bits: the quantiser (row form, column form or both from one read) and the
// SwiGLU activation between two dense products, forward (its output and what the backward pass keeps, both
// in 8 bits) and backward (from what was kept).
//
// All of these move memory once and compute little: the bound is HBM.  A block of 128 values is one
// 16-lane row of a wave, 8 values a lane, so a row's block maximum needs only rotations within the lane
// row.  The column form needs a maximum over 128 rows and the transposed codes: a workgroup owns a tile of
// 128 x 128 elements, each thread a patch of 4 rows x 8 columns, so that the codes of 4 rows of a column
// leave as one word through LDS and both forms store whole 128-byte lines.
#include "act_codes.h"
#include "ftmoe_internal.h"

namespace ftmoe {

constexpr int kActThreads = 512;   // a tile: 32 lane rows of 16 lanes, 4 matrix rows each
constexpr int kActRows = 4;
constexpr int kTPad = 132;         // bytes of a transposed row of the tile in LDS

struct ActTileShared {
    uint32_t colmax[kActThreads / 16][128];
    uint8_t t[128 * kTPad];
    uint8_t rowscale[128];
    uint8_t colscale[128];
};

// One block of a row by one lane row of 16 lanes, 8 values a lane; rows past T (zeros, up to f.Rp) leave only
// their scale byte.
__device__ __forceinline__ void put_row(const float (&v)[8], const ActForm &f, long row, int T, int kb, int sub) {
    const int byte = act_scale_byte(block_mag16(v));
    const float sc = act_scale_operand(byte);
    if (row < T)
        *reinterpret_cast<uint2 *>(f.codes + static_cast<size_t>(row) * f.Kp + kb * 128 + 8 * sub) =
            uint2{act_codes4(v[0], v[1], v[2], v[3], sc), act_codes4(v[4], v[5], v[6], v[7], sc)};
    if (sub == 0) f.scales[static_cast<size_t>(kb) * f.Rp + row] = static_cast<uint8_t>(byte);
}

// Row form of a tile: v holds rows 4 g .. 4 g + 3 (g = the thread's lane row), columns 8 sub .. + 7.
__device__ __forceinline__ void tile_rows(const float (&v)[kActRows][8], ActTileShared &sh, const ActForm &f, int row0,
                                          int kb, int g, int sub) {
#pragma unroll
    for (int r = 0; r < kActRows; ++r) {
        const int byte = act_scale_byte(block_mag16(v[r]));
        const float sc = act_scale_operand(byte);
        const int row = row0 + kActRows * g + r;
        if (row < f.R) {
            const uint2 w = {act_codes4(v[r][0], v[r][1], v[r][2], v[r][3], sc),
                             act_codes4(v[r][4], v[r][5], v[r][6], v[r][7], sc)};
            *reinterpret_cast<uint2 *>(f.codes + static_cast<size_t>(row) * f.Kp + kb * 128 + 8 * sub) = w;
        }
        if (sub == 0) sh.rowscale[kActRows * g + r] = static_cast<uint8_t>(byte);
    }
    __syncthreads();
    // rows past the last one are zeros here: their scale byte is 127
    if (threadIdx.x < 8)
        reinterpret_cast<uint4 *>(f.scales + static_cast<size_t>(kb) * f.Rp + row0)[threadIdx.x] =
            reinterpret_cast<const uint4 *>(sh.rowscale)[threadIdx.x];
}

// Column form of a tile: matrix columns become rows col0 .. of f, the tile's 128 matrix rows its block kb.
__device__ __forceinline__ void tile_cols(const float (&v)[kActRows][8], ActTileShared &sh, const ActForm &f, int col0,
                                          int kb, int g, int sub) {
    const int t = threadIdx.x;
#pragma unroll
    for (int c = 0; c < 8; ++c) {
        uint32_t m = 0;
#pragma unroll
        for (int r = 0; r < kActRows; ++r) m = max(m, act_mag_bits(v[r][c]));
        sh.colmax[g][8 * sub + c] = m;
    }
    __syncthreads();
    if (t < 128) {
        uint32_t m = 0;
#pragma unroll 8
        for (int i = 0; i < kActThreads / 16; ++i) m = max(m, sh.colmax[i][t]);
        sh.colscale[t] = static_cast<uint8_t>(act_scale_byte(m));
    }
    __syncthreads();
#pragma unroll
    for (int c = 0; c < 8; ++c) {
        const float sc = act_scale_operand(sh.colscale[8 * sub + c]);
        *reinterpret_cast<uint32_t *>(sh.t + (8 * sub + c) * kTPad + kActRows * g) =
            act_codes4(v[0][c], v[1][c], v[2][c], v[3][c], sc);
    }
    __syncthreads();
#pragma unroll
    for (int i = t; i < 128 * 8; i += kActThreads) {
        const int c = i / 8, p = i % 8;
        if (col0 + c < f.R) {
            const uint32_t *s = reinterpret_cast<const uint32_t *>(sh.t + c * kTPad + 16 * p);
            *reinterpret_cast<uint4 *>(f.codes + static_cast<size_t>(col0 + c) * f.Kp + kb * 128 + 16 * p) =
                uint4{s[0], s[1], s[2], s[3]};
        }
    }
    if (t < 8)
        reinterpret_cast<uint4 *>(f.scales + static_cast<size_t>(kb) * f.Rp + col0)[t] =
            reinterpret_cast<const uint4 *>(sh.colscale)[t];
    __syncthreads();   // the tile's LDS may be written again
}

// One 128 x 128 tile of x [T][C] per workgroup; row.codes or col.codes may be null.
template <class XT>
__global__ __launch_bounds__(kActThreads) void act_quantize(const XT *x, int T, int C, ActForm row, ActForm col) {
    __shared__ __attribute__((aligned(16))) ActTileShared sh;
    const int g = threadIdx.x / 16, sub = threadIdx.x % 16;
    const int cb = blockIdx.x, rb = blockIdx.y;
    float v[kActRows][8];
#pragma unroll
    for (int r = 0; r < kActRows; ++r) {
        const int i = rb * 128 + kActRows * g + r, c = cb * 128 + 8 * sub;
        if (i < T && c < C) load8(x + static_cast<size_t>(i) * C + c, v[r]);   // C is a multiple of 16
        else
#pragma unroll
            for (int q = 0; q < 8; ++q) v[r][q] = 0.0f;
    }
    if (row.codes) tile_rows(v, sh, row, rb * 128, cb, g, sub);
    if (col.codes) tile_cols(v, sh, col, cb * 128, rb, g, sub);
}

// The row form alone: no tile to share, one lane row per (matrix row, block).
template <class XT>
__global__ __launch_bounds__(256) void act_quantize_rows(const XT *x, int T, int C, ActForm f) {
    const int sub = threadIdx.x % 16, kb = blockIdx.y, c = kb * 128 + 8 * sub;
    const long row = static_cast<long>(blockIdx.x) * 16 + threadIdx.x / 16;   // up to f.Rp
    float v[8];
    if (row < T && c < C) load8(x + static_cast<size_t>(row) * C + c, v);
    else
#pragma unroll
        for (int q = 0; q < 8; ++q) v[q] = 0.0f;
    put_row(v, f, row, T, kb, sub);
}

hipError_t launch_act_quantize(const void *x, bool f32, int T, int C, const ActForm &row, const ActForm &col, hipStream_t s) {
    if (!col.codes) {
        const dim3 rows(row.Rp / 16, (C + 127) / 128);
        if (f32) hipLaunchKernelGGL(act_quantize_rows<float>, rows, dim3(256), 0, s, static_cast<const float *>(x), T, C, row);
        else hipLaunchKernelGGL(act_quantize_rows<uint16_t>, rows, dim3(256), 0, s, static_cast<const uint16_t *>(x), T, C, row);
        return hipGetLastError();
    }
    const dim3 grid((C + 127) / 128, (T + 127) / 128);
    if (f32)
        hipLaunchKernelGGL(act_quantize<float>, grid, dim3(kActThreads), 0, s, static_cast<const float *>(x), T, C, row, col);
    else
        hipLaunchKernelGGL(act_quantize<uint16_t>, grid, dim3(kActThreads), 0, s, static_cast<const uint16_t *>(x), T, C,
                           row, col);
    return hipGetLastError();
}

// SwiGLU forward: h = silu(g) u from gu [T][2 I] (gate columns first), h in the row form and, if asked for,
// gu itself.  One lane row per (matrix row, block of 128 channels of h).
template <class XT>
__global__ __launch_bounds__(256) void swiglu_quantize(const XT *gu, int T, int I, ActForm h, ActForm saved) {
    const int sub = threadIdx.x % 16, kb = blockIdx.y, nkb = I / 128;
    const long row = static_cast<long>(blockIdx.x) * 16 + threadIdx.x / 16;   // up to h.Rp
    float g[8], u[8], hv[8];
    if (row < T) {
        const XT *p = gu + static_cast<size_t>(row) * 2 * I + kb * 128 + 8 * sub;
        load8(p, g);
        load8(p + I, u);
    } else {
#pragma unroll
        for (int q = 0; q < 8; ++q) g[q] = u[q] = 0.0f;
    }
#pragma unroll
    for (int q = 0; q < 8; ++q) hv[q] = silu_f32(g[q]) * u[q];
    put_row(hv, h, row, T, kb, sub);
    if (saved.codes) {
        put_row(g, saved, row, T, kb, sub);
        put_row(u, saved, row, T, nkb + kb, sub);
    }
}

hipError_t launch_swiglu_quantize(const void *gu, bool f32, int T, int I, const ActForm &h, const ActForm &saved,
                                  hipStream_t s) {
    const dim3 grid(h.Rp / 16, I / 128);
    if (f32)
        hipLaunchKernelGGL(swiglu_quantize<float>, grid, dim3(256), 0, s, static_cast<const float *>(gu), T, I, h, saved);
    else
        hipLaunchKernelGGL(swiglu_quantize<uint16_t>, grid, dim3(256), 0, s, static_cast<const uint16_t *>(gu), T, I, h,
                           saved);
    return hipGetLastError();
}

// SwiGLU backward.  With s = 1 / (1 + exp(-g)):  h = g s u,  dg = dh u s (1 + g (1 - s)),  du = dh g s.
template <class XT>
__global__ __launch_bounds__(kActThreads) void swiglu_backward(ActForm saved, const XT *dh, int T, int I, ActForm drow,
                                                               ActForm dcol, ActForm hcol) {
    __shared__ __attribute__((aligned(16))) ActTileShared sh;
    const int lr = threadIdx.x / 16, sub = threadIdx.x % 16;
    const int cb = blockIdx.x, rb = blockIdx.y, nkb = I / 128;
    float dg[kActRows][8], du[kActRows][8], h[kActRows][8];
#pragma unroll
    for (int r = 0; r < kActRows; ++r) {
        const int i = rb * 128 + kActRows * lr + r;
        if (i < T) {
            const uint8_t *p = saved.codes + static_cast<size_t>(i) * saved.Kp + cb * 128 + 8 * sub;
            const uint2 cg = *reinterpret_cast<const uint2 *>(p), cu = *reinterpret_cast<const uint2 *>(p + I);
            const float sg = act_scale_operand(saved.scales[static_cast<size_t>(cb) * saved.Rp + i]);
            const float su = act_scale_operand(saved.scales[static_cast<size_t>(nkb + cb) * saved.Rp + i]);
            float g[8], u[8], d[8];
            act_values4(cg.x, sg, g);
            act_values4(cg.y, sg, g + 4);
            act_values4(cu.x, su, u);
            act_values4(cu.y, su, u + 4);
            load8(dh + static_cast<size_t>(i) * I + cb * 128 + 8 * sub, d);
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                const float e = __expf(-g[q]), s = 1.0f / (1.0f + e);
                const float gs = g[q] * s;
                h[r][q] = gs * u[q];
                du[r][q] = d[q] * gs;
                // 1 - s = e s; where e overflows s is 0 and 1 - s is 1
                const float one_s = s > 0.0f ? e * s : 1.0f;
                dg[r][q] = d[q] * u[q] * (s + gs * one_s);
            }
        } else {
#pragma unroll
            for (int q = 0; q < 8; ++q) h[r][q] = du[r][q] = dg[r][q] = 0.0f;
        }
    }
    if (drow.codes) {
        tile_rows(dg, sh, drow, rb * 128, cb, lr, sub);
        __syncthreads();
        tile_rows(du, sh, drow, rb * 128, nkb + cb, lr, sub);
    }
    if (dcol.codes) {
        tile_cols(dg, sh, dcol, cb * 128, rb, lr, sub);
        tile_cols(du, sh, dcol, I + cb * 128, rb, lr, sub);
    }
    if (hcol.codes) tile_cols(h, sh, hcol, cb * 128, rb, lr, sub);
}

hipError_t launch_swiglu_backward(const ActForm &saved, const void *dh, bool f32, int T, int I, const ActForm &drow,
                                  const ActForm &dcol, const ActForm &hcol, hipStream_t s) {
    const dim3 grid(I / 128, (T + 127) / 128);
    if (f32)
        hipLaunchKernelGGL(swiglu_backward<float>, grid, dim3(kActThreads), 0, s, saved, static_cast<const float *>(dh), T, I,
                           drow, dcol, hcol);
    else
        hipLaunchKernelGGL(swiglu_backward<uint16_t>, grid, dim3(kActThreads), 0, s, saved,
                           static_cast<const uint16_t *>(dh), T, I, drow, dcol, hcol);
    return hipGetLastError();
}

}  // namespace ftmoe
