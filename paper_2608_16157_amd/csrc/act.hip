// Activations and gradients in 8 bits: the quantiser (row form, column form or both from one read) and the
// SwiGLU activation between two dense products, forward (its output and what the backward pass keeps, both
// in 8 bits) and backward (from what was kept).
//
// All of these move memory once and compute little: the bound is HBM.
//
// The row form alone: 8 lanes per row and block of 128, 16 values a lane, so a block's maximum needs only
// rotations within a lane row and no LDS.  8192 x 7168 bf16: 29.7 us, 5.9 TB/s; float32 51 us,
// 5.8 TB/s.
//
// The column form needs a maximum over 128 rows and the transposed codes: a workgroup owns a tile of
// 128 x 128 elements, each thread a patch of 4 rows x 8 columns, so that the codes of 4 rows of a column
// leave as one word through LDS and both forms store whole 128-byte lines.  Both forms of 8192 x 7168:
// 39 us, 6.0 TB/s (float32 69 us, 5.1 TB/s).  SwiGLU backward, three such planes at 9 bytes a channel: 8192 x 2048 in
// 37 us, 4.1 TB/s; the vector unit works 0.45 of that, and with two tiles a CU (128 registers a thread, 76 KB of LDS a
// tile) its work and the loads overlap only between those two; the columns' scales are read from LDS one by one,
// each behind the write of the last one's codes.  A tile after the other by the same workgroup, the next one's loads on the
// way, spills registers and is slower.
#include "act_tile.h"

namespace ftmoe {

// One 128 x 128 tile of x [T][C] per workgroup; row.codes may be null.
template <class XT>
__global__ __launch_bounds__(kActThreads) void act_quantize(const XT *x, int T, int C, ActForm row, ActForm col) {
    __shared__ __attribute__((aligned(16))) ActTileShared<1> sh;
    const int g = threadIdx.x / 16, sub = threadIdx.x % 16;
    const int cb = blockIdx.x, rb = blockIdx.y, row0 = rb * 128 + kActRows * g, c = cb * 128 + 8 * sub;
    float v[1][kActRows][8];
#pragma unroll
    for (int r = 0; r < kActRows; ++r)
        load8(x + static_cast<size_t>(min(row0 + r, T - 1)) * C + min(c, C - 8), v[0][r]);
#pragma unroll
    for (int r = 0; r < kActRows; ++r) {
        quiet(v[0][r]);
        zero_unless(row0 + r < T && c < C, v[0][r]);   // C is a multiple of 16
    }
    const ActPlane to[1] = {{row, cb, col, cb * 128}};
    put_tile<1>(v, sh, to, rb * 128, rb);
}

// The row form alone: no tile to share, 8 lanes per (matrix row, block), two rows on the way at once.  The blocks
// of a row are consecutive workgroups, so that what runs together reads whole rows.
constexpr int kRowsPerLane = 2, kRowsPerWg = 32 * kRowsPerLane;
template <class XT>
__global__ __launch_bounds__(256) void act_quantize_rows(const XT *x, int T, int C, ActForm f) {
    const int sub = threadIdx.x % 8, kb = blockIdx.x, c = kb * 128 + 16 * sub;
    const long row0 = static_cast<long>(blockIdx.y) * kRowsPerWg + threadIdx.x / 8;   // rows up to f.Rp
    float v[kRowsPerLane][16];
#pragma unroll
    for (int r = 0; r < kRowsPerLane; ++r) {
        const long row = min(row0 + 32 * r, T - 1L);
        load16(x + static_cast<size_t>(row) * C + min(c, C - 16), v[r]);
    }
#pragma unroll
    for (int r = 0; r < kRowsPerLane; ++r) {
        quiet(v[r]);
        zero_unless(row0 + 32 * r < T && c < C, v[r]);   // C is a multiple of 16
        put_row(v[r], f, row0 + 32 * r, T, kb, sub);
    }
}

hipError_t launch_act_quantize(const void *x, bool f32, int T, int C, const ActForm &row, const ActForm &col, hipStream_t s) {
    if (!col.codes) {
        const dim3 rows((C + 127) / 128, row.Rp / kRowsPerWg);
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
// gu itself.  8 lanes per (matrix row, block of 128 channels of h).  Bound: HBM; 8192 x 2048 in 20.3 us, 5.8 TB/s.
template <class XT>
__global__ __launch_bounds__(256) void swiglu_quantize(const XT *gu, int T, int I, ActForm h, ActForm saved) {
    const int sub = threadIdx.x % 8, kb = blockIdx.x, nkb = I / 128;
    const long row = static_cast<long>(blockIdx.y) * 32 + threadIdx.x / 8;   // up to h.Rp
    const XT *p = gu + static_cast<size_t>(min(row, T - 1L)) * 2 * I + kb * 128 + 16 * sub;
    float g[16], u[16], hv[16];
    load16(p, g);
    load16(p + I, u);
    quiet(g);
    quiet(u);
    zero_unless(row < T, g);
    zero_unless(row < T, u);
#pragma unroll
    for (int q = 0; q < 16; ++q) hv[q] = silu_f32(g[q]) * u[q];
    put_row(hv, h, row, T, kb, sub);
    if (saved.codes) {
        put_row(g, saved, row, T, kb, sub);
        put_row(u, saved, row, T, nkb + kb, sub);
    }
}

hipError_t launch_swiglu_quantize(const void *gu, bool f32, int T, int I, const ActForm &h, const ActForm &saved,
                                  hipStream_t s) {
    const dim3 grid(I / 128, h.Rp / 32);
    if (f32)
        hipLaunchKernelGGL(swiglu_quantize<float>, grid, dim3(256), 0, s, static_cast<const float *>(gu), T, I, h, saved);
    else
        hipLaunchKernelGGL(swiglu_quantize<uint16_t>, grid, dim3(256), 0, s, static_cast<const uint16_t *>(gu), T, I, h,
                           saved);
    return hipGetLastError();
}

// SwiGLU backward.  With s = 1 / (1 + exp(-g)):  h = g s u,  dg = dh u s (1 + g (1 - s)),  du = dh g s.  The
// reciprocal is the hardware's, 1 ulp; results have 4 significant bits.
template <class XT>
__global__ __launch_bounds__(kActThreads, 4) void swiglu_backward(ActForm saved, const XT *dh, int T, int I, ActForm drow,
                                                                  ActForm dcol, ActForm hcol) {
    __shared__ __attribute__((aligned(16))) ActTileShared<3> sh;
    const int lr = threadIdx.x / 16, sub = threadIdx.x % 16;
    const int cb = blockIdx.x, rb = blockIdx.y, nkb = I / 128;
    const int row0 = rb * 128 + kActRows * lr;
    uint2 cg[kActRows], cu[kActRows];
    float sg[kActRows], su[kActRows], d[kActRows][8];
#pragma unroll
    for (int r = 0; r < kActRows; ++r) {
        const int i = min(row0 + r, T - 1);
        const uint8_t *p = saved.codes + static_cast<size_t>(i) * saved.Kp + cb * 128 + 8 * sub;
        cg[r] = *reinterpret_cast<const uint2 *>(p);
        cu[r] = *reinterpret_cast<const uint2 *>(p + I);
        sg[r] = act_scale_operand(saved.scales[static_cast<size_t>(cb) * saved.Rp + i]);
        su[r] = act_scale_operand(saved.scales[static_cast<size_t>(nkb + cb) * saved.Rp + i]);
        load8(dh + static_cast<size_t>(i) * I + cb * 128 + 8 * sub, d[r]);
    }
    float v[3][kActRows][8];   // dg, du, h
#pragma unroll
    for (int r = 0; r < kActRows; ++r) {
        float g[8], u[8];
        act_values4(cg[r].x, sg[r], g);
        act_values4(cg[r].y, sg[r], g + 4);
        act_values4(cu[r].x, su[r], u);
        act_values4(cu[r].y, su[r], u + 4);
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            const float s = __builtin_amdgcn_rcpf(1.0f + __expf(-g[q]));   // 0 where exp overflows
            const float gs = g[q] * s;
            v[2][r][q] = gs * u[q];
            v[1][r][q] = d[r][q] * gs;
            v[0][r][q] = d[r][q] * (u[q] * (s + gs * (1.0f - s)));   // dh u alone may overflow
        }
#pragma unroll
        for (int n = 0; n < 3; ++n) zero_unless(row0 + r < T, v[n][r]);
    }
    const ActPlane to[3] = {{drow, cb, dcol, cb * 128}, {drow, nkb + cb, dcol, I + cb * 128}, {ActForm{}, 0, hcol, cb * 128}};
    put_tile<3>(v, sh, to, rb * 128, rb);
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
