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
#include "act_codes.h"
#include "ftmoe_internal.h"

namespace ftmoe {

constexpr int kActThreads = 512;   // a tile: 32 lane rows of 16 lanes, 4 matrix rows each
constexpr int kActRows = 4;
constexpr int kTPad = 132;         // bytes of a transposed row of the tile in LDS

// LDS of a tile of NP planes (matrices of the same shape that leave together).
template <int NP>
struct ActTileShared {
    uint32_t colmax[NP][kActThreads / 16][64];   // 16 bits a column
    uint8_t t[NP][128 * kTPad];
    uint8_t rowscale[NP][128];
    uint8_t colscale[NP][128];
};

// Where a plane goes: its row form's block, and the first row of its column form; codes null where not at all.
struct ActPlane {
    ActForm row;
    int row_kb;
    ActForm col;
    int col_row0;
};

// One block of a row by 8 lanes, 16 values a lane; rows past T (zeros, up to f.Rp) leave only their scale byte.
__device__ __forceinline__ void put_row(const float (&v)[16], const ActForm &f, long row, int T, int kb, int sub) {
    const int byte = act_scale_byte(block_mag8(v));
    const float sc = act_scale_operand(byte);
    if (row < T)
        *reinterpret_cast<uint4 *>(f.codes + static_cast<size_t>(row) * f.Kp + kb * 128 + 16 * sub) =
            uint4{act_codes4(v[0], v[1], v[2], v[3], sc), act_codes4(v[4], v[5], v[6], v[7], sc),
                  act_codes4(v[8], v[9], v[10], v[11], sc), act_codes4(v[12], v[13], v[14], v[15], sc)};
    if (sub == 0) f.scales[static_cast<size_t>(kb) * f.Rp + row] = static_cast<uint8_t>(byte);
}
// Values outside the matrix are read from inside it (p is clamped by the caller) and dropped here: a load
// behind a branch would be waited for before the next one is sent.
template <int N>
__device__ __forceinline__ void zero_unless(bool in, float (&v)[N]) {
    if (!in)
#pragma unroll
        for (int q = 0; q < N; ++q) v[q] = 0.0f;
}
template <class XT>
__device__ __forceinline__ void load16(const XT *p, float (&v)[16]) {
    load8(p, v);
    load8(p + 8, v + 8);
}

// A tile of 128 x 128 elements: v[n] holds plane n's rows 4 g .. 4 g + 3 (g: the thread's lane row), columns
// 8 sub .. 8 sub + 7 of it.  Matrix rows row0 .., block col_kb of the column forms.
//
// A column's scale depends on its largest magnitude only through the exponent and through whether the mantissa
// is above 1.75: the upper 16 bits, rounded up, decide it exactly, so two columns share a word of LDS.
template <int NP>
__device__ __forceinline__ void put_tile(const float (&v)[NP][kActRows][8], ActTileShared<NP> &sh, const ActPlane (&to)[NP],
                                         int row0, int col_kb) {
    const int t = threadIdx.x, g = t / 16, sub = t % 16;
#pragma unroll
    for (int n = 0; n < NP; ++n) {
        if (to[n].row.codes) {
            const ActForm &f = to[n].row;
#pragma unroll
            for (int r = 0; r < kActRows; ++r) {
                const int byte = act_scale_byte(block_mag16(v[n][r])), row = row0 + kActRows * g + r;
                const float sc = act_scale_operand(byte);
                if (row < f.R)
                    *reinterpret_cast<uint2 *>(f.codes + static_cast<size_t>(row) * f.Kp + to[n].row_kb * 128 + 8 * sub) =
                        uint2{act_codes4(v[n][r][0], v[n][r][1], v[n][r][2], v[n][r][3], sc),
                              act_codes4(v[n][r][4], v[n][r][5], v[n][r][6], v[n][r][7], sc)};
                if (sub == 0) sh.rowscale[n][kActRows * g + r] = static_cast<uint8_t>(byte);
            }
        }
        if (to[n].col.codes) {
            uint32_t m[8];
            float all = 0.0f;
#pragma unroll
            for (int c = 0; c < 8; ++c) {
                const float f = max3_abs(max3_abs(0.0f, v[n][0][c], v[n][1][c]), v[n][2][c], v[n][3][c]);
                all += f;   // not finite if one of them is not
                m[c] = __float_as_uint(f) + 0xFFFFu;
            }
            if (!(all < INFINITY))   // as in mag_of
#pragma unroll
                for (int c = 0; c < 8; ++c)
                    m[c] = max(max(act_mag_bits(v[n][0][c]), act_mag_bits(v[n][1][c])),
                               max(act_mag_bits(v[n][2][c]), act_mag_bits(v[n][3][c]))) + 0xFFFFu;
            *reinterpret_cast<uint4 *>(&sh.colmax[n][g][4 * sub]) =
                uint4{m[0] >> 16 | (m[1] & 0xFFFF0000u), m[2] >> 16 | (m[3] & 0xFFFF0000u),
                      m[4] >> 16 | (m[5] & 0xFFFF0000u), m[6] >> 16 | (m[7] & 0xFFFF0000u)};
        }
    }
    __syncthreads();
    for (int i = t; i < NP * 128; i += kActThreads) {
        const int n = i / 128, c = i % 128;
        uint32_t m = 0;
#pragma unroll 8
        for (int q = 0; q < kActThreads / 16; ++q) m = max(m, (sh.colmax[n][q][c / 2] >> (16 * (c % 2))) & 0xFFFFu);
        sh.colscale[n][c] = static_cast<uint8_t>(act_scale_byte(m << 16));
    }
    __syncthreads();
#pragma unroll
    for (int n = 0; n < NP; ++n)
        if (to[n].col.codes)
#pragma unroll
            for (int c = 0; c < 8; ++c) {
                const float sc = act_scale_operand(sh.colscale[n][8 * sub + c]);
                *reinterpret_cast<uint32_t *>(sh.t[n] + (8 * sub + c) * kTPad + kActRows * g) =
                    act_codes4(v[n][0][c], v[n][1][c], v[n][2][c], v[n][3][c], sc);
            }
    __syncthreads();
#pragma unroll
    for (int n = 0; n < NP; ++n) {
        // rows past the last one are zeros here: their scale byte is 127
        if (to[n].row.codes && t < 8)
            reinterpret_cast<uint4 *>(to[n].row.scales + static_cast<size_t>(to[n].row_kb) * to[n].row.Rp + row0)[t] =
                reinterpret_cast<const uint4 *>(sh.rowscale[n])[t];
        if (!to[n].col.codes) continue;
        const ActForm &f = to[n].col;
#pragma unroll
        for (int i = t; i < 128 * 8; i += kActThreads) {
            const int c = i / 8, p = i % 8;
            if (to[n].col_row0 + c < f.R) {
                const uint32_t *s = reinterpret_cast<const uint32_t *>(sh.t[n] + c * kTPad + 16 * p);
                *reinterpret_cast<uint4 *>(f.codes + static_cast<size_t>(to[n].col_row0 + c) * f.Kp + col_kb * 128 + 16 * p) =
                    uint4{s[0], s[1], s[2], s[3]};
            }
        }
        if (t >= 64 && t < 72)
            reinterpret_cast<uint4 *>(f.scales + static_cast<size_t>(col_kb) * f.Rp + to[n].col_row0)[t - 64] =
                reinterpret_cast<const uint4 *>(sh.colscale[n])[t - 64];
    }
}

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
