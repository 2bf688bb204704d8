// Norms before and after a block, fused with the block's gates and residual scale (ft_block_norm), and their
// backward pass.  With 1/rms(v) = (mean v^2 + eps)^-1/2, g the gate per channel, h the gate per token:
//
//   u = post b / rms(b)  (or b),   r = x + scale g h u,   n = pre r / rms(r)
//
// Backward, from r, b and the gradients dr, dn of r and n; G = dn pre, sums over the channels of a token:
//   d  = dr + (G - r mean(G r) / rms(r)^2) / rms(r)                   gradient of x
//   S  = sum scale g d post b                                         dh = S / rms(b)
//   db = (scale g h post d - b (h S / C) / rms(b)^2) / rms(b)         (scale g h d without a norm after the block)
//   and over the tokens  A = sum h d b / rms(b),  B = sum dn r / rms(r):
//   d_post = scale g A,  d_gate = scale post A,  d_pre = B
//
// A row lies in the registers of its LANES threads (8 CH channels a thread, LANES x 8 channels a step), so each matrix
// is read once.  Row sums: lanes of a wave, then the waves in order through LDS.  Column sums: a thread's own over its
// rows, where a workgroup has several at once over these, then over the workgroups in order, in float64.
//
// The bound is HBM: forward with a norm on both sides 8192 x 7168 bf16 103 to 112 us, 4.7 to 5.1 TB/s; backward 151 us, 5 of them the
// join, 4.7 TB/s.
#include "act_tile.h"

#include <algorithm>
#include <type_traits>

namespace ftmoe {

// 8 channels of a weight or gate; ones where there is none
__device__ __forceinline__ void channels8(const void *w, bool f32, int c, float *v) {
    if (!w) {
#pragma unroll
        for (int q = 0; q < 8; ++q) v[q] = 1.0f;
    } else if (f32) {
        load8(static_cast<const float *>(w) + c, v);
    } else {
        load8(static_cast<const uint16_t *>(w) + c, v);
    }
}

// Sums of N values over the threads of a row, in every one of them.  `turn` alternates between two buffers: whoever
// writes one again has passed the barrier behind the last reading of it.
template <int LANES, int N>
__device__ __forceinline__ void row_sums(float (&v)[N], float (*buf)[N][16], int &turn) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = wave_sum_f32(v[i]);
    if constexpr (LANES > 64) {
        constexpr int kWaves = LANES / 64;
        if (lane_id() == 0)
#pragma unroll
            for (int i = 0; i < N; ++i) buf[turn][i][threadIdx.x / 64] = v[i];
        __syncthreads();
        // every lane row of 16 adds up the waves' sums for itself
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float p = buf[turn][i][lane_id() % kWaves];
            v[i] = lane_id() % 16 < kWaves ? p : 0.0f;
            v[i] += __uint_as_float(dpp_u32<kDppRowRor1>(__float_as_uint(v[i])));
            v[i] += __uint_as_float(dpp_u32<kDppRowRor2>(__float_as_uint(v[i])));
            v[i] += __uint_as_float(dpp_u32<kDppRowRor4>(__float_as_uint(v[i])));
            v[i] += __uint_as_float(dpp_u32<kDppRowRor8>(__float_as_uint(v[i])));
        }
        turn ^= 1;
    }
}

// 1 / rms.  All channels of a token share its error, so the two roundings of 1 / sqrt(m) are taken back by a Newton step
// whose residual 1 - m y^2 is exact to float32's square.
__device__ __forceinline__ float over_rms(float sum, const NormArgs &a) {
    const float m = sum / a.C + a.eps, y = 1.0f / sqrtf(m), t = m * y;
    const float left = fmaf(-t, y, 1.0f) - fmaf(m, y, -t) * y;
    return isfinite(left) ? fmaf(0.5f * y, left, y) : y;   // rows of zeros without eps, and what is not finite: as it is
}

// 8 channels as they lie in memory, and their values
template <class T>
struct Raw8 {
    uint4 w[sizeof(T) / 2];
};
template <class T>
__device__ __forceinline__ void fetch8(const void *p, size_t at, Raw8<T> &r) {
    const uint4 *q = reinterpret_cast<const uint4 *>(static_cast<const T *>(p) + at);
#pragma unroll
    for (int i = 0; i < static_cast<int>(sizeof(T) / 2); ++i) r.w[i] = q[i];
}
template <class T>
__device__ __forceinline__ void values8(const Raw8<T> &r, float *v) {
    uint32_t w[2 * sizeof(T)];
#pragma unroll
    for (int i = 0; i < static_cast<int>(sizeof(T) / 2); ++i) {
        w[4 * i] = r.w[i].x;
        w[4 * i + 1] = r.w[i].y;
        w[4 * i + 2] = r.w[i].z;
        w[4 * i + 3] = r.w[i].w;
    }
#pragma unroll
    for (int q = 0; q < 8; ++q)
        v[q] = __uint_as_float(sizeof(T) == 4 ? w[q] : q % 2 ? w[q / 2] & 0xFFFF0000u : w[q / 2] << 16);
}

// Threads past a row's end hold its last channels, which may be infinite: both factors are taken away.
__device__ __forceinline__ void add_square(bool in, float v, float &s) {
    const float own = in ? v : 0.0f;
    s = fmaf(own, own, s);
}

template <class XT, class YT, int LANES, int CH>
__global__ __launch_bounds__(LANES < 256 ? 256 : LANES, LANES == 1024 ? 4 : 5) void block_norm(NormArgs a, bool w_f32) {
    constexpr int kRows = LANES < 256 ? 256 / LANES : 1;   // rows of a workgroup at once
    constexpr bool kHold = CH == 1;                        // weights stay in registers
    __shared__ float buf[2][1][16];
    int turn = 0;
    const int lane = threadIdx.x % LANES;
    int c[CH];
    bool in[CH];
#pragma unroll
    for (int i = 0; i < CH; ++i) {
        c[i] = (i * LANES + lane) * 8;
        in[i] = c[i] < a.C;
    }
    float pre[kHold ? CH : 1][8], up[kHold ? CH : 1][8];   // up: scale gate post
    auto weights = [&](int i, float *wp, float *wu) {
        float g[8];
        const int at = min(c[i], a.C - 8);
        channels8(a.pre, w_f32, at, wp);
        channels8(a.post_norm ? a.post : nullptr, w_f32, at, wu);
        channels8(a.gate, w_f32, at, g);
#pragma unroll
        for (int q = 0; q < 8; ++q) wu[q] *= a.scale * g[q];
    };
    if constexpr (kHold)
#pragma unroll
        for (int i = 0; i < CH; ++i) weights(i, pre[i], up[i]);
    const long first = static_cast<long>(blockIdx.x) * kRows + threadIdx.x / LANES, stride = static_cast<long>(gridDim.x) * kRows;
    Raw8<XT> x8[CH];
    Raw8<YT> b8[CH] = {};
    float h8 = 1.0f;
    auto request = [&](long row) {   // of rows past the last one: the last one, unused
        row = min(row, a.T - 1L);
        const size_t at = static_cast<size_t>(row) * a.C;
#pragma unroll
        for (int i = 0; i < CH; ++i) fetch8<XT>(a.x, at + min(c[i], a.C - 8), x8[i]);
        if (a.b)
#pragma unroll
            for (int i = 0; i < CH; ++i) fetch8<YT>(a.b, at + min(c[i], a.C - 8), b8[i]);
        if (a.tgate) h8 = a.tgate[row];
    };
    request(first);
    for (long row = first; row < a.T; row += stride) {
        const size_t at = static_cast<size_t>(row) * a.C;
        float x[CH][8], b[CH][8], h = h8;
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            values8(x8[i], x[i]);
            values8(b8[i], b[i]);
        }
        request(row + stride);
        if (a.b) {
            if (a.post_norm) {
                float s[1] = {0.0f};
#pragma unroll
                for (int i = 0; i < CH; ++i)
#pragma unroll
                    for (int q = 0; q < 8; ++q) add_square(in[i], b[i][q], s[0]);
                row_sums<LANES, 1>(s, buf, turn);
                h *= over_rms(s[0], a);
            }
#pragma unroll
            for (int i = 0; i < CH; ++i) {
                float wp[8], wu[8];
                if constexpr (!kHold) weights(i, wp, wu);
#pragma unroll
                for (int q = 0; q < 8; ++q) x[i][q] = fmaf(kHold ? up[kHold ? i : 0][q] : wu[q], b[i][q] * h, x[i][q]);
                if (in[i] && a.r) store8<true>(static_cast<XT *>(a.r) + at + c[i], x[i]);
            }
        }
        if (!a.nout && !a.row.codes) continue;
        float s[1] = {0.0f};
#pragma unroll
        for (int i = 0; i < CH; ++i)
#pragma unroll
            for (int q = 0; q < 8; ++q) add_square(in[i], x[i][q], s[0]);
        row_sums<LANES, 1>(s, buf, turn);
        const float rr = over_rms(s[0], a);
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            float wp[8], wu[8], n[8];
            if constexpr (!kHold) weights(i, wp, wu);
#pragma unroll
            for (int q = 0; q < 8; ++q) n[q] = in[i] ? x[i][q] * rr * (kHold ? pre[kHold ? i : 0][q] : wp[q]) : 0.0f;
            if (in[i] && a.nout) store8<true>(static_cast<YT *>(a.nout) + at + c[i], n);
            if (a.row.codes && c[i] < a.row.Kp) {   // Kp is a multiple of 128: whole lane rows of 16
                const int byte = act_scale_byte(block_mag16(n));
                const float sc = act_scale_operand(byte);
                *reinterpret_cast<uint2 *>(a.row.codes + static_cast<size_t>(row) * a.row.Kp + c[i]) =
                    uint2{act_codes4(n[0], n[1], n[2], n[3], sc), act_codes4(n[4], n[5], n[6], n[7], sc)};
                if (lane % 16 == 0) a.row.scales[static_cast<size_t>(c[i] / 128) * a.row.Rp + row] = static_cast<uint8_t>(byte);
            }
        }
    }
    // scales of the rows that fill the form up
    if (a.row.codes && blockIdx.x == 0) {
        const int more = a.row.Rp - a.T;
        for (int i = threadIdx.x; i < more * (a.row.Kp / 128); i += blockDim.x)
            a.row.scales[static_cast<size_t>(i / more) * a.row.Rp + a.T + i % more] = 127;
    }
}

// A row's channels of a thread; up to 8192 channels the next row's are requested before the sums of this one are waited for: a
// workgroup of 1024 threads fills a CU, and without its next row on the way nothing is (8192 x 7168: 324 us; 16 channels a
// thread and half the threads spill).  Up to 16384 channels the weights are read again for every row and the column sums
// lie in LDS (3500 x 16384: 517 us with all of it in registers, 388 without the weights, 250 so); beyond, registers spill (1700 x
// 32768: 2479 us, the forward pass 596).
template <class XT, class YT, int LANES, int CH>
__global__ __launch_bounds__(LANES < 256 ? 256 : LANES, LANES == 1024 ? 4 : 3) void block_norm_backward(NormArgs a, bool w_f32) {
    constexpr int kRows = LANES < 256 ? 256 / LANES : 1;
    constexpr bool kHold = CH == 1;    // weights stay in registers, and the next row is on its way
    __shared__ float buf3[2][3][16], buf1[2][1][16];
    int turn3 = 0, turn1 = 0;
    const int lane = threadIdx.x % LANES;
    int c[CH];
    bool in[CH];
#pragma unroll
    for (int i = 0; i < CH; ++i) {
        c[i] = (i * LANES + lane) * 8;
        in[i] = c[i] < a.C;
    }
    float pre[kHold ? CH : 1][8], up[kHold ? CH : 1][8];
    auto weights = [&](int i, float *wp, float *wu) {
        float g[8];
        const int at = min(c[i], a.C - 8);
        channels8(a.pre, w_f32, at, wp);
        channels8(a.post_norm ? a.post : nullptr, w_f32, at, wu);
        channels8(a.gate, w_f32, at, g);
#pragma unroll
        for (int q = 0; q < 8; ++q) wu[q] *= a.scale * g[q];
    };
    if constexpr (kHold)
#pragma unroll
        for (int i = 0; i < CH; ++i) weights(i, pre[i], up[i]);
    // A and B over this workgroup's rows, each channel its thread's own: in registers, or, where those are short, in LDS
    constexpr bool kInLds = CH == 2;
    __shared__ __attribute__((aligned(16))) float column[kInLds ? 2 * LANES * CH * 8 : 4];
    float sa[kInLds ? 1 : CH][8], sb[kInLds ? 1 : CH][8];
    auto columns = [&](int i, int which) { return reinterpret_cast<floatx4_t *>(column + (which * CH + i) * LANES * 8 + lane * 8); };
    if constexpr (kInLds) {
#pragma unroll
        for (int i = 0; i < 2 * CH; ++i) columns(i, 0)[0] = columns(i, 0)[1] = floatx4_t{};
    } else {
#pragma unroll
        for (int i = 0; i < CH; ++i)
#pragma unroll
            for (int q = 0; q < 8; ++q) sa[i][q] = sb[i][q] = 0.0f;
    }
    const long part = static_cast<long>(blockIdx.x) * kRows + threadIdx.x / LANES, stride = static_cast<long>(gridDim.x) * kRows;
    Raw8<XT> r8[CH], d8[CH] = {};
    Raw8<YT> b8[CH] = {}, n8[CH] = {};
    float h8 = 1.0f;
    auto request = [&](long row) {   // of rows past the last one: the last one, unused
        row = min(row, a.T - 1L);
        const size_t at = static_cast<size_t>(row) * a.C;
#pragma unroll
        for (int i = 0; i < CH; ++i) fetch8<XT>(a.x, at + min(c[i], a.C - 8), r8[i]);
        if (a.dn)
#pragma unroll
            for (int i = 0; i < CH; ++i) fetch8<YT>(a.dn, at + min(c[i], a.C - 8), n8[i]);
        if (a.b)
#pragma unroll
            for (int i = 0; i < CH; ++i) fetch8<YT>(a.b, at + min(c[i], a.C - 8), b8[i]);
        if (a.dr)
#pragma unroll
            for (int i = 0; i < CH; ++i) fetch8<XT>(a.dr, at + min(c[i], a.C - 8), d8[i]);
        if (a.tgate) h8 = a.tgate[row];
    };
    if (kHold) request(part);
    for (long row = part; row < a.T; row += stride) {
        if (!kHold) request(row);
        const size_t at = static_cast<size_t>(row) * a.C;
        float r[CH][8], n[CH][8], b[CH][8], d[CH][8], s[3] = {0.0f, 0.0f, 0.0f};
        const float h = h8;
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            values8(r8[i], r[i]);
            values8(n8[i], n[i]);
            values8(b8[i], b[i]);
            values8(d8[i], d[i]);
        }
        if (kHold) request(row + stride);
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            float wp[8], wu[8];
            if constexpr (!kHold) weights(i, wp, wu);
            if (in[i])
#pragma unroll
                for (int q = 0; q < 8; ++q) {
                    s[0] = fmaf(r[i][q], r[i][q], s[0]);
                    s[1] = fmaf(n[i][q] * (kHold ? pre[kHold ? i : 0][q] : wp[q]), r[i][q], s[1]);
                    s[2] = fmaf(b[i][q], b[i][q], s[2]);
                }
        }
        row_sums<LANES, 3>(s, buf3, turn3);
        const float rr = over_rms(s[0], a), rb = a.post_norm ? over_rms(s[2], a) : 1.0f;
        const float mean = s[1] / a.C * rr * rr, hb = h * rb;
        float t[1] = {0.0f};
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            float wp[8], wu[8];
            if constexpr (!kHold) weights(i, wp, wu);
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                const float g = n[i][q] * (kHold ? pre[kHold ? i : 0][q] : wp[q]);
                if (a.dn) d[i][q] = fmaf(rr, fmaf(-mean, r[i][q], g), d[i][q]);
                if constexpr (!kInLds) {
                    sb[i][q] = fmaf(n[i][q], r[i][q] * rr, sb[i][q]);
                    sa[i][q] = fmaf(hb * d[i][q], b[i][q], sa[i][q]);
                }
            }
            if constexpr (kInLds)
#pragma unroll
                for (int v = 0; v < 2; ++v) {
                    floatx4_t ca = columns(i, 0)[v], cb = columns(i, 1)[v];
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        ca[q] = fmaf(hb * d[i][4 * v + q], b[i][4 * v + q], ca[q]);
                        cb[q] = fmaf(n[i][4 * v + q], r[i][4 * v + q] * rr, cb[q]);
                    }
                    columns(i, 0)[v] = ca;
                    columns(i, 1)[v] = cb;
                }
            if (in[i] && a.r) store8<true>(static_cast<XT *>(a.r) + at + c[i], d[i]);
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                d[i][q] *= kHold ? up[kHold ? i : 0][q] : wu[q];   // scale gate post d
                if (in[i]) t[0] = fmaf(d[i][q], b[i][q], t[0]);
            }
        }
        if (!a.b) continue;
        if (a.post_norm || a.d_tgate) row_sums<LANES, 1>(t, buf1, turn1);
        if (a.d_tgate && lane == 0) a.d_tgate[row] = t[0] * rb;
        const float off = a.post_norm ? t[0] / a.C * rb * rb : 0.0f;
        if (!a.nout) continue;
#pragma unroll
        for (int i = 0; i < CH; ++i) {
#pragma unroll
            for (int q = 0; q < 8; ++q) d[i][q] = hb * fmaf(-off, b[i][q], d[i][q]);
            if (in[i]) store8<true>(static_cast<YT *>(a.nout) + at + c[i], d[i]);
        }
    }
    if (!a.parts) return;
    float *mine = a.parts + static_cast<size_t>(blockIdx.x) * 2 * a.C;
    if constexpr (kRows > 1) {   // the rows' waves, in order
        static_assert(CH == 1 && LANES * 16 == 4 * 256);
        __shared__ __attribute__((aligned(16))) float rows[kRows][2][LANES * 8];
        store8(rows[threadIdx.x / LANES][0] + lane * 8, sa[0]);
        store8(rows[threadIdx.x / LANES][1] + lane * 8, sb[0]);
        __syncthreads();
        const int which = threadIdx.x / (2 * LANES), at = 4 * (threadIdx.x % (2 * LANES));
        if (at >= a.C) return;
        floatx4_t sum = *reinterpret_cast<const floatx4_t *>(&rows[0][which][at]);
#pragma unroll
        for (int r = 1; r < kRows; ++r) sum += *reinterpret_cast<const floatx4_t *>(&rows[r][which][at]);
        *reinterpret_cast<floatx4_t *>(mine + which * a.C + at) = sum;
        return;
    }
#pragma unroll
    for (int i = 0; i < CH; ++i)
        if (in[i]) {
            if constexpr (kInLds)
#pragma unroll
                for (int v = 0; v < 2; ++v) {
                    *reinterpret_cast<floatx4_t *>(mine + c[i] + 4 * v) = columns(i, 0)[v];
                    *reinterpret_cast<floatx4_t *>(mine + a.C + c[i] + 4 * v) = columns(i, 1)[v];
                }
            else {
                store8(mine + c[i], sa[i]);
                store8(mine + a.C + c[i], sb[i]);
            }
        }
}

// Column sums of the parts: 64 columns of A or B per workgroup, RUNS runs of parts by 16 threads of 4 columns.  Few columns have few
// workgroups and up to 1024 parts: 64 runs there (27648 x 368, with the waves' sums joined before: 52 -> 37 us; from 2048 columns on 16 are better).
template <int RUNS>
__global__ __launch_bounds__(16 * RUNS) void block_norm_join(NormArgs a, bool w_f32, float *d_pre, float *d_post, float *d_gate) {
    __shared__ double sums[RUNS][64];
    const int run = threadIdx.x / 16, col = blockIdx.x * 64 + 4 * (threadIdx.x % 16);
    const bool second = blockIdx.y == 1;
    double v[4] = {0.0, 0.0, 0.0, 0.0};
    if (col < a.C) {
        const float *p = a.parts + (second ? a.C : 0) + col;
#pragma unroll 8
        for (int i = run; i < a.n_parts; i += RUNS) {
            const float4 f = *reinterpret_cast<const float4 *>(p + static_cast<size_t>(i) * 2 * a.C);
            v[0] += f.x;
            v[1] += f.y;
            v[2] += f.z;
            v[3] += f.w;
        }
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) sums[run][4 * (threadIdx.x % 16) + q] = v[q];
    __syncthreads();
    const int c = blockIdx.x * 64 + threadIdx.x;
    if (threadIdx.x >= 64 || c >= a.C) return;
    double s = 0.0;
#pragma unroll
    for (int i = 0; i < RUNS; ++i) s += sums[i][threadIdx.x];
    if (second) {
        if (d_pre) d_pre[c] = static_cast<float>(s);
        return;
    }
    auto at = [&](const void *w) {
        if (!w) return 1.0f;
        return w_f32 ? static_cast<const float *>(w)[c] : __uint_as_float(static_cast<uint32_t>(static_cast<const uint16_t *>(w)[c]) << 16);
    };
    if (d_post) d_post[c] = static_cast<float>(s * a.scale * at(a.gate));
    if (d_gate) d_gate[c] = static_cast<float>(s * a.scale * at(a.post_norm ? a.post : nullptr));
}

// Threads of a row, and rows of a workgroup, by the channels.
struct NormShape {
    int lanes, rows;
};
static NormShape norm_shape(int C) {
    if (C <= 512) return {64, 4};
    if (C <= 2048) return {256, 1};
    return {C <= 4096 ? 512 : 1024, 1};
}
// Workgroups: as many as run at once, so that each holds its weights for several rows and leaves one part.
static int norm_blocks(int T, int C, bool back) {
    const NormShape n = norm_shape(C);
    return std::min((T + n.rows - 1) / n.rows, (back || n.lanes == 1024 ? 256 : 384) * 1024 / std::max(n.lanes, 256));
}
int norm_parts(int T, int C) { return norm_blocks(T, C, true); }

template <class XT, class YT, bool BACK>
static void norm_go(const NormArgs &a, bool w_f32, hipStream_t s) {
    const dim3 grid(norm_blocks(a.T, a.C, BACK));
    auto go = [&](auto lanes, auto chunks) {
        constexpr int L = decltype(lanes)::value, CH = decltype(chunks)::value;
        if constexpr (BACK) hipLaunchKernelGGL((block_norm_backward<XT, YT, L, CH>), grid, dim3(std::max(L, 256)), 0, s, a, w_f32);
        else hipLaunchKernelGGL((block_norm<XT, YT, L, CH>), grid, dim3(std::max(L, 256)), 0, s, a, w_f32);
    };
    std::integral_constant<int, 64> l64;
    std::integral_constant<int, 256> l256;
    std::integral_constant<int, 512> l512;
    std::integral_constant<int, 1024> l1024;
    std::integral_constant<int, 1> c1;
    std::integral_constant<int, 2> c2;
    std::integral_constant<int, 8> c8;
    if (a.C <= 512) go(l64, c1);
    else if (a.C <= 2048) go(l256, c1);
    else if (a.C <= 4096) go(l512, c1);
    else if (a.C <= 8192) go(l1024, c1);
    else if (a.C <= 16384) go(l1024, c2);
    else go(l1024, c8);
}

template <bool BACK>
static void norm_types(const NormArgs &a, bool x_f32, bool y_f32, bool w_f32, hipStream_t s) {
    if (x_f32) y_f32 ? norm_go<float, float, BACK>(a, w_f32, s) : norm_go<float, uint16_t, BACK>(a, w_f32, s);
    else y_f32 ? norm_go<uint16_t, float, BACK>(a, w_f32, s) : norm_go<uint16_t, uint16_t, BACK>(a, w_f32, s);
}

hipError_t launch_block_norm(const NormArgs &a, bool x_f32, bool y_f32, bool w_f32, hipStream_t s) {
    norm_types<false>(a, x_f32, y_f32, w_f32, s);
    return hipGetLastError();
}

hipError_t launch_block_norm_backward(const NormArgs &a, bool x_f32, bool y_f32, bool w_f32, float *d_pre, float *d_post,
                                      float *d_gate, hipStream_t s) {
    if (a.T > 0) norm_types<true>(a, x_f32, y_f32, w_f32, s);
    const dim3 grid((a.C + 63) / 64, 2);
    if (a.parts && a.C <= 1024) hipLaunchKernelGGL(block_norm_join<64>, grid, dim3(1024), 0, s, a, w_f32, d_pre, d_post, d_gate);
    else if (a.parts) hipLaunchKernelGGL(block_norm_join<16>, grid, dim3(256), 0, s, a, w_f32, d_pre, d_post, d_gate);
    return hipGetLastError();
}

}  // namespace ftmoe
