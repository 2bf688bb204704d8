// Rows of tokens in the order of the groups (ft_expert_gather), back to their tokens (ft_expert_combine), and the
// gradient of the gates (ft_expert_gate_grad).  row_pair and pair_row come from sort.hip; what lies outside their
// ranges counts as no pair and no row.
//
// All of these move memory and compute little: the bound is HBM, and for the 8-bit forms the vector units, where a value is
// handled in its own register (float32, weights); bf16 rows without weights are handled in pairs.  8192 tokens of 7168 channels, 8
// experts each (62000 to 65536 rows, 78000 to 82000 with padding), replayed over buffers that no cache holds: both forms 270 us, 4.6 TB/s, the row form
// 190, plain rows 285; back to the tokens 202 us, 5.2 TB/s; the gates 190.
#include "act_tile.h"
#include "gemm_tile.h"

#include <algorithm>
#include <type_traits>

namespace ftmoe {

// The token of a row and the factor of its values: (-1, 0) where the row has no pair.
__device__ __forceinline__ int row_token(const RowsArgs &a, long row, float &w) {
    const int p = a.row_pair[row];
    w = 1.0f;
    if (static_cast<uint32_t>(p) >= static_cast<uint32_t>(a.T) * static_cast<uint32_t>(a.k)) return -1;
    if (a.w) w = a.w[p];
    return a.over_k ? __umulhi(p, a.over_k) : p;
}
// The same of four rows in every lane of a lane row: each lane asks for one of them.
__device__ __forceinline__ void row_tokens4(const RowsArgs &a, int row0, int sub, int (&t)[4], float (&w)[4]) {
    float one;
    const uint32_t mine = row_token(a, row0 + sub % 4, one), f = __float_as_uint(one);
    t[0] = dpp_u32<kDppRowCopy0>(mine);
    t[1] = dpp_u32<kDppRowCopy0 + 1>(mine);
    t[2] = dpp_u32<kDppRowCopy0 + 2>(mine);
    t[3] = dpp_u32<kDppRowCopy0 + 3>(mine);
    w[0] = __uint_as_float(dpp_u32<kDppRowCopy0>(f));
    w[1] = __uint_as_float(dpp_u32<kDppRowCopy0 + 1>(f));
    w[2] = __uint_as_float(dpp_u32<kDppRowCopy0 + 2>(f));
    w[3] = __uint_as_float(dpp_u32<kDppRowCopy0 + 3>(f));
}
// one past the last group's rows
__device__ __forceinline__ int rows_end(const RowsArgs &a) { return min(a.off[a.n], a.rows); }

// Block of 128 columns and block of `rows` rows of a workgroup, the columns outermost: what runs together on an XCD then
// reads the same columns, of all tokens (2 MB of 8192 in bf16), and each is read from memory once however many rows want
// it (both forms of 8192 x 7168, 8 experts a token, with the sort, one value a register: 347 us; two, four and eight blocks of columns side by
// side 363, 370, 361; rows outermost 440).  False past the groups' rows.
__device__ __forceinline__ bool gather_place(const RowsArgs &a, int columns, int rows, int &cb, int &rb, int &end) {
    end = rows_end(a);
    const int nkb = (columns + 127) / 128, nrb = (end + rows - 1) / rows;
    if (end <= 0 || static_cast<long>(blockIdx.x) >= static_cast<long>(nkb) * nrb) return false;
    const int L = xcd_remap(blockIdx.x, nkb * nrb);
    cb = L / nrb;
    rb = L - cb * nrb;
    return true;
}

// Plain rows: 16 lanes per (row, block of 128), four rows on the way at once.  Where rows are not whole lines of 128 bytes a
// row's blocks begin as many columns before it as its start lies behind a line's, so that stores are whole lines all the same
// (2000 x 8 of 7376 channels bf16, with the sort: 72 us; blocks from the row's start on, which straddle lines, 128).
template <class OT>
__host__ __device__ constexpr int plain_columns(int C) {
    constexpr int kLine = 128 / sizeof(OT);
    return C % kLine == 0 ? C : C + kLine - 16;   // C is a multiple of 16
}
template <class XT, class OT>
__global__ __launch_bounds__(256) void gather_plain(RowsArgs a, const XT *x, OT *out) {
    int cb, rb, end;
    if (!gather_place(a, plain_columns<OT>(a.C), 64, cb, rb, end)) return;
    const int row0 = rb * 64 + threadIdx.x / 16;
    float v[4][8], w[4];
    int t[4], c[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        c[r] = cb * 128 + 8 * static_cast<int>(threadIdx.x % 16) - static_cast<int>(static_cast<uint32_t>(row0 + 16 * r) * a.C % (128 / sizeof(OT)));
        t[r] = row_token(a, min(row0 + 16 * r, end - 1), w[r]);
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) load8(x + static_cast<size_t>(max(t[r], 0)) * a.C + min(max(c[r], 0), a.C - 8), v[r]);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        if (a.w)
#pragma unroll
            for (int q = 0; q < 8; ++q) v[r][q] *= w[r];
        zero_unless(t[r] >= 0, v[r]);
        if (row0 + 16 * r < end && c[r] >= 0 && c[r] < a.C) store8<true>(out + static_cast<size_t>(row0 + 16 * r) * a.C + c[r], v[r]);
    }
}

// The row form alone: 8 lanes per (row, block of 128), two rows on the way at once.
template <class XT>
__global__ __launch_bounds__(256) void gather_rows(RowsArgs a, const XT *x, ActForm f) {
    int kb, rb, end;
    if (!gather_place(a, a.C, 64, kb, rb, end)) return;
    const int sub = threadIdx.x % 8, c = kb * 128 + 16 * sub;
    const long row0 = rb * 64L + threadIdx.x / 8;
    float v[2][16], w[2];
    int t[2];
#pragma unroll
    for (int r = 0; r < 2; ++r) t[r] = row_token(a, min(row0 + 32 * r, end - 1L), w[r]);
#pragma unroll
    for (int r = 0; r < 2; ++r) load16(x + static_cast<size_t>(max(t[r], 0)) * a.C + min(c, a.C - 16), v[r]);
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        if (a.w)   // products are quiet
#pragma unroll
            for (int q = 0; q < 16; ++q) v[r][q] *= w[r];
        else quiet(v[r]);
        zero_unless(t[r] >= 0 && c < a.C, v[r]);   // C is a multiple of 16
        if (row0 + 32 * r < end) put_row<true>(v[r], f, row0 + 32 * r, end, kb, sub);
    }
}

// The same of bf16 rows without weights.
__global__ __launch_bounds__(256) void gather_rows_pairs(RowsArgs a, const uint16_t *x, ActForm f) {
    int kb, rb, end;
    if (!gather_place(a, a.C, 64, kb, rb, end)) return;
    const int sub = threadIdx.x % 8, c = kb * 128 + 16 * sub, g = threadIdx.x / 8, row0 = rb * 64;
    float none;
    int t[2];
    uint32_t w[2][8];
#pragma unroll
    for (int r = 0; r < 2; ++r) t[r] = row_token(a, min(row0 + g + 32 * r, end - 1), none);
#pragma unroll
    for (int r = 0; r < 2; ++r)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint4 q = *reinterpret_cast<const uint4 *>(x + static_cast<size_t>(max(t[r], 0)) * a.C + min(c, a.C - 16) + 8 * i);
            w[r][4 * i] = q.x;
            w[r][4 * i + 1] = q.y;
            w[r][4 * i + 2] = q.z;
            w[r][4 * i + 3] = q.w;
        }
    uint8_t *codes = f.codes + static_cast<size_t>(row0) * f.Kp + kb * 128, *scales = f.scales + static_cast<size_t>(kb) * f.Rp + row0;
#pragma unroll
    for (int r = 0; r < 2; ++r) {
#pragma unroll
        for (int i = 0; i < 8; ++i) w[r][i] = t[r] >= 0 && c < a.C ? w[r][i] : 0u;
        const int row = g + 32 * r, byte = act_scale_byte(eight_max_u32(mag_of_pairs(w[r])));
        const float sc = act_scale_operand(byte);
        if (row0 + row >= end) continue;
        put_words<true>(codes + (static_cast<uint32_t>(row) * f.Kp + 16 * sub),
                        u32x4_t{act_codes4_bf16(w[r][0], w[r][1], sc, 0), act_codes4_bf16(w[r][2], w[r][3], sc, 0),
                                act_codes4_bf16(w[r][4], w[r][5], sc, 0), act_codes4_bf16(w[r][6], w[r][7], sc, 0)});
        if (sub == 0) scales[row] = static_cast<uint8_t>(byte);
    }
}

// Both forms, or the column form alone: one 128 x 128 tile per workgroup; groups start at multiples of 128.
template <class XT>
__global__ __launch_bounds__(kActThreads) void gather_tiles(RowsArgs a, const XT *x, ActForm row, ActForm col) {
    __shared__ __attribute__((aligned(16))) ActTileShared<1> sh;
    const int g = threadIdx.x / 16, sub = threadIdx.x % 16;
    int cb, rb, end;
    if (!gather_place(a, a.C, 128, cb, rb, end)) return;
    const int row0 = rb * 128 + kActRows * g, c = cb * 128 + 8 * sub;
    float v[1][kActRows][8], w[kActRows];
    int t[kActRows];
    row_tokens4(a, row0, sub, t, w);
#pragma unroll
    for (int r = 0; r < kActRows; ++r) load8(x + static_cast<size_t>(max(t[r], 0)) * a.C + min(c, a.C - 8), v[0][r]);
#pragma unroll
    for (int r = 0; r < kActRows; ++r) {
        if (a.w)   // products are quiet
#pragma unroll
            for (int q = 0; q < 8; ++q) v[0][r][q] *= w[r];
        else quiet(v[0][r]);
        zero_unless(t[r] >= 0 && c < a.C, v[0][r]);   // C is a multiple of 16
    }
    const ActPlane to[1] = {{row, cb, col, cb * 128}};
    put_tile<1, true>(v, sh, to, rb * 128, rb);
}

// The same of bf16 rows without weights.
__global__ __launch_bounds__(kActThreads) void gather_tiles_pairs(RowsArgs a, const uint16_t *x, ActForm row, ActForm col) {
    __shared__ __attribute__((aligned(16))) PairTileShared sh;
    const int g = threadIdx.x / 16, sub = threadIdx.x % 16;
    int cb, rb, end;
    if (!gather_place(a, a.C, 128, cb, rb, end)) return;
    const int c = cb * 128 + 8 * sub;
    int t[kActRows];
    float none[kActRows];
    row_tokens4(a, rb * 128 + kActRows * g, sub, t, none);
    uint32_t w[kActRows][4];
#pragma unroll
    for (int r = 0; r < kActRows; ++r) {
        const uint4 q = *reinterpret_cast<const uint4 *>(x + static_cast<size_t>(max(t[r], 0)) * a.C + min(c, a.C - 8));
        w[r][0] = q.x;
        w[r][1] = q.y;
        w[r][2] = q.z;
        w[r][3] = q.w;
    }
    if (__ballot((t[0] | t[1] | t[2] | t[3]) >= 0 && c < a.C) != ~0ull)   // C is a multiple of 16
#pragma unroll
        for (int r = 0; r < kActRows; ++r)
#pragma unroll
            for (int i = 0; i < 4; ++i) w[r][i] = t[r] >= 0 && c < a.C ? w[r][i] : 0u;
    put_tile_pairs<true>(w, sh, ActPlane{row, cb, col, cb * 128}, rb * 128, rb);
}

template <class XT>
static void gather(const RowsArgs &a, const XT *x, void *plain, bool plain_f32, const ActForm &row, const ActForm &col,
                   hipStream_t s) {
    if (plain) {
        auto grid = [&](int columns) { return dim3((columns + 127) / 128 * ((a.rows + 63) / 64)); };
        if (plain_f32)
            hipLaunchKernelGGL((gather_plain<XT, float>), grid(plain_columns<float>(a.C)), dim3(256), 0, s, a, x, static_cast<float *>(plain));
        else
            hipLaunchKernelGGL((gather_plain<XT, uint16_t>), grid(plain_columns<uint16_t>(a.C)), dim3(256), 0, s, a, x, static_cast<uint16_t *>(plain));
    }
    const unsigned nkb = (a.C + 127) / 128;
    if constexpr (std::is_same_v<XT, uint16_t>)
        if (!a.w) {
            if (col.codes)
                hipLaunchKernelGGL(gather_tiles_pairs, dim3(nkb * (a.rows / 128)), dim3(kActThreads), 0, s, a, x, row, col);
            else if (row.codes)
                hipLaunchKernelGGL(gather_rows_pairs, dim3(nkb * ((a.rows + 63) / 64)), dim3(256), 0, s, a, x, row);
            return;
        }
    if (col.codes)
        hipLaunchKernelGGL(gather_tiles<XT>, dim3(nkb * (a.rows / 128)), dim3(kActThreads), 0, s, a, x, row, col);
    else if (row.codes)
        hipLaunchKernelGGL(gather_rows<XT>, dim3(nkb * ((a.rows + 63) / 64)), dim3(256), 0, s, a, x, row);
}

hipError_t launch_gather(const RowsArgs &a, const void *x, bool x_f32, void *plain, bool plain_f32, const ActForm &row,
                         const ActForm &col, hipStream_t s) {
    if (x_f32) gather(a, static_cast<const float *>(x), plain, plain_f32, row, col, s);
    else gather(a, static_cast<const uint16_t *>(x), plain, plain_f32, row, col, s);
    return hipGetLastError();
}

// y[t] = base[t] + sum_j w_tj rows[row of (t, j)], ascending j, in float32.  A wave takes 512 channels of a token; the
// rows of 8 pairs are on the way at once.  2048 channels a workgroup in place of a wave's: 17144 x 1 of 2512 channels 56 us against 41,
// 38454 x 2 of 432 26 against 18, 8192 x 8 of 7168, one in eight here, 58 against 53, all here 205 against 202.
constexpr int kPairsOnWay = 8;

template <class RT, class YT>
__global__ __launch_bounds__(256) void combine_rows(RowsArgs a, const RT *rows, const YT *base, YT *y, int cblocks) {
    const int block = (blockIdx.y * gridDim.x + blockIdx.x) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int t = block / cblocks, c = (block - t * cblocks) * 512 + 8 * lane_id();
    if (t >= a.T) return;
    if (c >= a.C) return;
    float sum[8];
    if (base) load8(base + static_cast<size_t>(t) * a.C + c, sum);
    else
#pragma unroll
        for (int q = 0; q < 8; ++q) sum[q] = 0.0f;
    const int32_t *at = a.pair_row + static_cast<size_t>(t) * a.k;
    const float *w = a.w ? a.w + static_cast<size_t>(t) * a.k : nullptr;
    for (int j0 = 0; j0 < a.k; j0 += kPairsOnWay) {
        float v[kPairsOnWay][8];
        bool in[kPairsOnWay];
#pragma unroll
        for (int j = 0; j < kPairsOnWay; ++j) {
            const int row = at[min(j0 + j, a.k - 1)];
            in[j] = j0 + j < a.k && static_cast<uint32_t>(row) < static_cast<uint32_t>(a.rows);
            load8(rows + static_cast<size_t>(in[j] ? row : 0) * a.C + c, v[j]);
        }
#pragma unroll
        for (int j = 0; j < kPairsOnWay; ++j) {
            if (!in[j]) continue;
            const float f = w ? w[j0 + j] : 1.0f;
#pragma unroll
            for (int q = 0; q < 8; ++q) sum[q] = fmaf(f, v[j][q], sum[q]);
        }
    }
    store8<true>(y + static_cast<size_t>(t) * a.C + c, sum);
}

hipError_t launch_combine(const RowsArgs &a, const void *rows, bool rows_f32, const void *base, void *y, bool y_f32, hipStream_t s) {
    // a token's blocks follow each other (all tokens' first blocks first: 216 us in place of 205 for 8192 x 7168); past
    // 2^23 of them into the second dimension, which holds a launch's threads below 2^32
    const int cblocks = (a.C + 511) / 512, blocks = (a.T * cblocks + 3) / 4;   // at most 2^25
    constexpr int kMost = 1 << 23;
    const dim3 grid(std::min(blocks, kMost), (blocks + kMost - 1) / kMost);
    auto go = [&](auto *r, auto *o) {
        using RT = std::remove_pointer_t<decltype(r)>;
        using YT = std::remove_pointer_t<decltype(o)>;
        hipLaunchKernelGGL((combine_rows<RT, YT>), grid, dim3(256), 0, s, a, static_cast<const RT *>(rows),
                           static_cast<const YT *>(base), static_cast<YT *>(y), cblocks);
    };
    float *f = nullptr;
    uint16_t *h = nullptr;
    if (rows_f32) y_f32 ? go(f, f) : go(f, h);
    else y_f32 ? go(h, f) : go(h, h);
    return hipGetLastError();
}

// d_w[t][j] = <dy[t], rows[row of (t, j)]>, 0 without a row.  WAVES waves per token, each every WAVES-th run of 512
// channels; sums of a lane, of a wave and of the waves in a fixed order.  A lane looks one pair up, and only pairs with a row are
// read, in lots of 8, 4, 2 and 1 (a lot past the last one reads it again: 6 of 8, 3 of 4).
//
// One wave a token where tokens are many and small: 30000 x 2 of 512 channels 18.9 us, four waves 41.8; 41261 x 1 of 3968, one in eight
// here, 26.9 and 37.3; 8192 x 8 of 512, 15.5 and 18.9; of 1024 alike.  Four where not: 300 x 4 of 4096, 7.7 and 5.9; 4096 x 8 of
// 4096, 67 and 63.  Eight loads for every eight pairs, with a row or without: 30000 x 2 82 us, 41261 x 1 228, 1500 x 8 of 2048 15.0
// in place of 12.7.
template <class RT, class YT, int WAVES>
__global__ __launch_bounds__(256) void gate_grad(RowsArgs a, const RT *rows, const YT *dy, float *d_w) {
    __shared__ float part[WAVES][kMaxTopK];
    const int all = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), wave = all % WAVES, lane = lane_id();
    const int t = blockIdx.x * (4 / WAVES) + all / WAVES;
    if (t >= a.T) return;   // waves that meet no barrier
    const YT *d = dy + static_cast<size_t>(t) * a.C;
    const int row = lane < a.k ? a.pair_row[static_cast<size_t>(t) * a.k + lane] : -1;
    uint64_t left = __ballot(static_cast<uint32_t>(row) < static_cast<uint32_t>(a.rows));
    float mine = 0.0f;   // of pair `lane`, over this wave's channels
    auto lot = [&](auto n) {
        constexpr int P = decltype(n)::value;
        const RT *from[P];
        int pair[P];
        float sum[P];
#pragma unroll
        for (int j = 0; j < P; ++j) {
            pair[j] = left ? __builtin_ctzll(left) : pair[max(j - 1, 0)];
            left &= left - 1;
            from[j] = rows + static_cast<size_t>(readlane_u32(row, pair[j])) * a.C;
            sum[j] = 0.0f;
        }
        for (int c = 512 * wave + 8 * lane; c < a.C; c += 512 * WAVES) {
            float g[8], v[P][8];
            load8(d + c, g);
#pragma unroll
            for (int j = 0; j < P; ++j) load8(from[j] + c, v[j]);
#pragma unroll
            for (int j = 0; j < P; ++j)
#pragma unroll
                for (int q = 0; q < 8; ++q) sum[j] = fmaf(g[q], v[j][q], sum[j]);
        }
#pragma unroll
        for (int j = 0; j < P; ++j) {
            const float whole = wave_sum_f32(sum[j]);
            mine = lane == pair[j] ? whole : mine;
        }
    };
    while (left) {
        const int n = __popcll(left);
        if (n >= 6) lot(std::integral_constant<int, 8>{});
        else if (n >= 3) lot(std::integral_constant<int, 4>{});
        else if (n == 2) lot(std::integral_constant<int, 2>{});
        else lot(std::integral_constant<int, 1>{});
    }
    if constexpr (WAVES > 1) {
        part[wave][lane] = mine;
        __syncthreads();
        if (wave > 0) return;
        mine = (part[0][lane] + part[1][lane]) + (part[2][lane] + part[3][lane]);
    }
    if (lane < a.k) d_w[static_cast<size_t>(t) * a.k + lane] = mine;
}

hipError_t launch_gate_grad(const RowsArgs &a, const void *rows, bool rows_f32, const void *dy, bool dy_f32, float *d_w, hipStream_t s) {
    auto go = [&](auto *r, auto *o) {
        using RT = std::remove_pointer_t<decltype(r)>;
        using YT = std::remove_pointer_t<decltype(o)>;
        if (a.T >= 2048 && a.C * a.k <= 8192)
            hipLaunchKernelGGL((gate_grad<RT, YT, 1>), dim3((a.T + 3) / 4), dim3(256), 0, s, a, static_cast<const RT *>(rows),
                               static_cast<const YT *>(dy), d_w);
        else
            hipLaunchKernelGGL((gate_grad<RT, YT, 4>), dim3(a.T), dim3(256), 0, s, a, static_cast<const RT *>(rows),
                               static_cast<const YT *>(dy), d_w);
    };
    float *f = nullptr;
    uint16_t *h = nullptr;
    if (rows_f32) dy_f32 ? go(f, f) : go(f, h);
    else dy_f32 ? go(h, f) : go(h, h);
    return hipGetLastError();
}

}  // namespace ftmoe
