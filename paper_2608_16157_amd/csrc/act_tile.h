// Writers of 8-bit forms from values in registers: rows by 8 lanes a block, and tiles of 128 x 128 for both forms
// (act.hip, dispatch.hip); internal.
#pragma once

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

// A store of 8 or 16 bytes.  STREAM: of what no kernel reads again soon enough, past the caches, so that it neither
// displaces what is read nor comes back to write it out.
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
template <bool STREAM, class V>
__device__ __forceinline__ void put_words(void *p, V v) {
    if constexpr (STREAM) __builtin_nontemporal_store(v, static_cast<V *>(p));
    else *static_cast<V *>(p) = v;
}

// One block of a row by 8 lanes, 16 values a lane; rows past T (zeros, up to f.Rp) leave only their scale byte.
template <bool STREAM = false>
__device__ __forceinline__ void put_row(const float (&v)[16], const ActForm &f, long row, int T, int kb, int sub) {
    const int byte = act_scale_byte(block_mag8(v));
    const float sc = act_scale_operand(byte);
    if (row < T)
        put_words<STREAM>(f.codes + static_cast<size_t>(row) * f.Kp + kb * 128 + 16 * sub,
                          u32x4_t{act_codes4(v[0], v[1], v[2], v[3], sc), act_codes4(v[4], v[5], v[6], v[7], sc),
                                  act_codes4(v[8], v[9], v[10], v[11], sc), act_codes4(v[12], v[13], v[14], v[15], sc)});
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
// eight values out, rounded to nearest even where they are bf16
template <bool STREAM = false>
__device__ __forceinline__ void store8(uint16_t *p, const float *v) {
    put_words<STREAM>(p, u32x4_t{bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]), bf16_pair(v[6], v[7])});
}
template <bool STREAM = false>
__device__ __forceinline__ void store8(float *p, const float *v) {
    put_words<STREAM>(p, floatx4_t{v[0], v[1], v[2], v[3]});
    put_words<STREAM>(p + 4, floatx4_t{v[4], v[5], v[6], v[7]});
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
// STREAM: the codes' stores do not stay in the caches.
template <int NP, bool STREAM = false>
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
                    put_words<STREAM>(f.codes + static_cast<size_t>(row) * f.Kp + to[n].row_kb * 128 + 8 * sub,
                                      u32x2_t{act_codes4(v[n][r][0], v[n][r][1], v[n][r][2], v[n][r][3], sc),
                                              act_codes4(v[n][r][4], v[n][r][5], v[n][r][6], v[n][r][7], sc)});
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
                put_words<STREAM>(f.codes + static_cast<size_t>(to[n].col_row0 + c) * f.Kp + col_kb * 128 + 16 * p,
                                  u32x4_t{s[0], s[1], s[2], s[3]});
            }
        }
        if (t >= 64 && t < 72)
            reinterpret_cast<uint4 *>(f.scales + static_cast<size_t>(col_kb) * f.Rp + to[n].col_row0)[t - 64] =
                reinterpret_cast<const uint4 *>(sh.colscale[n])[t - 64];
    }
}

// The same of values that are bf16 already, two in a word: w[r] holds the words of row 4 g + r.  Magnitudes are compared in
// pairs, as 16-bit integers, which order as the values do; the conversions take pairs as they lie, and for the column
// form pairs of rows; a lane ends with one row's maximum, whose scale it forms for the others.  Both forms of 78000 x 7168
// out of 8192 rows: 270 vector instructions a wave in place of 531, with which the vector units were busy all of the time: 313 us,
// 266 (0.64 busy; stores to memory bound it now).
typedef uint16_t u16x2_t __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t max_pairs(uint32_t a, uint32_t b) {
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2_t, a), __builtin_bit_cast(u16x2_t, b)));
}
// a magnitude pair without what is not finite
__device__ __forceinline__ uint32_t finite_pair(uint32_t m) {
    return ((m & 0xFFFFu) < 0x7F80u ? m & 0xFFFFu : 0u) | (m >> 16 < 0x7F80u ? m & 0xFFFF0000u : 0u);
}
// codes of the four values of two words.  The conversions write a half word each: `over` is what the first one's other
// half holds until the second, any word that nobody needs (a register less to clear).
__device__ __forceinline__ uint32_t act_codes4_bf16(uint32_t w0, uint32_t w1, float scale, uint32_t over) {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    i16x2_vec_t r = __builtin_bit_cast(i16x2_vec_t, over);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, __builtin_bit_cast(bf16x2, w0), scale, false);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, __builtin_bit_cast(bf16x2, w1), scale, true);
    return __builtin_bit_cast(uint32_t, r);
}
// bits of the largest finite magnitude of 2 N values
template <int N>
__device__ __forceinline__ uint32_t mag_of_pairs(const uint32_t (&w)[N]) {
    uint32_t m = w[0] & 0x7FFF7FFFu;
#pragma unroll
    for (int i = 1; i < N; ++i) m = max_pairs(m, w[i] & 0x7FFF7FFFu);
    m = max(m << 16, m & 0xFFFF0000u);
    if (m >= 0x7F800000u) {
        m = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) m = max_pairs(m, finite_pair(w[i] & 0x7FFF7FFFu));
        m = max(m << 16, m & 0xFFFF0000u);
    }
    return m;
}

struct PairTileShared {
    uint32_t colmax[kActThreads / 16][64];   // two columns a word
    uint8_t t[128 * kTPad];
    uint8_t rowscale[128];
    uint16_t colscale[64];
    float colop[128];
};
// The whole tile is inside the rows.
template <bool STREAM>
__device__ __forceinline__ void put_tile_pairs(const uint32_t (&w)[kActRows][4], PairTileShared &sh, const ActPlane &to, int row0, int col_kb) {
    const int t = threadIdx.x, g = t / 16, sub = t % 16;
    uint32_t mag[kActRows][4], m[kActRows], cm[4], all;
#pragma unroll
    for (int r = 0; r < kActRows; ++r)
#pragma unroll
        for (int i = 0; i < 4; ++i) mag[r][i] = w[r][i] & 0x7FFF7FFFu;
    auto largest = [&] {
#pragma unroll
        for (int i = 0; i < 4; ++i) cm[i] = max_pairs(max_pairs(mag[0][i], mag[1][i]), max_pairs(mag[2][i], mag[3][i]));
        all = max_pairs(max_pairs(cm[0], cm[1]), max_pairs(cm[2], cm[3]));
    };
    largest();
    if (max(all << 16, all & 0xFFFF0000u) >= 0x7F800000u) {
#pragma unroll
        for (int r = 0; r < kActRows; ++r)
#pragma unroll
            for (int i = 0; i < 4; ++i) mag[r][i] = finite_pair(mag[r][i]);
        largest();
    }
    if (to.col.codes) *reinterpret_cast<uint4 *>(&sh.colmax[g][4 * sub]) = uint4{cm[0], cm[1], cm[2], cm[3]};
    if (to.row.codes) {
        const ActForm &f = to.row;
#pragma unroll
        for (int r = 0; r < kActRows; ++r) {
            const uint32_t p = max_pairs(max_pairs(mag[r][0], mag[r][1]), max_pairs(mag[r][2], mag[r][3]));
            m[r] = max(p << 16, p & 0xFFFF0000u);
        }
        // over the lane row: a lane keeps half of its rows for each of the lanes 8 and 4 on, and ends with row sub / 4
        const bool up = sub & 8, odd = sub & 4;
        uint32_t k0 = max(up ? m[2] : m[0], dpp_u32<kDppRowRor8>(up ? m[0] : m[2]));
        uint32_t k1 = max(up ? m[3] : m[1], dpp_u32<kDppRowRor8>(up ? m[1] : m[3]));
        uint32_t k = max(odd ? k1 : k0, dpp_u32<0x1B>(dpp_u32<0x141>(odd ? k0 : k1)));   // lane ^ 4: 7 - (3 - i)
        k = max(k, dpp_u32<0xB1>(k));
        k = max(k, dpp_u32<0x4E>(k));
        const uint32_t byte = act_scale_byte(k);
        if (sub % 4 == 0) sh.rowscale[kActRows * g + sub / 4] = static_cast<uint8_t>(byte);
        const uint32_t scale = byte << 23;
        const float op[kActRows] = {__uint_as_float(dpp_u32<kDppRowCopy0>(scale)), __uint_as_float(dpp_u32<kDppRowCopy0 + 4>(scale)),
                                    __uint_as_float(dpp_u32<kDppRowCopy0 + 8>(scale)), __uint_as_float(dpp_u32<kDppRowCopy0 + 12>(scale))};
        uint8_t *base = f.codes + static_cast<size_t>(row0) * f.Kp + to.row_kb * 128;
#pragma unroll
        for (int r = 0; r < kActRows; ++r)
            put_words<STREAM>(base + (static_cast<uint32_t>(kActRows * g + r) * f.Kp + 8 * sub),
                              u32x2_t{act_codes4_bf16(w[r][0], w[r][1], op[r], mag[r][0]), act_codes4_bf16(w[r][2], w[r][3], op[r], mag[r][2])});
    }
    __syncthreads();
    if (to.row.codes && t >= 64 && t < 72)   // rows past the last one are zeros here: their scale byte is 127
        reinterpret_cast<uint4 *>(to.row.scales + static_cast<size_t>(to.row_kb) * to.row.Rp + row0)[t - 64] =
            reinterpret_cast<const uint4 *>(sh.rowscale)[t - 64];
    if (!to.col.codes) return;
    const ActForm &f = to.col;
    if (t < 64) {
        uint32_t p = sh.colmax[0][t];
#pragma unroll
        for (int q = 1; q < kActThreads / 16; ++q) p = max_pairs(p, sh.colmax[q][t]);
        const int b0 = act_scale_byte(p << 16), b1 = act_scale_byte(p & 0xFFFF0000u);
        sh.colscale[t] = static_cast<uint16_t>(b0 | b1 << 8);
        *reinterpret_cast<float2 *>(&sh.colop[2 * t]) = float2{act_scale_operand(b0), act_scale_operand(b1)};
    }
    __syncthreads();
    float op[8];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const float4 o = *reinterpret_cast<const float4 *>(&sh.colop[8 * sub + 4 * i]);
        op[4 * i] = o.x;
        op[4 * i + 1] = o.y;
        op[4 * i + 2] = o.z;
        op[4 * i + 3] = o.w;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint32_t pick = h ? 0x07060302u : 0x05040100u;
            const uint32_t low = __builtin_amdgcn_perm(w[1][i], w[0][i], pick), high = __builtin_amdgcn_perm(w[3][i], w[2][i], pick);
            *reinterpret_cast<uint32_t *>(sh.t + (8 * sub + 2 * i + h) * kTPad + kActRows * g) = act_codes4_bf16(low, high, op[2 * i + h], low);
        }
    __syncthreads();
    uint8_t *base = f.codes + static_cast<size_t>(to.col_row0) * f.Kp + static_cast<size_t>(col_kb) * 128;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int c = (t + i * kActThreads) / 8, p = t % 8;
        if (to.col_row0 + c < f.R) {
            const uint32_t *s = reinterpret_cast<const uint32_t *>(sh.t + c * kTPad + 16 * p);
            put_words<STREAM>(base + (static_cast<size_t>(c) * f.Kp + 16 * p), u32x4_t{s[0], s[1], s[2], s[3]});
        }
    }
    if (t >= 64 && t < 72)
        reinterpret_cast<uint4 *>(f.scales + static_cast<size_t>(col_kb) * f.Rp + to.col_row0)[t - 64] =
            reinterpret_cast<const uint4 *>(sh.colscale)[t - 64];
}

}  // namespace ftmoe
