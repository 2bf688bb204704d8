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

}  // namespace ftmoe
