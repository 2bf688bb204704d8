// Balance loss of the router, its per-expert counts, and the gradient of the router logits.
//
// For a sequence s of n counted tokens, c_e of whose routed pairs go to expert e, with p_t the router
// probabilities of token t over all E experts (softmax of the logits, or their sigmoids normalised):
//
//   P_e = (1/n) sum_t p_te,   f_e = coef E c_e / (k n),   L_s = sum_e f_e P_e
//
//   dL_s / dl_te = (1/n) p_te a_te (f_e - sum_i f_i p_ti),   a = 1 (softmax) or 1 - sigmoid(l_te)
//
// and, for the renormalised gates g_j of the selected experts, dl_tej += g_j a_tej (dg_j - sum_i g_i dg_i).
//
// Bound: one read of the logits (forward) or a read and a write (backward); below some thousand tokens
// the launches' latency.  A wave holds a token's E logits, lane l the experts l, l + 64, ..., so the row's
// maximum and sums are wave reductions and the sums over tokens stay in the lanes' registers.  Every sum is
// in float32 in a fixed order: the results are the same in every run.
#include "ftmoe_device.h"
#include "ftmoe_internal.h"

#include <type_traits>

namespace ftmoe {

constexpr int kBalThreads = 1024;
constexpr int kBalWaves = kBalThreads / 64;

__device__ __forceinline__ float wave_max_f32(float v) {
    auto ror = [](float x, auto c) {
        return __uint_as_float(dpp_u32<decltype(c)::value>(__float_as_uint(x)));
    };
    v = fmaxf(v, ror(v, std::integral_constant<int, kDppRowRor1>{}));
    v = fmaxf(v, ror(v, std::integral_constant<int, kDppRowRor2>{}));
    v = fmaxf(v, ror(v, std::integral_constant<int, kDppRowRor4>{}));
    v = fmaxf(v, ror(v, std::integral_constant<int, kDppRowRor8>{}));
    auto at = [&](int l) { return __uint_as_float(readlane_u32(__float_as_uint(v), l)); };
    return fmaxf(fmaxf(at(0), at(16)), fmaxf(at(32), at(48)));
}

// Router probabilities p of one token from its logits l (lanes' experts past E hold -inf), and a = 1 -
// sigmoid(l) in the sigmoid mode.  The sigmoids of a token whose logits are all negative are taken relative
// to exp of the largest, exp(l - c) / (1 + exp(l)), so that they do not all vanish in float32.  A token
// whose logits are all -inf has no probabilities: p = 0.
template <int NE>
__device__ __forceinline__ void router_probs(const float (&l)[NE], int gating, float (&p)[NE], float (&a)[NE]) {
    float m = l[0];
#pragma unroll
    for (int i = 1; i < NE; ++i) m = fmaxf(m, l[i]);
    m = wave_max_f32(m);
    float sum = 0.0f;
    if (gating == FT_GATE_SOFTMAX_TOPK_RENORM) {
#pragma unroll
        for (int i = 0; i < NE; ++i) {
            p[i] = __expf(l[i] - m);
            a[i] = 1.0f;
            sum += p[i];
        }
    } else {
        const float c = fminf(m, 0.0f);
#pragma unroll
        for (int i = 0; i < NE; ++i) {
            const float e = __expf(-fabsf(l[i])), r = 1.0f / (1.0f + e);
            const float neg = c < 0.0f ? __expf(l[i] - c) : e;
            p[i] = l[i] > 0.0f ? r : neg * r;
            a[i] = l[i] > 0.0f ? e * r : r;
            sum += p[i];
        }
    }
    const float inv = 1.0f / wave_sum_f32(sum);
    const bool none = m == -INFINITY;
#pragma unroll
    for (int i = 0; i < NE; ++i) p[i] = none ? 0.0f : p[i] * inv;
}

template <int NE>
__device__ __forceinline__ void load_logits(const float *row, int E, int lane, float (&l)[NE]) {
#pragma unroll
    for (int i = 0; i < NE; ++i) l[i] = lane + 64 * i < E ? row[lane + 64 * i] : -INFINITY;
}

// bounds of sequence s, whatever the offsets hold
__device__ __forceinline__ void seq_bounds(const BalanceArgs &b, int s, int &beg, int &end) {
    beg = b.seq_off ? min(max(b.seq_off[s], 0), b.T) : 0;
    end = b.seq_off ? min(max(b.seq_off[s + 1], beg), b.T) : b.T;
}

// first sequence that ends behind token t (n_seq if none does)
__device__ __forceinline__ int first_seq(const BalanceArgs &b, int t) {
    if (!b.seq_off) return 0;
    int lo = 0, hi = b.n_seq;
    while (lo < hi) {
        const int mid = (lo + hi) / 2;
        if (b.seq_off[mid + 1] > t) hi = mid;
        else lo = mid + 1;
    }
    return lo;
}

template <int NE>
struct BalanceShared {
    float prob[kBalWaves][64 * NE];
    int32_t count[64 * NE];
    int32_t tokens;
};

// Sums of the tokens [beg, end) over the workgroup: thread e < E gets its expert's probability sum and
// count, every thread the number of counted tokens.
template <int NE>
__device__ __forceinline__ void sum_tokens(const BalanceArgs &b, BalanceShared<NE> &sh, int beg, int end, float &prob,
                                           int &count, int &tokens) {
    const int t = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(t / 64), lane = lane_id();
    for (int e = t; e < 64 * NE; e += kBalThreads) sh.count[e] = 0;
    if (t == 0) sh.tokens = 0;
    __syncthreads();
    float acc[NE];
#pragma unroll
    for (int i = 0; i < NE; ++i) acc[i] = 0.0f;
    int n = 0;
    for (int tok = beg + wave; tok < end; tok += kBalWaves) {
        if (b.mask && !b.mask[tok]) continue;
        float l[NE], p[NE], a[NE];
        load_logits<NE>(b.logits + static_cast<size_t>(tok) * b.E, b.E, lane, l);
        if (lane < b.k) {
            const int id = b.topk_ids[static_cast<size_t>(tok) * b.k + lane];
            if (id >= 0 && id < b.E) atomicAdd(&sh.count[id], 1);
        }
        router_probs<NE>(l, b.gating, p, a);
#pragma unroll
        for (int i = 0; i < NE; ++i) acc[i] += p[i];
        ++n;
    }
#pragma unroll
    for (int i = 0; i < NE; ++i) sh.prob[wave][lane + 64 * i] = acc[i];
    if (lane == 0 && n) atomicAdd(&sh.tokens, n);
    __syncthreads();
    prob = 0.0f;
    count = 0;
    tokens = sh.tokens;
    if (t < 64 * NE) {
#pragma unroll
        for (int w = 0; w < kBalWaves; ++w) prob += sh.prob[w][t];
        count = sh.count[t];
    }
    __syncthreads();
}

// Outputs of sequence s from its sums (thread e holds expert e's).
__device__ __forceinline__ void finish_seq(const BalanceArgs &b, int s, float prob, int count, int tokens, float *red) {
    const int t = threadIdx.x;
    float term = 0.0f;
    if (t < b.E) {
        const float n = static_cast<float>(max(tokens, 1));
        const float P = prob / n, f = b.coef * static_cast<float>(b.E) * static_cast<float>(count) / (static_cast<float>(b.k) * n);
        const size_t o = static_cast<size_t>(s) * b.E + t;
        b.counts[o] = count;
        b.prob[o] = P;
        b.frac[o] = f;
        term = f * P;
    }
    const float ws = wave_sum_f32(term);
    if (lane_id() == 0) red[t / 64] = ws;
    __syncthreads();
    if (t == 0) {
        float L = 0.0f;
        for (int w = 0; w < kBalWaves; ++w) L += red[w];
        b.loss[s] = L;
        b.tokens[s] = tokens;
    }
}

// One workgroup per sequence, one launch.
template <int NE>
__global__ __launch_bounds__(kBalThreads) void balance_whole(BalanceArgs b) {
    __shared__ BalanceShared<NE> sh;
    __shared__ float red[kBalWaves];
    const int s = blockIdx.x;
    int beg, end, count, tokens;
    float prob;
    seq_bounds(b, s, beg, end);
    sum_tokens<NE>(b, sh, beg, end, prob, count, tokens);
    finish_seq(b, s, prob, count, tokens, red);
}

// One workgroup per part of the tokens; what sequence s has in part q goes to workspace row q + s.  (Two
// intersections never share a row: an earlier sequence cannot meet a later part than a later sequence does.)
template <int NE>
__global__ __launch_bounds__(kBalThreads) void balance_parts(BalanceArgs b) {
    __shared__ BalanceShared<NE> sh;
    const int q = blockIdx.x, p0 = q * b.part_tokens, p1 = min(p0 + b.part_tokens, b.T);
    for (int s = first_seq(b, p0); s < b.n_seq; ++s) {
        int beg, end, count, tokens;
        float prob;
        seq_bounds(b, s, beg, end);
        if (beg >= p1) break;
        beg = max(beg, p0);
        end = min(end, p1);
        if (beg >= end) continue;
        sum_tokens<NE>(b, sh, beg, end, prob, count, tokens);
        const size_t row = static_cast<size_t>(q) + s;
        if (threadIdx.x < b.E) {
            b.ws_prob[row * b.E + threadIdx.x] = prob;
            b.ws_count[row * b.E + threadIdx.x] = count;
        }
        if (threadIdx.x == 0) b.ws_tokens[row] = tokens;
    }
}

// One workgroup per sequence: sums its workspace rows in order, 1024 / (64 NE) of them side by side.
template <int NE>
__global__ __launch_bounds__(kBalThreads) void balance_join(BalanceArgs b) {
    constexpr int kSide = kBalThreads / (64 * NE);
    __shared__ float s_prob[kSide][64 * NE];
    __shared__ int32_t s_count[kSide][64 * NE];
    __shared__ int32_t s_tokens;
    __shared__ float red[kBalWaves];
    const int s = blockIdx.x, t = threadIdx.x, e = t % (64 * NE), side = t / (64 * NE);
    int beg, end;
    seq_bounds(b, s, beg, end);
    if (t == 0) s_tokens = 0;
    __syncthreads();
    float prob = 0.0f;
    int count = 0;
    if (beg < end) {
        const int q0 = beg / b.part_tokens, q1 = (end - 1) / b.part_tokens;
        if (e < b.E) {
#pragma unroll 8
            for (int q = q0 + side; q <= q1; q += kSide) {
                const size_t o = (static_cast<size_t>(q) + s) * b.E + e;
                prob += b.ws_prob[o];
                count += b.ws_count[o];
            }
        }
        int n = 0;
        for (int q = q0 + t; q <= q1; q += kBalThreads) n += b.ws_tokens[q + s];
        if (n) atomicAdd(&s_tokens, n);
    }
    s_prob[side][e] = prob;
    s_count[side][e] = count;
    __syncthreads();
    if (t < 64 * NE) {
#pragma unroll
        for (int i = 1; i < kSide; ++i) {
            prob += s_prob[i][t];
            count += s_count[i][t];
        }
    }
    finish_seq(b, s, prob, count, s_tokens, red);
}

constexpr int kGradTokens = 4;   // consecutive tokens per wave

// One wave per kGradTokens consecutive tokens.  Rows of tokens outside every sequence are not touched.
template <int NE>
__global__ __launch_bounds__(256) void router_grad(BalanceArgs b) {
    __shared__ float s_gate[4][64 * NE];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = lane_id();
    const int t0 = (static_cast<int>(blockIdx.x) * 4 + wave) * kGradTokens;
    if (t0 >= b.T) return;
    float *gate = s_gate[wave];
    int s = first_seq(b, t0), have = -1, beg = 0, end = 0;
    float f[NE], weight = 0.0f;
    for (int t = t0; t < min(t0 + kGradTokens, b.T); ++t) {
        while (s < b.n_seq) {
            seq_bounds(b, s, beg, end);
            if (end > t) break;
            ++s;
        }
        if (s >= b.n_seq) return;
        if (t < beg) continue;
        const size_t row = static_cast<size_t>(t);
        float l[NE], p[NE], a[NE], d[NE];
        load_logits<NE>(b.logits + row * b.E, b.E, lane, l);
        if (b.d_loss && have != s) {
            have = s;
            weight = b.d_loss[s] / static_cast<float>(max(b.tokens[s], 1));
#pragma unroll
            for (int i = 0; i < NE; ++i) f[i] = lane + 64 * i < b.E ? b.frac[static_cast<size_t>(s) * b.E + lane + 64 * i] : 0.0f;
        }
        if (b.d_topk_w) {
            float g = 0.0f, dg = 0.0f, ag = 1.0f;
            int id = -1;
            if (lane < b.k) {
                const size_t o = row * b.k + lane;
                id = b.topk_ids[o];
                if (id >= 0 && id < b.E) {
                    g = b.topk_w[o];
                    dg = b.d_topk_w[o];
                    if (b.gating != FT_GATE_SOFTMAX_TOPK_RENORM) {
                        const float x = b.logits[row * b.E + id], e = __expf(-fabsf(x)), r = 1.0f / (1.0f + e);
                        ag = x > 0.0f ? e * r : r;
                    }
                } else {
                    id = -1;
                }
            }
            const float dot = wave_sum_f32(g * dg);
#pragma unroll
            for (int i = 0; i < NE; ++i) gate[lane + 64 * i] = 0.0f;
            // the wave's own LDS operations execute in order
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            if (id >= 0) atomicAdd(&gate[id], g * ag * (dg - dot));
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
            for (int i = 0; i < NE; ++i) d[i] = gate[lane + 64 * i];
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        } else {
#pragma unroll
            for (int i = 0; i < NE; ++i) d[i] = 0.0f;
        }
        if (b.d_loss && (!b.mask || b.mask[t])) {
            router_probs<NE>(l, b.gating, p, a);
            float dot = 0.0f;
#pragma unroll
            for (int i = 0; i < NE; ++i) dot += f[i] * p[i];
            dot = wave_sum_f32(dot);
#pragma unroll
            for (int i = 0; i < NE; ++i) d[i] += weight * p[i] * a[i] * (f[i] - dot);
        }
#pragma unroll
        for (int i = 0; i < NE; ++i)
            if (lane + 64 * i < b.E) b.d_logits[row * b.E + lane + 64 * i] = d[i];
    }
}

template <class F>
static void with_ne(int E, F &&f) {
    if (E <= 64) f(std::integral_constant<int, 1>{});
    else if (E <= 128) f(std::integral_constant<int, 2>{});
    else if (E <= 256) f(std::integral_constant<int, 4>{});
    else if (E <= 512) f(std::integral_constant<int, 8>{});
    else f(std::integral_constant<int, 16>{});
}

hipError_t launch_balance(const BalanceArgs &a, hipStream_t s) {
    with_ne(a.E, [&](auto ne) {
        constexpr int NE = decltype(ne)::value;
        if (a.parts == 0) {
            hipLaunchKernelGGL(balance_whole<NE>, dim3(a.n_seq), dim3(kBalThreads), 0, s, a);
        } else {
            hipLaunchKernelGGL(balance_parts<NE>, dim3(a.parts), dim3(kBalThreads), 0, s, a);
            hipLaunchKernelGGL(balance_join<NE>, dim3(a.n_seq), dim3(kBalThreads), 0, s, a);
        }
    });
    return hipGetLastError();
}

hipError_t launch_router_backward(const BalanceArgs &a, hipStream_t s) {
    with_ne(a.E, [&](auto ne) {
        constexpr int NE = decltype(ne)::value;
        const int per = 4 * kGradTokens;
        hipLaunchKernelGGL(router_grad<NE>, dim3((a.T + per - 1) / per), dim3(256), 0, s, a);
    });
    return hipGetLastError();
}

}  // namespace ftmoe
