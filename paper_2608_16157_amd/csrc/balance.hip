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
// the launches' latency.  Up to 128 experts a token is held by one 16-lane row of a wave, whose reductions need
// no step across rows and serve four tokens at once, above by the whole wave (256 experts in a row take 138
// registers: backward 49.8 us against 48.5 for 65536 tokens).  The next token is requested before the current
// one is worked on: 65536 tokens of 256 experts backward 34.7 us, 4.1 TB/s (a copy of as much 25.5; the vector unit
// works half of the time).  The sums over tokens stay in the lanes' registers.  Every sum runs in a fixed order: the
// results are the same in every run.  Sums over tokens are in float64 and rounded to float32 once for each wave
// and once for each part, so that their error does not grow with the tokens: of equal probabilities, whose roundings
// all point one way, float32 sums were off by 2e-6 for 20011 tokens.
//
// Forward: up to 512 tokens one launch, a workgroup per sequence (48 tokens of 128 experts 4.6 us); above, parts of the
// tokens over up to 256 workgroups and a join (8192 tokens of 256 experts in 9 sequences 13.0 us: two launches,
// each some round trips to memory long).  One long sequence would gain from the second form earlier: 512 tokens of
// 256 experts in one workgroup take 27 us, 2000 of 128 in parts 9.7.
#include "ftmoe_device.h"
#include "ftmoe_internal.h"

#include <type_traits>

namespace ftmoe {

constexpr int kBalThreads = 1024;
constexpr int kBalWaves = kBalThreads / 64;

// Reductions over the LPT lanes of a token, in every lane of it.
template <int LPT>
__device__ __forceinline__ float lanes_max(float v) {
    auto ror = [](float x, auto c) { return __uint_as_float(dpp_u32<decltype(c)::value>(__float_as_uint(x))); };
    v = fmaxf(v, ror(v, std::integral_constant<int, kDppRowRor1>{}));
    v = fmaxf(v, ror(v, std::integral_constant<int, kDppRowRor2>{}));
    v = fmaxf(v, ror(v, std::integral_constant<int, kDppRowRor4>{}));
    v = fmaxf(v, ror(v, std::integral_constant<int, kDppRowRor8>{}));
    if constexpr (LPT == 64) {
        auto at = [&](int l) { return __uint_as_float(readlane_u32(__float_as_uint(v), l)); };
        v = fmaxf(fmaxf(at(0), at(16)), fmaxf(at(32), at(48)));
    }
    return v;
}
template <int LPT>
__device__ __forceinline__ float lanes_sum(float v) {
    if constexpr (LPT == 64) return wave_sum_f32(v);
    auto ror = [](float x, auto c) { return __uint_as_float(dpp_u32<decltype(c)::value>(__float_as_uint(x))); };
    v += ror(v, std::integral_constant<int, kDppRowRor1>{});
    v += ror(v, std::integral_constant<int, kDppRowRor2>{});
    v += ror(v, std::integral_constant<int, kDppRowRor4>{});
    v += ror(v, std::integral_constant<int, kDppRowRor8>{});
    return v;
}

// The same in float64 over the 16 lanes of a row, and over the lanes of the four rows that are one above the other.
__device__ __forceinline__ double row_sum_f64(double v) {
    auto ror = [](double x, auto c) {
        constexpr int C = decltype(c)::value;
        return __hiloint2double(static_cast<int>(dpp_u32<C>(__double2hiint(x))), static_cast<int>(dpp_u32<C>(__double2loint(x))));
    };
    v += ror(v, std::integral_constant<int, kDppRowRor1>{});
    v += ror(v, std::integral_constant<int, kDppRowRor2>{});
    v += ror(v, std::integral_constant<int, kDppRowRor4>{});
    v += ror(v, std::integral_constant<int, kDppRowRor8>{});
    return v;
}
__device__ __forceinline__ double rows_sum_f64(double v) {
    uint32_t lo = __double2loint(v), hi = __double2hiint(v);
    const auto l16 = __builtin_amdgcn_permlane16_swap(lo, lo, false, false), h16 = __builtin_amdgcn_permlane16_swap(hi, hi, false, false);
    v = __hiloint2double(h16[0], l16[0]) + __hiloint2double(h16[1], l16[1]);
    lo = __double2loint(v), hi = __double2hiint(v);
    const auto l32 = __builtin_amdgcn_permlane32_swap(lo, lo, false, false), h32 = __builtin_amdgcn_permlane32_swap(hi, hi, false, false);
    return __hiloint2double(h32[0], l32[0]) + __hiloint2double(h32[1], l32[1]);
}

// How a token's E values lie in its LPT lanes, NE each: four consecutive ones at a time where every row is
// 16-byte aligned (V4), one at a time otherwise.
template <int LPT_, int NE_, bool V4>
struct TokenLayout {
    static constexpr int LPT = LPT_, NE = NE_, kTokens = 64 / LPT;   // tokens of a wave
    static __device__ __forceinline__ int expert(int sub, int i) {
        return V4 ? 4 * (sub + LPT * (i / 4)) + i % 4 : sub + LPT * i;
    }
    static __device__ __forceinline__ void load(const float *row, int E, int sub, float past, float (&v)[NE]) {
        if constexpr (V4) {
#pragma unroll
            for (int i = 0; i < NE; i += 4) {
                const int e = expert(sub, i);
                const float4 q = e < E ? *reinterpret_cast<const float4 *>(row + e) : make_float4(past, past, past, past);
                v[i] = q.x;
                v[i + 1] = q.y;
                v[i + 2] = q.z;
                v[i + 3] = q.w;
            }
        } else {
#pragma unroll
            for (int i = 0; i < NE; ++i) v[i] = expert(sub, i) < E ? row[expert(sub, i)] : past;
        }
    }
    static __device__ __forceinline__ void store(float *row, int E, int sub, const float (&v)[NE]) {
        if constexpr (V4) {
#pragma unroll
            for (int i = 0; i < NE; i += 4)
                if (expert(sub, i) < E)
                    *reinterpret_cast<float4 *>(row + expert(sub, i)) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
        } else {
#pragma unroll
            for (int i = 0; i < NE; ++i)
                if (expert(sub, i) < E) row[expert(sub, i)] = v[i];
        }
    }
};

// sigmoid of x as r or e r with e = exp(-|x|), r = 1 / (1 + e) by the hardware's reciprocal (1 ulp)
__device__ __forceinline__ void sigmoid_parts(float x, float &e, float &r) {
    e = __expf(-fabsf(x));
    r = __builtin_amdgcn_rcpf(1.0f + e);
}

// Router probabilities p of one token from its logits l (experts past E hold -inf), and in the sigmoid
// mode a = 1 - sigmoid(l).  The sigmoids of a token whose logits are all negative are taken relative to exp
// of the largest, exp(l - c) / (1 + exp(l)), so that they do not all vanish in float32.  A token whose
// logits are all -inf has no probabilities: p = 0.
template <class L, bool kA>   // kA: a is asked for (its registers otherwise hold the sums over the tokens)
__device__ __forceinline__ void router_probs(const float (&l)[L::NE], int gating, float (&p)[L::NE], float (&a)[kA ? L::NE : 1]) {
    float m = l[0];
#pragma unroll
    for (int i = 1; i < L::NE; ++i) m = fmaxf(m, l[i]);
    float sum = 0.0f;
    if (gating == FT_GATE_SOFTMAX_TOPK_RENORM) {
        m = lanes_max<L::LPT>(m);
#pragma unroll
        for (int i = 0; i < L::NE; ++i) {
            p[i] = __expf(l[i] - m);
            if constexpr (kA) a[i] = 1.0f;
            sum += p[i];
        }
    } else {
#pragma unroll
        for (int i = 0; i < L::NE; ++i) {
            float e, r;
            sigmoid_parts(l[i], e, r);
            p[i] = l[i] > 0.0f ? r : e * r;
            if constexpr (kA) a[i] = l[i] > 0.0f ? e * r : r;
        }
        // a positive logit anywhere in the wave is the common case; without one the maximum is looked for
        if (L::LPT != 64 || !__any(m > 0.0f)) {
            m = lanes_max<L::LPT>(m);
            if (m < 0.0f)
#pragma unroll
                for (int i = 0; i < L::NE; ++i) {
                    float e, r;
                    if constexpr (kA) r = a[i];
                    else sigmoid_parts(l[i], e, r);
                    p[i] = __expf(l[i] - m) * r;
                }
        } else {
            m = 1.0f;   // not -inf
        }
#pragma unroll
        for (int i = 0; i < L::NE; ++i) sum += p[i];
    }
    const float inv = 1.0f / lanes_sum<L::LPT>(sum);
    const bool none = m == -INFINITY;
#pragma unroll
    for (int i = 0; i < L::NE; ++i) p[i] = none ? 0.0f : p[i] * inv;
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

// The sequences for a whole wave, s and t the same in all lanes: up to 64 of them are read by one load, one
// end per lane, instead of a chain of loads.
struct WaveSeqs {
    const BalanceArgs &b;
    bool held;
    int first, ends;
    __device__ __forceinline__ explicit WaveSeqs(const BalanceArgs &args) : b(args), held(args.seq_off && args.n_seq <= 64), first(0), ends(0) {
        if (held) {
            first = b.seq_off[0];
            ends = b.seq_off[min(lane_id() + 1, b.n_seq)];
        }
    }
    __device__ __forceinline__ int first_after(int t) const {
        return held ? __popcll(__ballot(lane_id() < b.n_seq && ends <= t)) : first_seq(b, t);
    }
    __device__ __forceinline__ void bounds(int s, int &beg, int &end) const {
        if (!held) return seq_bounds(b, s, beg, end);
        beg = min(max(s ? static_cast<int>(readlane_u32(ends, s - 1)) : first, 0), b.T);
        end = min(max(static_cast<int>(readlane_u32(ends, s)), beg), b.T);
    }
};

template <class L>
struct BalanceShared {
    static constexpr int kE = L::LPT * L::NE;   // experts, rounded up
    float prob[kBalWaves][kE];
    int32_t count[kE];
    int32_t tokens;
};

// Sums of the tokens [beg, end) over the workgroup: thread e < E gets its expert's probability sum and
// count, every thread the number of counted tokens.
template <class L>
__device__ __forceinline__ void sum_tokens(const BalanceArgs &b, BalanceShared<L> &sh, int beg, int end, double &prob,
                                           int &count, int &tokens) {
    constexpr int kE = BalanceShared<L>::kE;
    const int t = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(t / 64), lane = lane_id(), sub = lane % L::LPT;
    double acc[L::NE];
#pragma unroll
    for (int i = 0; i < L::NE; ++i) acc[i] = 0.0;
    // the next token's logits and ids are requested before the current one is worked on
    constexpr int kStep = kBalWaves * L::kTokens;
    int n = 0, tok = beg + wave * L::kTokens + lane / L::LPT;
    float next[L::NE];
    int id_next = -1;
    uint8_t live_next = 1;
    auto request = [&](int at) {
        const size_t row = static_cast<size_t>(at);
        L::load(b.logits + row * b.E, b.E, sub, -INFINITY, next);
        id_next = b.topk_ids[row * b.k + min(sub, b.k - 1)];
        live_next = b.mask ? b.mask[at] : 1;
    };
    if (tok < end) request(tok);
    for (int e = t; e < kE; e += kBalThreads) sh.count[e] = 0;
    if (t == 0) sh.tokens = 0;
    __syncthreads();
    for (; tok < end; tok += kStep) {
        float l[L::NE], p[L::NE], a[1];
#pragma unroll
        for (int i = 0; i < L::NE; ++i) l[i] = next[i];
        int id = id_next;
        const bool live = live_next != 0;
        request(min(tok + kStep, end - 1));
        if (!live) continue;
        for (int j = sub; j < b.k; j += L::LPT) {
            if (j != sub) id = b.topk_ids[static_cast<size_t>(tok) * b.k + j];
            if (id >= 0 && id < b.E) atomicAdd(&sh.count[id], 1);
        }
        router_probs<L, false>(l, b.gating, p, a);
#pragma unroll
        for (int i = 0; i < L::NE; ++i) acc[i] += p[i];
        ++n;
    }
    if (sub == 0 && n) atomicAdd(&sh.tokens, n);
#pragma unroll
    for (int i = 0; i < L::NE; ++i) {
        if constexpr (L::LPT == 16) acc[i] = rows_sum_f64(acc[i]);   // the wave's four tokens
        if (lane < L::LPT) sh.prob[wave][L::expert(sub, i)] = static_cast<float>(acc[i]);
    }
    __syncthreads();
    prob = 0.0;
    count = 0;
    tokens = sh.tokens;
    if (t < kE) {
        double part[4] = {};   // four sums at once: their additions wait for one another
#pragma unroll
        for (int w = 0; w < kBalWaves; ++w) part[w % 4] += sh.prob[w][t];
        prob = (part[0] + part[1]) + (part[2] + part[3]);
        count = sh.count[t];
    }
    __syncthreads();
}

// Outputs of sequence s from its sums (thread e holds expert e's).
__device__ __forceinline__ void finish_seq(const BalanceArgs &b, int s, double prob, int count, int tokens, double *red) {
    const int t = threadIdx.x;
    double term = 0.0;
    if (t < b.E) {
        const double inv = 1.0 / max(tokens, 1), P = prob * inv, f = b.frac_scale * count * inv;
        const size_t o = static_cast<size_t>(s) * b.E + t;
        b.counts[o] = count;
        b.prob[o] = static_cast<float>(P);
        b.frac[o] = static_cast<float>(f);
        term = f * P;
    }
    term = rows_sum_f64(row_sum_f64(term));
    if (lane_id() == 0) red[t / 64] = term;
    __syncthreads();
    if (t >= 16) return;
    static_assert(kBalWaves == 16, "a row of lanes");
    const double loss = row_sum_f64(red[t]);
    if (t == 0) {
        b.loss[s] = static_cast<float>(loss);
        b.tokens[s] = tokens;
    }
}

// One workgroup per sequence, one launch.
template <class L>
__global__ __launch_bounds__(kBalThreads) void balance_whole(BalanceArgs b) {
    __shared__ BalanceShared<L> sh;
    __shared__ double red[kBalWaves];
    const int s = blockIdx.x;
    int beg, end, count, tokens;
    double prob;
    seq_bounds(b, s, beg, end);
    sum_tokens<L>(b, sh, beg, end, prob, count, tokens);
    finish_seq(b, s, prob, count, tokens, red);
}

// One workgroup per part of the tokens; what sequence s has in part q goes to workspace row q + s.  (Two
// intersections never share a row: an earlier sequence cannot meet a later part than a later sequence does.)
template <class L>
__global__ __launch_bounds__(kBalThreads) void balance_parts(BalanceArgs b) {
    __shared__ BalanceShared<L> sh;
    const int q = blockIdx.x, p0 = q * b.part_tokens, p1 = min(p0 + b.part_tokens, b.T);
    const WaveSeqs seqs(b);
    for (int s = seqs.first_after(p0); s < b.n_seq; ++s) {
        int beg, end, count, tokens;
        double prob;
        seqs.bounds(s, beg, end);
        if (beg >= p1) break;
        beg = max(beg, p0);
        end = min(end, p1);
        if (beg >= end) continue;
        sum_tokens<L>(b, sh, beg, end, prob, count, tokens);
        const size_t row = static_cast<size_t>(q) + s;
        if (threadIdx.x < b.E) {
            b.ws_sums[row * b.E + threadIdx.x] = float2{static_cast<float>(prob), __int_as_float(count)};
        }
        if (threadIdx.x == 0) b.ws_tokens[row] = tokens;
    }
}

// One workgroup per sequence: sums its workspace rows in order, 1024 / EP of them side by side (EP: E up to a
// power of two, 64 at least).
template <int EP>
__global__ __launch_bounds__(kBalThreads) void balance_join(BalanceArgs b) {
    constexpr int kSide = kBalThreads / EP;
    __shared__ double s_prob[kSide][EP];
    __shared__ int32_t s_count[kSide][EP];
    __shared__ int32_t s_tokens;
    __shared__ double red[kBalWaves];
    const int s = blockIdx.x, t = threadIdx.x, e = t % EP, side = t / EP;
    int beg, end;
    seq_bounds(b, s, beg, end);
    if (t == 0) s_tokens = 0;
    __syncthreads();
    double prob = 0.0;
    int count = 0;
    if (beg < end) {
        const int q0 = beg / b.part_tokens, q1 = (end - 1) / b.part_tokens;
        static_assert(kBalMaxParts <= kBalThreads, "one part a thread");
        const int n = b.ws_tokens[min(q0 + t, q1) + s];
        // eight rows on the way at a time; behind the last one it again, unused
        constexpr int kAhead = 8;
        if (e < b.E)
            for (int q = q0 + side; q <= q1; q += kAhead * kSide) {
                float2 v[kAhead];
                double part[4] = {};
#pragma unroll
                for (int i = 0; i < kAhead; ++i) v[i] = b.ws_sums[(static_cast<size_t>(min(q + i * kSide, q1)) + s) * b.E + e];
#pragma unroll
                for (int i = 0; i < kAhead; ++i)
                    if (q + i * kSide <= q1) {
                        part[i % 4] += v[i].x;
                        count += __float_as_int(v[i].y);
                    }
                prob += (part[0] + part[1]) + (part[2] + part[3]);
            }
        if (q0 + t <= q1 && n) atomicAdd(&s_tokens, n);
    }
    s_prob[side][e] = prob;
    s_count[side][e] = count;
    __syncthreads();
    if (t < EP) {
#pragma unroll
        for (int i = 1; i < kSide; ++i) {
            prob += s_prob[i][t];
            count += s_count[i][t];
        }
    }
    finish_seq(b, s, prob, count, s_tokens, red);
}

// What the backward pass reads of one token: its logits, and its selected experts with gates and their
// gradients, one per lane and LPT of them.
template <class L>
struct GradToken {
    static constexpr int kPerLane = kMaxTopK / L::LPT;
    float l[L::NE], g[kPerLane], dg[kPerLane];
    int id[kPerLane];
    uint8_t counted;

    __device__ __forceinline__ void load(const BalanceArgs &b, int t, int sub) {
        const size_t row = static_cast<size_t>(t);
        L::load(b.logits + row * b.E, b.E, sub, -INFINITY, l);
        if (b.d_topk_w)
#pragma unroll
            for (int q = 0; q < kPerLane; ++q) {
                if (q * L::LPT >= b.k) break;
                const size_t o = row * b.k + min(sub + q * L::LPT, b.k - 1);
                id[q] = b.topk_ids[o];
                g[q] = b.topk_w[o];
                dg[q] = b.d_topk_w[o];
            }
        counted = b.mask ? b.mask[t] : 1;
    }
};

// `run` consecutive tokens per LPT lanes, the next one requested before the current one is worked on.  The
// gates' gradients are brought from the lanes of the selected experts to those of the logits through a row
// of LDS; the factor a is applied behind it, where the logit is at hand.  Rows of tokens outside every
// sequence are not touched.
template <class L>
__global__ __launch_bounds__(256) void router_grad(BalanceArgs b, int run) {
    constexpr int kE = L::LPT * L::NE, kSlots = 4 * L::kTokens;
    using Token = GradToken<L>;
    __shared__ __attribute__((aligned(16))) float s_gate[kSlots][kE];
    const int lane = lane_id(), sub = lane % L::LPT;
    const int slot = L::LPT == 64 ? __builtin_amdgcn_readfirstlane(threadIdx.x / 64) : threadIdx.x / L::LPT;
    const int t0 = (static_cast<int>(blockIdx.x) * kSlots + slot) * run;
    if (t0 >= b.T) return;
    const int t1 = min(t0 + run, b.T);
    Token cur, next;
    next.load(b, t0, sub);
    float *gate = s_gate[slot];
    int s = L::LPT == 64 ? WaveSeqs(b).first_after(t0) : first_seq(b, t0), have = -1, beg = 0, end = 0;
    float f[L::NE], weight = 0.0f;
#pragma unroll
    for (int i = 0; i < L::NE; ++i) f[i] = 0.0f;
    for (int t = t0; t < t1; ++t) {
        cur = next;
        if (run > 1) next.load(b, min(t + 1, t1 - 1), sub);
        while (s < b.n_seq) {
            seq_bounds(b, s, beg, end);
            if (end > t) break;
            ++s;
        }
        if (s >= b.n_seq) return;
        if (t < beg) continue;
        if (b.d_loss && have != s) {
            have = s;
            weight = b.d_loss[s] / static_cast<float>(max(b.tokens[s], 1));
            L::load(b.frac + static_cast<size_t>(s) * b.E, b.E, sub, 0.0f, f);
        }
        float p[L::NE], a[L::NE], d[L::NE];
        router_probs<L, true>(cur.l, b.gating, p, a);
        if (b.d_topk_w) {
            float dot = 0.0f;
#pragma unroll
            for (int q = 0; q < Token::kPerLane; ++q) {
                if (q * L::LPT >= b.k) break;
                if (sub + q * L::LPT >= b.k || cur.id[q] < 0 || cur.id[q] >= b.E) cur.id[q] = -1;
                else dot += cur.g[q] * cur.dg[q];
            }
            dot = lanes_sum<L::LPT>(dot);
#pragma unroll
            for (int i = 0; i < L::NE; ++i) gate[L::expert(sub, i)] = 0.0f;
            // a wave's own LDS operations execute in order
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
            for (int q = 0; q < Token::kPerLane; ++q) {
                if (q * L::LPT >= b.k) break;
                if (cur.id[q] >= 0) atomicAdd(&gate[cur.id[q]], cur.g[q] * (cur.dg[q] - dot));
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
            for (int i = 0; i < L::NE; ++i) {
                const float q = gate[L::expert(sub, i)];
                d[i] = q == 0.0f ? 0.0f : a[i] * q;   // a padding token's logits may be anything
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        } else {
#pragma unroll
            for (int i = 0; i < L::NE; ++i) d[i] = 0.0f;
        }
        if (b.d_loss && cur.counted) {
            float dot = 0.0f;
#pragma unroll
            for (int i = 0; i < L::NE; ++i) dot += f[i] * p[i];
            dot = lanes_sum<L::LPT>(dot);
#pragma unroll
            for (int i = 0; i < L::NE; ++i) d[i] += weight * p[i] * a[i] * (f[i] - dot);
        }
        L::store(b.d_logits + static_cast<size_t>(t) * b.E, b.E, sub, d);
    }
}

template <bool V4, class F>
static void with_layout(int E, F &&f) {
    if (E <= 64) f(TokenLayout<16, 4, V4>{});
    else if (E <= 128) f(TokenLayout<16, 8, V4>{});
    else if (E <= 256) f(TokenLayout<64, 4, V4>{});
    else if (E <= 512) f(TokenLayout<64, 8, V4>{});
    else f(TokenLayout<64, 16, V4>{});
}
template <class F>
static void with_layout(const BalanceArgs &a, F &&f) {
    const uintptr_t p = reinterpret_cast<uintptr_t>(a.logits) | reinterpret_cast<uintptr_t>(a.frac) |
                        reinterpret_cast<uintptr_t>(a.d_logits);
    if (a.E % 4 == 0 && p % 16 == 0) with_layout<true>(a.E, f);
    else with_layout<false>(a.E, f);
}

hipError_t launch_balance(const BalanceArgs &a, hipStream_t s) {
    with_layout(a, [&](auto layout) {
        using L = decltype(layout);
        constexpr int EP = L::LPT * L::NE;
        if (a.parts == 0) {
            hipLaunchKernelGGL(balance_whole<L>, dim3(a.n_seq), dim3(kBalThreads), 0, s, a);
        } else {
            hipLaunchKernelGGL(balance_parts<L>, dim3(a.parts), dim3(kBalThreads), 0, s, a);
            hipLaunchKernelGGL(balance_join<EP>, dim3(a.n_seq), dim3(kBalThreads), 0, s, a);
        }
    });
    return hipGetLastError();
}

hipError_t launch_router_backward(const BalanceArgs &a, hipStream_t s) {
    with_layout(a, [&](auto layout) {
        using L = decltype(layout);
        // with tokens enough for the chip, runs of four share the look-up of their sequence
        const int run = a.T >= 16384 ? 4 : 1, per = 4 * L::kTokens * run;
        hipLaunchKernelGGL(router_grad<L>, dim3((a.T + per - 1) / per), dim3(256), 0, s, a, run);
    });
    return hipGetLastError();
}

}  // namespace ftmoe
