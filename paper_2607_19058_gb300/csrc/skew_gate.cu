// Routing of tokens to experts and its gradient (skew_gate_* in include/skewadam.h).
//
// Forward, bound by instructions (the logits are read once): a thread to a token for many tokens of few experts
// (k_gate_thread), else a warp to a token, N consecutive logits a lane (k_gate_wide), with
// route_token for what that does not settle. Experts are chosen by the logits themselves, or by fp32
// scores plus biases, never by quicker ones; the lowest index first among equals.
// One GB300, 65536 tokens, whole calls: 8 of 256 experts in 4 of 8 groups, sigmoid scores and a bias, 58 us (674 instructions a
// token and warp; 98 us with fp32 scores throughout and the k largest one after another); 8 of 512 by sigmoid scores and a bias 68; 2 of 128 28;
// 6 of 64 23; 2 of 8 8. What is issued once for a token, and not for an expert, is most of it.
//
// Backward: as many lanes as top_k, rounded up to a power of two, own a token, one chosen expert each. Only the
// softmax that is not renormalised has a gradient elsewhere, and reads whole rows. 65536 tokens of 128 experts, whole calls: 2 chosen 13 us
// (the kernel 11: 33.5 MB of zeros, each sector written by two stores of half of it, and 131072 values over them; laid out
// in shared memory first 12.4), the plain softmax 21.
#include "skew_ops.h"

#include <cfloat>
#include <cmath>

namespace skew {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kMaxExperts = 512, kMaxK = 32, kMaxGroups = 32;
// A thread routes a token of up to kThreadExperts experts, where the tokens give the SMs enough threads: kThreadTokens to an
// expert (thread and warp to a token, us: 2 of 8 experts 4096 tokens 6.3 5.7, 8192 6.4 7.7, 65536 7.7 29; 6 of 64
// 16384 15 12, 32768 18 19, 65536 22 33; 11 of 56 16384 17 13, 65536 30 38).
constexpr int kThreadExperts = 64;
constexpr int64_t kThreadTokens = 600;

struct GateArgs {
    const void *x;
    const float *bias;
    int32_t *chosen;
    float *weights;
    int32_t *counts;
    uint32_t *ws;  // [0, E): tokens of each expert so far, [E]: CTAs done; zero between calls
    int64_t ld, tokens;
    int32_t E, k, groups, top_groups, group_top, group_size, sigmoid, renorm, vec;
    int32_t warp_floats;  // shared memory of a warp (k_gate_thread)
    int32_t per, lane_n;  // lanes to a group, experts to a lane (k_gate_wide)
    float scale;
};

// Larger keys for larger values; -0 is +0. 0 is left for what may not be chosen.
__device__ __forceinline__ uint32_t order_key(float x) {
    const uint32_t b = __float_as_uint(x + 0.f);
    return b ^ (uint32_t(int32_t(b) >> 31) | 0x80000000u);
}

__device__ __forceinline__ float key_value(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k); }

__device__ __forceinline__ bool choosable(float x) { return x > -INFINITY; }  // not -Inf, not NaN

__device__ __forceinline__ float sigmoid(float x) { return 1.f / (1.f + expf(-x)); }

// A chosen score over the chosen ones' sum, at most 1 (0 where that is 0): the scale comes after it, as the scale over a sum of tiny
// scores may leave fp32. Most lanes have no score, and a numerator of 0 takes the division's long way (us for 65536 tokens, 2 of 128
// experts and 8 of 256 in 4 of 8 groups: 30.7 and 61.3 without the 1, 28.5 and 58.3 with it).
__device__ __forceinline__ float share_of(float s, float sum) {
    const float share = (s == 0.f ? 1.f : s) / sum;
    return s == 0.f && sum == sum ? 0.f : share;
}

__device__ __forceinline__ uint32_t lanes_max(uint32_t v) { return __reduce_max_sync(kFullMask, v); }

__device__ __forceinline__ float lanes_max(float v) {
#pragma unroll
    for (int d = 16; d; d >>= 1) v = fmaxf(v, __shfl_xor_sync(kFullMask, v, d));
    return v;
}

__device__ __forceinline__ float lanes_sum(float v) {
#pragma unroll
    for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(kFullMask, v, d);
    return v;
}

// The two largest of (a1 >= a2) and (b1 >= b2).
__device__ __forceinline__ void merge_two(float &a1, float &a2, float b1, float b2) {
    a2 = fmaxf(fminf(a1, b1), fmaxf(a2, b2));
    a1 = fmaxf(a1, b1);
}

// A lane's N logits from `e0` on; what lies past E as -Inf.
template <bool F32, int N>
__device__ __forceinline__ void load_logits(const GateArgs &A, int64_t t, int e0, float (&x)[N]) {
    if (A.vec && e0 < A.E) {
        const char *p = elem_ptr<F32>(A.x, t * A.ld + e0);
        if constexpr (F32) {
#pragma unroll
            for (int q = 0; q < N / 4; ++q) {
                const uint4 u = ld_stream(p + 16 * q);
                x[4 * q] = __uint_as_float(u.x), x[4 * q + 1] = __uint_as_float(u.y);
                x[4 * q + 2] = __uint_as_float(u.z), x[4 * q + 3] = __uint_as_float(u.w);
            }
        } else if constexpr (N == 4) {
            const uint2 u = *reinterpret_cast<const uint2 *>(p);
            x[0] = bf16_low(u.x), x[1] = bf16_high(u.x), x[2] = bf16_low(u.y), x[3] = bf16_high(u.y);
        } else {
#pragma unroll
            for (int q = 0; q < N / 8; ++q) {
                const uint4 u = ld_stream(p + 16 * q);
                const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
                for (int i = 0; i < 4; ++i) x[8 * q + 2 * i] = bf16_low(w[i]), x[8 * q + 2 * i + 1] = bf16_high(w[i]);
            }
        }
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j) x[j] = e0 + j < A.E ? load1<F32>(A.x, t * A.ld + e0 + j) : -INFINITY;
    }
}

// Routes a token by a warp, whatever it and the config hold. row: kMaxExperts floats of the warp's own.
template <bool F32, int N>
__device__ __forceinline__ void route_token(const GateArgs &A, int64_t t, int32_t *hist, float *row) {
    const int lane = threadIdx.x & 31, e0 = lane * N;
    const bool shows = A.bias || (A.groups > 1 && A.group_top == 2);
    float x[N];
    load_logits<F32, N>(A, t, e0, x);
    bool is_nan = false;
#pragma unroll
    for (int j = 0; j < N; ++j) is_nan |= x[j] != x[j];
    const bool nan = __any_sync(kFullMask, is_nan);

    // what experts are chosen by: the logits (they order as the scores do), or the scores plus the bias
    float shown[N], row_max = 0.f, row_sum = 0.f;
    uint32_t key[N];
    if (!A.sigmoid && (shows || !A.renorm)) {
        float m = -INFINITY;
#pragma unroll
        for (int j = 0; j < N; ++j) m = fmaxf(m, x[j]);
        row_max = lanes_max(m);
        if (row_max == -INFINITY) row_max = 0.f;
        float s = 0.f;
#pragma unroll
        for (int j = 0; j < N; ++j) {
            shown[j] = expf(x[j] - row_max);  // without a bias the row's sum changes no order
            s += shown[j];
        }
        row_sum = lanes_sum(s);
        if (A.bias)
#pragma unroll
            for (int j = 0; j < N; ++j) shown[j] = shown[j] / row_sum + (e0 + j < A.E ? A.bias[e0 + j] : 0.f);
    } else if (shows) {
#pragma unroll
        for (int j = 0; j < N; ++j) shown[j] = sigmoid(x[j]) + (A.bias && e0 + j < A.E ? A.bias[e0 + j] : 0.f);
    }
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const float c = A.bias ? shown[j] : x[j];
        key[j] = choosable(c) && choosable(x[j]) ? order_key(c) : 0u;
    }

    if (A.groups > 1) {  // `share` lanes to a group
        const int share = 32 >> (32 - __clz(A.groups - 1)), group = lane / share;
#pragma unroll
        for (int j = 0; j < N; ++j) row[e0 + j] = !key[j] ? -INFINITY : A.group_top == 2 ? shown[j] : key_value(key[j]);
        __syncwarp();
        float a1 = -INFINITY, a2 = -INFINITY;
        if (group < A.groups)
            for (int i = lane % share; i < A.group_size; i += share) merge_two(a1, a2, row[group * A.group_size + i], -INFINITY);
        for (int d = 1; d < share; d <<= 1) {
            const float b1 = __shfl_xor_sync(kFullMask, a1, d), b2 = __shfl_xor_sync(kFullMask, a2, d);
            merge_two(a1, a2, b1, b2);
        }
        __syncwarp();
        uint32_t gkey = choosable(a1) && lane % share == 0 ? order_key(A.group_top == 2 && choosable(a2) ? a1 + a2 : a1) : 0u, taken = 0;
        for (int g = 0; g < A.top_groups; ++g) {
            const uint32_t best = lanes_max(gkey);
            const int win = __ffs(__ballot_sync(kFullMask, gkey == best)) - 1;
            if (best) taken |= 1u << (win / share);
            if (lane == win) gkey = 0;
        }
#pragma unroll
        for (int j = 0; j < N; ++j)
            if (e0 + j >= A.E || !(taken >> ((e0 + j) / A.group_size) & 1)) key[j] = 0;
    }

    // the k largest, one after another
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < N; ++j) m = max(m, key[j]);
    int32_t mine = -1;
    for (int i = 0; i < A.k; ++i) {
        const uint32_t best = lanes_max(m);
        const int win = __ffs(__ballot_sync(kFullMask, m == best)) - 1;
        int at = 0;
#pragma unroll
        for (int j = N - 1; j >= 0; --j)
            if (key[j] == best) at = j;
        const int e = __shfl_sync(kFullMask, e0 + at, win);
        if (lane == win) {
            m = 0;
#pragma unroll
            for (int j = 0; j < N; ++j) {
                if (j == at) key[j] = 0;
                m = max(m, key[j]);
            }
        }
        if (best && i == lane) mine = e;
    }

    // weights of the chosen
    const float xc = mine >= 0 ? load1<F32>(A.x, t * A.ld + mine) : -INFINITY;
    float s = 0.f;
    if (A.sigmoid) {
        s = sigmoid(xc);
    } else {
        const float top = A.renorm ? lanes_max(xc) : row_max;  // renormalised: the softmax of the chosen
        if (mine >= 0) s = A.renorm ? expf(xc - top) : expf(xc - top) / row_sum;
    }
    if (A.renorm) s = share_of(s, lanes_sum(s));
    if (lane < A.k) {
        A.chosen[t * A.k + lane] = mine;
        A.weights[t * A.k + lane] = nan ? NAN : s * A.scale;
        if (A.counts && mine >= 0) atomicAdd(hist + mine, 1);
    }
}

// Adds the CTA's counts to those of all CTAs; the last one hands them out and leaves zeros.
__device__ __forceinline__ void put_counts(const GateArgs &A, const int32_t *hist) {
    if (!A.counts) return;
    __syncthreads();
    if (gridDim.x == 1) {
        for (int e = threadIdx.x; e < A.E; e += blockDim.x) A.counts[e] = hist[e];
        return;
    }
    for (int e = threadIdx.x; e < A.E; e += blockDim.x)
        if (hist[e]) atomicAdd(A.ws + e, (uint32_t)hist[e]);
    __shared__ bool last;
    __threadfence();
    __syncthreads();
    if (threadIdx.x == 0) last = atomicInc(A.ws + A.E, gridDim.x - 1) == gridDim.x - 1;  // back at 0
    __syncthreads();
    if (!last) return;
    __threadfence();
    for (int e = threadIdx.x; e < A.E; e += blockDim.x) A.counts[e] = (int32_t)atomicExch(A.ws + e, 0u);
}

// A warp to a token, by route_token alone.
template <bool F32, int N>
__global__ void __launch_bounds__(kThreads, 3) k_gate(const __grid_constant__ GateArgs A) {
    __shared__ float rows[kWarps][N * 32];
    __shared__ int32_t hist[kMaxExperts];
    for (int e = threadIdx.x; e < A.E; e += kThreads) hist[e] = 0;
    __syncthreads();
    for (int64_t t = int64_t(blockIdx.x) * kWarps + (threadIdx.x >> 5); t < A.tokens; t += int64_t(gridDim.x) * kWarps)
        route_token<F32, N>(A, t, hist, rows[threadIdx.x >> 5]);
    put_counts(A, hist);
}

// A thread to a token, for up to kThreadExperts experts: its logits in shared memory, its KM best experts in registers, sorted
// by insertion; a warp's results go out in one piece.
template <bool F32, int KM>
__global__ void __launch_bounds__(64) k_gate_thread(const __grid_constant__ GateArgs A) {
    extern __shared__ float dyn[];
    __shared__ int32_t hist[kThreadExperts];
    __shared__ float biases[kThreadExperts];
    const int lane = threadIdx.x & 31, warps = blockDim.x >> 5, E = A.E, pitch = E | 1;
    const bool shows = A.bias || (A.groups > 1 && A.group_top == 2), grouped = A.groups > 1;
    for (int e = threadIdx.x; e < E; e += blockDim.x) {
        hist[e] = 0;
        biases[e] = A.bias ? A.bias[e] : 0.f;
    }
    __syncthreads();
    float *rows = dyn + (threadIdx.x >> 5) * A.warp_floats;
    // a thread's logits, its scores plus biases (where experts or groups go by them), its groups' scores
    float *x = rows + lane * pitch, *shown = x + 32 * pitch, *scores = rows + (shows ? 64 : 32) * pitch + lane * (A.groups | 1);
    const float *choices = A.bias ? shown : x, *by = shows ? shown : x;
    for (int64_t w = int64_t(blockIdx.x) * warps + (threadIdx.x >> 5); w * 32 < A.tokens; w += int64_t(gridDim.x) * warps) {
        const int64_t t0 = w * 32;
        const int n = int(A.tokens - t0 < 32 ? A.tokens - t0 : 32);
        for (int r0 = 0; r0 < n; r0 += 8) {  // a row to the lanes
            float a[8], b[8];
#pragma unroll
            for (int r = 0; r < 8; ++r) {
                const int64_t at = (t0 + (r0 + r < n ? r0 + r : n - 1)) * A.ld;
                a[r] = load1<F32>(A.x, at + (lane < E ? lane : 0));
                b[r] = E > 32 ? load1<F32>(A.x, at + (lane + 32 < E ? lane + 32 : 0)) : 0.f;
            }
#pragma unroll
            for (int r = 0; r < 8; ++r) {
                if (lane < E) rows[(r0 + r) * pitch + lane] = a[r];
                if (lane + 32 < E) rows[(r0 + r) * pitch + lane + 32] = b[r];
            }
            if (shows && A.sigmoid) {
                float *at = rows + (32 + r0) * pitch + lane;
#pragma unroll
                for (int r = 0; r < 8; ++r)
                    if (lane < E) at[r * pitch] = sigmoid(a[r]) + biases[lane];
                if (E > 32)
#pragma unroll
                    for (int r = 0; r < 8; ++r)
                        if (lane + 32 < E) at[r * pitch + 32] = sigmoid(b[r]) + biases[lane + 32];
            }
        }
        __syncwarp();
        float row_max = 0.f, row_sum = 0.f;
        if (!A.sigmoid && (shows || !A.renorm)) {
            float m = -INFINITY;
#pragma unroll 4
            for (int e = 0; e < E; ++e) m = fmaxf(m, x[e]);
            row_max = m == -INFINITY ? 0.f : m;
#pragma unroll 4
            for (int e = 0; e < E; ++e) {
                const float s = expf(x[e] - row_max);
                if (shows) shown[e] = s;
                row_sum += s;
            }
            if (A.bias)
#pragma unroll 4
                for (int e = 0; e < E; ++e) shown[e] = shown[e] / row_sum + biases[e];
        }
        uint32_t taken = 1;
        if (grouped) {
            for (int g = 0, e = 0; g < A.groups; ++g) {
                float a1 = -INFINITY, a2 = -INFINITY;
#pragma unroll 4
                for (int i = 0; i < A.group_size; ++i, ++e) {
                    const float s = by[e];
                    merge_two(a1, a2, choosable(s) && choosable(x[e]) ? s : -INFINITY, -INFINITY);
                }
                scores[g] = choosable(a1) ? fmaxf(A.group_top == 2 && choosable(a2) ? a1 + a2 : a1, -FLT_MAX) : -INFINITY;
            }
            taken = 0;
            for (int g = 0; g < A.groups; ++g) {
                const float mine = scores[g];
                int rank = 0;
                for (int o = 0; o < A.groups; ++o) rank += scores[o] > mine || (scores[o] == mine && o < g);
                if (choosable(mine) && rank < A.top_groups) taken |= 1u << g;
            }
        }
        float best[KM];
        int32_t which[KM];
#pragma unroll
        for (int j = 0; j < KM; ++j) best[j] = -INFINITY, which[j] = -1;
        bool nan = false;
        for (int g = 0, e = 0; g < A.groups; ++g) {
            const bool in = taken >> g & 1;
#pragma unroll 4
            for (int i = 0; i < A.group_size; ++i, ++e) {
                const float v = x[e];
                float c = choices[e];
                nan |= v != v;
                if (!in || !(c > best[KM - 1]) || !choosable(v)) continue;  // (a NaN neither)
                int32_t ce = e;
                bool below = false;  // from the first that is smaller on, each moves one down
#pragma unroll
                for (int j = 0; j < KM; ++j) {
                    below = below || c > best[j];
                    const float tc = best[j];
                    const int32_t te = which[j];
                    best[j] = below ? c : tc;
                    which[j] = below ? ce : te;
                    c = below ? tc : c;
                    ce = below ? te : ce;
                }
            }
        }
        // weights of the chosen
        float s[KM], top = row_max, sum = 0.f;
#pragma unroll
        for (int j = 0; j < KM; ++j) {
            if (j >= A.k) which[j] = -1;
            s[j] = which[j] >= 0 ? x[which[j]] : -INFINITY;
        }
        if (!A.sigmoid && A.renorm) {  // the softmax of the chosen
            top = -INFINITY;
#pragma unroll
            for (int j = 0; j < KM; ++j) top = fmaxf(top, s[j]);
        }
#pragma unroll
        for (int j = 0; j < KM; ++j) {
            s[j] = A.sigmoid ? sigmoid(s[j]) : which[j] < 0 ? 0.f : A.renorm ? expf(s[j] - top) : expf(s[j] - top) / row_sum;
            sum += s[j];
        }
        if (A.renorm)
#pragma unroll
            for (int j = 0; j < KM; ++j) s[j] = share_of(s[j], sum);
        if (A.counts && lane < n)
#pragma unroll
            for (int j = 0; j < KM; ++j)
                if (which[j] >= 0) atomicAdd(hist + which[j], 1);
        __syncwarp();
#pragma unroll
        for (int j = 0; j < KM; ++j)
            if (j < A.k) rows[lane * A.k + j] = __int_as_float(which[j]);
        __syncwarp();
        for (int i = lane; i < n * A.k; i += 32) A.chosen[t0 * A.k + i] = __float_as_int(rows[i]);
        __syncwarp();
#pragma unroll
        for (int j = 0; j < KM; ++j)
            if (j < A.k) rows[lane * A.k + j] = nan ? NAN : s[j] * A.scale;
        __syncwarp();
        for (int i = lane; i < n * A.k; i += 32) A.weights[t0 * A.k + i] = rows[i];
        __syncwarp();
    }
    put_counts(A, hist);
}

// Within 2^-21 of expf for x <= 0, and of sigmoid: quick scores, which settle all but near ties.
__device__ __forceinline__ float exp2_approx(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float quick_exp(float x) { return exp2_approx(x * 1.4426950408889634f); }
__device__ __forceinline__ float quick_sigmoid(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(1.f + exp2_approx(x * -1.4426950408889634f)));
    return y;
}

// An expert that may be among the top_k.
struct alignas(16) Cand {
    float c;
    int32_t e;
    float x, bias;
};

template <bool F32, int N>
__device__ __noinline__ void route_hard_token(const GateArgs &A, int64_t t, int32_t *hist, float *row) {
    route_token<F32, N>(A, t, hist, row);
}

// A warp to a token. A group has `per` lanes, a power of two, and a lane lane_n consecutive experts of it (fewer at the group's
// end). Near ties aside, quick scores settle which groups are taken, and which experts may be among the top_k: at
// least k values are no less than the k-th of the lanes' two largest each, and few more; a lane to one of those, with its fp32
// score, ranks it among the others. A token that this does not settle (near ties, a logit that is not finite, over 32
// such experts) takes route_token.
// N = 16 spills up to 192 bytes (softmax scores of bf16 logits) at the 128 registers that two CTAs an SM leave.
// SCORE: kLogits (experts and groups by the logits alone), kSigmoid, kSoftmax (both: quick scores are needed).
enum { kLogits, kSigmoid, kSoftmax };
template <bool F32, int N, int SCORE>
__global__ void __launch_bounds__(kThreads, N == 16 ? 2 : 3) k_gate_wide(const __grid_constant__ GateArgs A) {
    __shared__ int32_t hist[kMaxExperts];
    __shared__ Cand cands[kWarps][32];
    __shared__ float rows[kWarps][N * 32];
    for (int e = threadIdx.x; e < A.E; e += kThreads) hist[e] = 0;
    __syncthreads();
    const int lane = threadIdx.x & 31, per = A.per, group = lane / per, sub = lane % per;
    const int e0 = group * A.group_size + sub * A.lane_n;
    const int left_n = group < A.groups ? A.group_size - sub * A.lane_n : 0, mine_n = left_n < 0 ? 0 : left_n < A.lane_n ? left_n : A.lane_n;
    const bool full = __all_sync(kFullMask, mine_n == N), biased = SCORE == kSigmoid && A.bias;
    Cand *cand = cands[threadIdx.x >> 5];
    const uint32_t before = (1u << lane) - 1;
    float bias[N], bias_max = 0.f;
#pragma unroll
    for (int j = 0; j < N; ++j) {
        bias[j] = biased && j < mine_n ? A.bias[e0 + j] : 0.f;
        bias_max = fmaxf(bias_max, fabsf(bias[j]) < INFINITY ? fabsf(bias[j]) : 0.f);
        if (j < mine_n && !choosable(bias[j])) bias[j] = -INFINITY;
    }
    // How far a quick choice may be from the fp32 one: the score's 2^-21 and the sum's rounding, with room to spare.
    const float off = 0x1p-20f * (2.f + lanes_max(bias_max));
    // The top_groups best of the groups' scores `a` (in all lanes of a group); false where that hangs on less than `far` or a tie.
    auto take_groups = [&](float a, float far, bool &taken) {
        const uint32_t key = group < A.groups && choosable(a) ? order_key(a) : 0u;
        uint32_t left = key, least = 0;
        for (int g = 0; g < A.top_groups; ++g) {
            least = lanes_max(left);
            if (left == least) left = 0;
        }
        const uint32_t next = lanes_max(left);
        taken = least && key >= least;
        return __popc(__ballot_sync(kFullMask, taken && sub == 0)) == A.top_groups && (!next || key_value(least) - key_value(next) > far);
    };
    auto load = [&](int64_t t, float(&x)[N]) {
        if (A.vec) {
            load_logits<F32, N>(A, t, e0, x);
        } else {
#pragma unroll
            for (int j = 0; j < N; ++j) x[j] = j < mine_n ? load1<F32>(A.x, t * A.ld + e0 + j) : -INFINITY;
        }
    };
    const uint32_t tokens = uint32_t(A.tokens), step = gridDim.x * kWarps;  // (t + step stays below 2^32)
    uint32_t t = blockIdx.x * kWarps + (threadIdx.x >> 5);
    float x[N];
    if (t < tokens) load(t, x);
    for (; t < tokens; t += step) {
        float next[N];  // the token after, under way
        if (t + step < tokens) load(t + step, next);
        bool fine = true;
        if (full) {
#pragma unroll
            for (int j = 0; j < N; ++j) fine = fine && fabsf(x[j]) < INFINITY;
        } else {
#pragma unroll
            for (int j = 0; j < N; ++j) fine = fine && (fabsf(x[j]) < INFINITY || j >= mine_n);
        }
        bool easy = __all_sync(kFullMask, fine);
        float row_max = 0.f;
        if (SCORE == kSoftmax || (SCORE == kLogits && !A.sigmoid && !A.renorm)) {
            float m = x[0];
#pragma unroll
            for (int j = 1; j < N; ++j) m = fmaxf(m, x[j]);
            row_max = key_value(lanes_max(order_key(m)));
        }
        float c[N], top = -INFINITY, second = -INFINITY;  // what experts are chosen by, and the lane's two largest
        bool taken = true;
        if constexpr (SCORE == kLogits) {
#pragma unroll
            for (int j = 0; j < N; ++j) c[j] = x[j];
            if (A.groups > 1) {  // by their largest logit
                float a = c[0];
#pragma unroll
                for (int j = 1; j < N; ++j) a = fmaxf(a, c[j]);
                for (int d = 1; d < per; d <<= 1) a = fmaxf(a, __shfl_xor_sync(kFullMask, a, d));
                easy = take_groups(a, 0.f, taken) && easy;
            }
        } else {
            float a1 = -INFINITY, a2 = -INFINITY;
#pragma unroll
            for (int j = 0; j < N; ++j) {
                float s = SCORE == kSigmoid ? quick_sigmoid(x[j]) + bias[j] : quick_exp(x[j] - row_max);
                if (!full && j >= mine_n) s = -INFINITY;
                merge_two(a1, a2, s, -INFINITY);
                c[j] = biased ? s : x[j];
            }
            top = a1;
            second = a2;
            if (A.groups > 1) {
                for (int d = 1; d < per; d <<= 1) {
                    const float b1 = __shfl_xor_sync(kFullMask, a1, d), b2 = __shfl_xor_sync(kFullMask, a2, d);
                    merge_two(a1, a2, b1, b2);
                }
                const float a = A.group_top == 2 && choosable(a2) ? a1 + a2 : a1;
                easy = take_groups(a, 6.f * off, taken) && easy;
            }
        }
        if (!biased) {
            top = second = -INFINITY;
#pragma unroll
            for (int j = 0; j < N; ++j) merge_two(top, second, c[j], -INFINITY);
        }
        uint32_t left = taken && choosable(top) ? order_key(top) : 0u, then = taken && choosable(second) ? order_key(second) : 0u;
        uint32_t best = 0, first = 0;
        for (int i = 0; i < A.k; ++i) {
            best = lanes_max(left);
            if (i == 0) first = best;
            if (left == best) left = then, then = 0;
        }
        float least = best ? key_value(best) : -INFINITY;
        if (biased) least -= 2.f * off;
        least = taken ? fmaxf(least, -FLT_MAX) : INFINITY;
        // their places: in the order of their indices
        uint32_t some = 0;
#pragma unroll
        for (int j = 0; j < N; ++j) some += c[j] >= least;
        int at = 0, n = 0;
#pragma unroll
        for (int i = 0; 1 << i <= N; ++i) {
            const uint32_t who = __ballot_sync(kFullMask, some >> i & 1);
            at += __popc(who & before) << i;
            n += __popc(who) << i;
        }
        if (n <= 32) {
#pragma unroll
            for (int j = 0; j < N; ++j)
                if (c[j] >= least) cand[at++] = Cand{c[j], e0 + j, x[j], bias[j]};
        }
        __syncwarp();
        if (!easy || n > 32) {
            route_hard_token<F32, N>(A, t, hist, rows[threadIdx.x >> 5]);
        } else {
            Cand own{-INFINITY, -1, -INFINITY, 0.f};
            if (lane < n) own = cand[lane];
            float s = 0.f;  // the score, up to the row's or the chosen's sum
            if (A.sigmoid) s = sigmoid(own.x);
            if (biased) {
                own.c = s + own.bias;
                if (lane < n) cand[lane].c = own.c;
                __syncwarp();
            }
            int rank = lane < n ? 0 : lane;  // slots from n on find no expert
            if (lane < n)
                for (int i = 0; i < n; ++i) {
                    const float o = cand[i].c;
                    rank += o > own.c || (o == own.c && i < lane);
                }
            const bool is = lane < n && rank < A.k;
            if (!A.sigmoid) {
                if (A.renorm) {
                    s = expf(own.x - key_value(first));  // the largest of the chosen
                } else {
                    float sum = 0.f;
#pragma unroll
                    for (int j = 0; j < N; ++j) sum += expf(x[j] - row_max);
                    s = expf(own.x - row_max) / lanes_sum(sum);
                }
            }
            if (!is) s = 0.f;
            if (A.renorm) s = share_of(s, lanes_sum(s));
            if (rank < A.k) {
                const int64_t at = int64_t(t) * A.k + rank;
                A.chosen[at] = own.e;
                A.weights[at] = s * A.scale;
                if (is && A.counts) atomicAdd(hist + own.e, 1);
            }
        }
        __syncwarp();
#pragma unroll
        for (int j = 0; j < N; ++j) x[j] = next[j];
    }
    put_counts(A, hist);
}

struct GateGradArgs {
    const void *x;
    const int32_t *chosen;
    const float *dw;
    void *dx;
    int64_t ld, ld_out, tokens;
    int32_t E, k, kp_log2, sigmoid, renorm, flat;
    float scale;
};

// Sums and maxima over a token's 2^log2 lanes.
__device__ __forceinline__ float slots_sum(float v, int log2) {
    for (int d = 1 << log2 >> 1; d; d >>= 1) v += __shfl_xor_sync(kFullMask, v, d);
    return v;
}
__device__ __forceinline__ float slots_max(float v, int log2) {
    for (int d = 1 << log2 >> 1; d; d >>= 1) v = fmaxf(v, __shfl_xor_sync(kFullMask, v, d));
    return v;
}

// Scores whose gradient is zero but for the chosen: with q the weights over `scale`,
//   softmax, renormalised   dx = scale q (g - sum g q)
//   sigmoid, renormalised   dx = scale q (g - sum g q) (1 - s)
//   sigmoid                 dx = scale g s (1 - s)
// A warp writes its tokens' rows as zeros while its loads are under way, then the chosen over them.
template <bool F32>
__global__ void __launch_bounds__(kThreads) k_gate_grad_chosen(const __grid_constant__ GateGradArgs A) {
    const int lane = threadIdx.x & 31, slot = lane & ((1 << A.kp_log2) - 1), tt = lane >> A.kp_log2, per_warp = 32 >> A.kp_log2;
    const float zero[8] = {};
    for (int64_t w = int64_t(blockIdx.x) * kWarps + (threadIdx.x >> 5); w * per_warp < A.tokens; w += int64_t(gridDim.x) * kWarps) {
        const int64_t t0 = w * per_warp, t = t0 + tt;
        const int n = int(A.tokens - t0 < per_warp ? A.tokens - t0 : per_warp);
        int e = -1;
        float g = 0.f;
        if (tt < n && slot < A.k) {
            e = A.chosen[t * A.k + slot];
            g = A.dw[t * A.k + slot];
        }
        if (uint32_t(e) >= uint32_t(A.E)) e = -1, g = 0.f;
        float x = -INFINITY;
        if (e >= 0) x = load1<F32>(A.x, t * A.ld + e);
        if (A.flat) {  // whole 8-element units, rows one after another
            const int units = n * A.E >> 3;
            for (int u = lane; u < units; u += 32) store8<F32>(A.dx, t0 * A.E + 8 * u, zero);
            if ((units << 3) + lane < n * A.E) store1<F32>(A.dx, t0 * A.E + (units << 3) + lane, 0.f);
        } else {
            for (int r = 0; r < n; ++r)
                for (int i = lane; i < A.E; i += 32) store1<F32>(A.dx, (t0 + r) * A.ld_out + i, 0.f);
        }
        __syncwarp();  // zeros before values
        float q, rest = 1.f;  // weight over `scale` before its sum; 1 - s
        if (A.sigmoid) {
            q = e >= 0 ? sigmoid(x) : 0.f;
            rest = sigmoid(-x);
        } else {
            const float top = slots_max(x, A.kp_log2);
            q = e >= 0 && top > -INFINITY ? expf(x - top) : 0.f;
        }
        if (A.renorm) {
            const float sum = slots_sum(q, A.kp_log2);
            q = sum == 0.f ? 0.f : q / sum;
            g -= slots_sum(e >= 0 ? g * q : 0.f, A.kp_log2);
        }
        if (e >= 0) store1<F32>(A.dx, t * A.ld_out + e, A.scale * q * g * rest);
    }
}

// The softmax itself: dx_j = scale p_j (g_j - sum g p), g zero but for the chosen. A warp to a token.
template <bool F32, int N>
__global__ void __launch_bounds__(kThreads) k_gate_grad_softmax(const __grid_constant__ GateGradArgs A) {
    extern __shared__ __align__(16) float dyn[];
    const int lane = threadIdx.x & 31;
    float *row = dyn + (threadIdx.x >> 5) * (N * 32);
    for (int64_t t = int64_t(blockIdx.x) * kWarps + (threadIdx.x >> 5); t < A.tokens; t += int64_t(gridDim.x) * kWarps) {
        int e = -1;
        float g = 0.f;
        if (lane < A.k) {
            e = A.chosen[t * A.k + lane];
            if (uint32_t(e) < uint32_t(A.E))
                g = A.dw[t * A.k + lane];
            else
                e = -1;
        }
        float p[N], m = -INFINITY;
#pragma unroll
        for (int j = 0; j < N; ++j) {
            p[j] = lane + 32 * j < A.E ? load1<F32>(A.x, t * A.ld + lane + 32 * j) : -INFINITY;
            m = fmaxf(m, p[j]);
        }
        m = lanes_max(m);
        if (m == -INFINITY) m = 0.f;
        float s = 0.f;
#pragma unroll
        for (int j = 0; j < N; ++j) s += p[j] = expf(p[j] - m);
        s = lanes_sum(s);
        const float r = s == 0.f ? 0.f : 1.f / s;
#pragma unroll
        for (int j = 0; j < N; ++j) row[lane + 32 * j] = p[j] *= r;
        __syncwarp();
        const float pe = e >= 0 ? row[e] : 0.f;
        const float dot = lanes_sum(e >= 0 ? g * pe : 0.f);
        __syncwarp();
#pragma unroll
        for (int j = 0; j < N; ++j) row[lane + 32 * j] = -A.scale * p[j] * dot;
        __syncwarp();
        if (e >= 0) row[e] = A.scale * pe * (g - dot);
        __syncwarp();
#pragma unroll
        for (int j = 0; j < N; ++j)
            if (lane + 32 * j < A.E) store1<F32>(A.dx, t * A.ld_out + lane + 32 * j, row[lane + 32 * j]);
        __syncwarp();
    }
}

int check(const skew_gate_config_t *c) {
    if (!c) return ops_fail(SKEW_EINVAL, "config is NULL");
    if (c->experts < 1 || c->experts > kMaxExperts) return ops_fail(SKEW_EINVAL, "experts must be in [1, %d]", kMaxExperts);
    if (c->groups < 1 || c->groups > kMaxGroups || c->experts % c->groups) return ops_fail(SKEW_EINVAL, "groups must divide experts and be at most %d", kMaxGroups);
    if (c->top_groups < 1 || c->top_groups > c->groups) return ops_fail(SKEW_EINVAL, "top_groups must be in [1, groups]");
    if (c->group_top < 1 || c->group_top > 2) return ops_fail(SKEW_EINVAL, "group_top must be 1 or 2");
    const int most = c->experts / c->groups * c->top_groups;
    if (c->top_k < 1 || c->top_k > most || c->top_k > kMaxK)
        return ops_fail(SKEW_EINVAL, "top_k must be in [1, %d]", most < kMaxK ? most : kMaxK);
    if (c->score != SKEW_GATE_SOFTMAX && c->score != SKEW_GATE_SIGMOID) return ops_fail(SKEW_EINVAL, "unknown score %d", c->score);
    if (c->flags & ~(SKEW_GATE_RENORM | SKEW_GATE_FP32)) return ops_fail(SKEW_EINVAL, "unknown flags");
    if (!std::isfinite(c->scale)) return ops_fail(SKEW_EINVAL, "scale must be finite");
    return SKEW_OK;
}

int check_rows(const skew_gate_config_t *c, const char *what, const void *p, int64_t ld, int64_t tokens) {
    const uintptr_t es = c->flags & SKEW_GATE_FP32 ? 4 : 2;
    if ((tokens && !p) || ((uintptr_t)p & (es - 1))) return ops_fail(SKEW_EINVAL, "%s must be a device pointer aligned to its type", what);
    if (ld < c->experts || ld > int64_t(1) << 31) return ops_fail(SKEW_EINVAL, "%s: row stride must be in [experts, 2^31]", what);
    return SKEW_OK;
}

bool misaligned4(const void *p) { return !p || ((uintptr_t)p & 3); }

size_t gate_ws_bytes(const skew_gate_config_t *c) { return (size_t(c->experts) + 1) * 4; }

uint32_t grid_for(int64_t warps, int per_sm) {
    const int64_t most = int64_t(ops_sm_count()) * per_sm, need = (warps + kWarps - 1) / kWarps;
    return (uint32_t)(need < 1 ? 1 : need < most ? need : most < 1 ? 1 : most);
}

template <bool F32, int KM>
cudaError_t launch_thread(GateArgs &A, cudaStream_t s) {
    const bool shows = A.bias || (A.groups > 1 && A.group_top == 2);
    A.warp_floats = 32 * ((A.E | 1) * (shows ? 2 : 1) + (A.groups > 1 ? A.groups | 1 : 0));
    // one warp to a CTA until that fills the SMs
    const int64_t need = (A.tokens + 31) / 32, sms = ops_sm_count() > 0 ? ops_sm_count() : 1;
    const int warps = need > 8 * sms ? 2 : 1;
    const int64_t ctas = (need + warps - 1) / warps, most = 16 * sms;
    return ops_launch(false, k_gate_thread<F32, KM>, uint32_t(ctas < 1 ? 1 : ctas < most ? ctas : most), 32 * warps, size_t(warps) * A.warp_floats * sizeof(float), s, A);
}

// A warp to a token, N experts to a lane (a multiple of 4, so that vectors can be loaded).
template <bool F32, int N>
cudaError_t launch_wide(GateArgs &A, bool quick, cudaStream_t s) {
    const bool shows = A.bias || (A.groups > 1 && A.group_top == 2);
    const uint32_t grid = grid_for(A.tokens, N == 16 ? 2 : 3);
    constexpr uintptr_t kAlign = N * (F32 ? 4 : 2) < 16 ? N * (F32 ? 4 : 2) : 16;
    // rows on such boundaries; each lane's experts at its lane number times N
    A.vec = A.E % N == 0 && A.ld * (F32 ? 4 : 2) % kAlign == 0 && ((uintptr_t)A.x & (kAlign - 1)) == 0 &&
            (!quick || (A.lane_n == N && (A.groups == 1 || A.group_size == A.per * N)));
    auto go = [&](auto k) { return ops_launch(false, k, grid, kThreads, 0, s, A); };
    if (!quick) return go(k_gate<F32, N>);
    return !shows ? go(k_gate_wide<F32, N, kLogits>) : A.sigmoid ? go(k_gate_wide<F32, N, kSigmoid>) : go(k_gate_wide<F32, N, kSoftmax>);
}

template <bool F32>
cudaError_t pick_gate(GateArgs &A, cudaStream_t s) {
    if (A.E <= kThreadExperts && A.tokens >= kThreadTokens * A.E)
        return A.k <= 2 ? launch_thread<F32, 2>(A, s) : A.k <= 4 ? launch_thread<F32, 4>(A, s) : A.k <= 8 ? launch_thread<F32, 8>(A, s)
             : A.k <= 16 ? launch_thread<F32, 16>(A, s) : launch_thread<F32, 32>(A, s);
    const bool shows = A.bias || (A.groups > 1 && A.group_top == 2);
    A.per = 32;
    while (A.per * A.groups > 32) A.per >>= 1;
    A.lane_n = (A.group_size + A.per - 1) / A.per;
    if (A.groups == 1 && A.E % 4 == 0) A.lane_n = A.E <= 128 ? 4 : A.E <= 256 ? 8 : 16;  // vectors
    // not so: few lanes to large groups; scores that need the row's sum to be chosen by, or to be weights (8 of 256 by softmax
    // scores and a bias, 65536 tokens: 82 us)
    const bool quick = A.lane_n <= 16 && !(A.bias && !A.sigmoid) && !(shows && !A.sigmoid && !A.renorm);
    const int n = quick ? A.lane_n : (A.E + 31) / 32;
    return n <= 4 ? launch_wide<F32, 4>(A, quick, s) : n <= 8 ? launch_wide<F32, 8>(A, quick, s) : launch_wide<F32, 16>(A, quick, s);
}

template <bool F32, int N>
cudaError_t launch_softmax_grad(const GateGradArgs &A, cudaStream_t s) {
    return ops_launch(false, k_gate_grad_softmax<F32, N>, grid_for(A.tokens, 8), kThreads, kWarps * N * 32 * sizeof(float), s, A);
}

template <bool F32>
cudaError_t pick_grad(GateGradArgs &A, cudaStream_t s) {
    if (!A.sigmoid && !A.renorm) {
        if (A.E <= 32) return launch_softmax_grad<F32, 1>(A, s);
        if (A.E <= 64) return launch_softmax_grad<F32, 2>(A, s);
        if (A.E <= 128) return launch_softmax_grad<F32, 4>(A, s);
        if (A.E <= 256) return launch_softmax_grad<F32, 8>(A, s);
        return launch_softmax_grad<F32, 16>(A, s);
    }
    while (1 << A.kp_log2 < A.k) ++A.kp_log2;
    const int per_warp = 32 >> A.kp_log2;
    A.flat = A.ld_out == A.E && ((uintptr_t)A.dx & 15) == 0 && per_warp * A.E % 8 == 0;
    return ops_launch(false, k_gate_grad_chosen<F32>, grid_for((A.tokens + per_warp - 1) / per_warp, 8), kThreads, 0, s, A);
}

}  // namespace
}  // namespace skew

using namespace skew;

extern "C" {

size_t skew_gate_workspace_bytes(const skew_gate_config_t *c) { return check(c) == SKEW_OK ? gate_ws_bytes(c) : 0; }

int skew_gate_forward(const skew_gate_config_t *c, const void *logits, int64_t ld, const float *bias, int64_t tokens, int32_t *chosen,
                      float *weights, int32_t *counts, void *workspace, size_t workspace_bytes, void *stream) {
    if (const int rc = check(c)) return rc;
    if (tokens < 0 || tokens > INT32_MAX) return ops_fail(SKEW_EINVAL, "tokens must be in [0, 2^31)");
    if (const int rc = check_rows(c, "logits", logits, ld, tokens)) return rc;
    if (bias && misaligned4(bias)) return ops_fail(SKEW_EINVAL, "bias must be 4-byte aligned");
    if (tokens && (misaligned4(chosen) || misaligned4(weights))) return ops_fail(SKEW_EINVAL, "chosen and weights must be 4-byte aligned device pointers");
    if (counts && (misaligned4(counts) || misaligned4(workspace) || workspace_bytes < gate_ws_bytes(c)))
        return ops_fail(SKEW_EINVAL, "counts need a 4-byte aligned workspace of %zu bytes", gate_ws_bytes(c));
    if (!tokens && !counts) return SKEW_OK;
    GateArgs A{};
    A.x = logits;
    A.bias = bias;
    A.chosen = chosen;
    A.weights = weights;
    A.counts = counts;
    A.ws = (uint32_t *)workspace;
    A.ld = ld;
    A.tokens = tokens;
    A.E = c->experts;
    A.k = c->top_k;
    A.groups = c->groups;
    A.top_groups = c->top_groups;
    A.group_top = c->group_top;
    A.group_size = c->experts / c->groups;
    A.sigmoid = c->score == SKEW_GATE_SIGMOID;
    A.renorm = (c->flags & SKEW_GATE_RENORM) != 0;
    A.scale = c->scale;
    return ops_cuda(c->flags & SKEW_GATE_FP32 ? pick_gate<true>(A, (cudaStream_t)stream) : pick_gate<false>(A, (cudaStream_t)stream), "k_gate");
}

int skew_gate_grad(const skew_gate_config_t *c, const void *logits, int64_t ld, const int32_t *chosen, const float *dweights, int64_t tokens,
                   void *dlogits, int64_t ld_out, void *stream) {
    if (const int rc = check(c)) return rc;
    if (tokens < 0 || tokens > INT32_MAX) return ops_fail(SKEW_EINVAL, "tokens must be in [0, 2^31)");
    if (const int rc = check_rows(c, "logits", logits, ld, tokens)) return rc;
    if (const int rc = check_rows(c, "dlogits", dlogits, ld_out, tokens)) return rc;
    if (!tokens) return SKEW_OK;
    if (misaligned4(chosen) || misaligned4(dweights)) return ops_fail(SKEW_EINVAL, "chosen and dweights must be 4-byte aligned device pointers");
    GateGradArgs A{};
    A.x = logits;
    A.chosen = chosen;
    A.dw = dweights;
    A.dx = dlogits;
    A.ld = ld;
    A.ld_out = ld_out;
    A.tokens = tokens;
    A.E = c->experts;
    A.k = c->top_k;
    A.sigmoid = c->score == SKEW_GATE_SIGMOID;
    A.renorm = (c->flags & SKEW_GATE_RENORM) != 0;
    A.scale = c->scale;
    return ops_cuda(c->flags & SKEW_GATE_FP32 ? pick_grad<true>(A, (cudaStream_t)stream) : pick_grad<false>(A, (cudaStream_t)stream), "k_gate_grad");
}

}  // extern "C"
