// Routing of tokens to experts and its gradient (skew_gate_* in include/skewadam.h).
//
// Forward: L lanes of a warp own a token, N consecutive logits each. Scores and choices stay in registers;
// an expert is picked as the maximum over the lanes' own maxima of order-preserving integer keys, the lowest
// lane first among equals, so ties go to the lowest index. Reads the logits once (bound by memory at few
// experts a token, by instructions at many).
//
// Backward: as many lanes as top_k, rounded up to a power of two, own a token, one chosen expert each. Only the
// softmax that is not renormalised has a gradient elsewhere, and reads whole rows.
#include "skew_ops.h"

#include <cfloat>
#include <cmath>

namespace skew {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kMaxExperts = 512, kMaxK = 32, kMaxGroups = 32;

struct GateArgs {
    const void *x;
    const float *bias;
    int32_t *chosen;
    float *weights;
    int32_t *counts;
    uint32_t *ws;  // [0, E): tokens of each expert so far, [E]: CTAs done; zero between calls
    int64_t ld, tokens;
    int32_t E, k, groups, top_groups, group_top, group_size, sigmoid, renorm, vec;
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

template <int L>
__device__ __forceinline__ uint32_t lanes_max(uint32_t v) {
    if constexpr (L == 32) {
        return __reduce_max_sync(kFullMask, v);
    } else {
#pragma unroll
        for (int d = L / 2; d; d >>= 1) v = max(v, __shfl_xor_sync(kFullMask, v, d));
        return v;
    }
}

template <int L>
__device__ __forceinline__ float lanes_max(float v) {
#pragma unroll
    for (int d = L / 2; d; d >>= 1) v = fmaxf(v, __shfl_xor_sync(kFullMask, v, d));
    return v;
}

template <int L>
__device__ __forceinline__ float lanes_sum(float v) {
#pragma unroll
    for (int d = L / 2; d; d >>= 1) v += __shfl_xor_sync(kFullMask, v, d);
    return v;
}

// The two largest of (a1 >= a2) and (b1 >= b2).
__device__ __forceinline__ void merge_two(float &a1, float &a2, float b1, float b2) {
    a2 = fmaxf(fminf(a1, b1), fmaxf(a2, b2));
    a1 = fmaxf(a1, b1);
}

// A lane's N logits from `e0` on; what lies past E, and rows past the last, as -Inf.
template <bool F32, int N>
__device__ __forceinline__ void load_logits(const GateArgs &A, int64_t t, bool there, int e0, float (&x)[N]) {
    if (there && A.vec && e0 < A.E) {
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
        for (int j = 0; j < N; ++j) x[j] = there && e0 + j < A.E ? load1<F32>(A.x, t * A.ld + e0 + j) : -INFINITY;
    }
}

// Routes 32 / L tokens from t0 on, whatever they and the config hold.
template <bool F32, int L, int N>
__device__ __forceinline__ void route_tokens(const GateArgs &A, int64_t t0, int32_t *hist, float *rows) {
    constexpr int SL = N < kMaxK / L ? N : kMaxK / L;  // chosen experts a lane keeps
    const int lane = threadIdx.x & 31, l = lane & (L - 1), e0 = l * N;
    const uint32_t lanes = L == 32 ? kFullMask : ((1u << (L & 31)) - 1) << (lane & ~(L - 1));
    const bool shows = A.bias || (A.groups > 1 && A.group_top == 2);
    const bool whole_lanes = A.group_size % N == 0 && ((A.group_size / N) & (A.group_size / N - 1)) == 0;
    float bias[N];
#pragma unroll
    for (int j = 0; j < N; ++j) bias[j] = A.bias && e0 + j < A.E ? A.bias[e0 + j] : 0.f;
    const int64_t t = t0 + lane / L;
    const bool there = t < A.tokens;
    float x[N];
    load_logits<F32, N>(A, t, there, e0, x);
    bool is_nan = false;
#pragma unroll
    for (int j = 0; j < N; ++j) is_nan |= x[j] != x[j];
    const bool nan = (__ballot_sync(kFullMask, is_nan) & lanes) != 0;

    // what experts are chosen by: the logits (they order as the scores do), or the scores plus the bias
    float shown[N], row_max = 0.f, row_sum = 0.f;
    uint32_t key[N];
    if (!A.sigmoid && (shows || !A.renorm)) {
        float m = -INFINITY;
#pragma unroll
        for (int j = 0; j < N; ++j) m = fmaxf(m, x[j]);
        row_max = lanes_max<L>(m);
        if (row_max == -INFINITY) row_max = 0.f;
        float s = 0.f;
#pragma unroll
        for (int j = 0; j < N; ++j) {
            shown[j] = expf(x[j] - row_max);  // without a bias the row's sum changes no order
            s += shown[j];
        }
        row_sum = lanes_sum<L>(s);
        if (A.bias)
#pragma unroll
            for (int j = 0; j < N; ++j) shown[j] = shown[j] / row_sum + bias[j];
    } else if (shows) {
#pragma unroll
        for (int j = 0; j < N; ++j) shown[j] = sigmoid(x[j]) + bias[j];
    }
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const float c = A.bias ? shown[j] : x[j];
        key[j] = choosable(c) && choosable(x[j]) ? order_key(c) : 0u;
    }

    if (A.groups > 1) {
        uint32_t gkey = 0, taken = 0;
        int per = 1;  // lanes from one group's key to the next
        if (whole_lanes) {
            per = A.group_size / N;
            if (A.group_top == 1) {
#pragma unroll
                for (int j = 0; j < N; ++j) gkey = max(gkey, key[j]);
                for (int d = 1; d < per; d <<= 1) gkey = max(gkey, __shfl_xor_sync(kFullMask, gkey, d));
            } else {
                float a1 = -INFINITY, a2 = -INFINITY;
#pragma unroll
                for (int j = 0; j < N; ++j) merge_two(a1, a2, key[j] ? shown[j] : -INFINITY, -INFINITY);
                for (int d = 1; d < per; d <<= 1) {
                    const float b1 = __shfl_xor_sync(kFullMask, a1, d), b2 = __shfl_xor_sync(kFullMask, a2, d);
                    merge_two(a1, a2, b1, b2);
                }
                if (choosable(a1)) gkey = order_key(choosable(a2) ? a1 + a2 : a1);
            }
            if (l % per) gkey = 0;
        } else if constexpr (L == 32) {  // one lane to a group
            float *row = rows + (threadIdx.x >> 5) * kMaxExperts;
            uint32_t *keys = reinterpret_cast<uint32_t *>(row);
            if (A.group_top == 1) {
#pragma unroll
                for (int j = 0; j < N; ++j) keys[e0 + j] = key[j];
                __syncwarp();
                if (l < A.groups)
                    for (int i = 0; i < A.group_size; ++i) gkey = max(gkey, keys[l * A.group_size + i]);
            } else {
#pragma unroll
                for (int j = 0; j < N; ++j) row[e0 + j] = key[j] ? shown[j] : -INFINITY;
                __syncwarp();
                float a1 = -INFINITY, a2 = -INFINITY;
                if (l < A.groups)
                    for (int i = 0; i < A.group_size; ++i) merge_two(a1, a2, row[l * A.group_size + i], -INFINITY);
                if (choosable(a1)) gkey = order_key(choosable(a2) ? a1 + a2 : a1);
            }
            __syncwarp();
        }
        for (int g = 0; g < A.top_groups; ++g) {
            const uint32_t best = lanes_max<L>(gkey);
            const uint32_t who = __ballot_sync(kFullMask, gkey == best) & lanes;
            const int win = __ffs(who) - 1;
            if (best) taken |= 1u << ((win & (L - 1)) / per);
            if (lane == win) gkey = 0;
        }
        if (whole_lanes) {
            if (!(taken >> (l / per) & 1))
#pragma unroll
                for (int j = 0; j < N; ++j) key[j] = 0;
        } else {
#pragma unroll
            for (int j = 0; j < N; ++j)
                if (e0 + j >= A.E || !(taken >> ((e0 + j) / A.group_size) & 1)) key[j] = 0;
        }
    }

    // the k largest, one after another
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < N; ++j) m = max(m, key[j]);
    int32_t mine[SL];
#pragma unroll
    for (int q = 0; q < SL; ++q) mine[q] = -1;
    for (int i = 0; i < A.k; ++i) {
        const uint32_t best = lanes_max<L>(m);
        const int win = __ffs(__ballot_sync(kFullMask, m == best) & lanes) - 1;
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
#pragma unroll
        for (int q = 0; q < SL; ++q)
            if (best && i == q * L + l) mine[q] = e;
    }

    // weights of the chosen
    float sc[SL], sum = 0.f;
    if (A.sigmoid || !A.renorm) {
#pragma unroll
        for (int q = 0; q < SL; ++q) {
            const float xc = mine[q] >= 0 ? load1<F32>(A.x, t * A.ld + mine[q]) : -INFINITY;
            sc[q] = A.sigmoid ? sigmoid(xc) : mine[q] >= 0 ? expf(xc - row_max) / row_sum : 0.f;
            sum += sc[q];
        }
    } else {  // the softmax of the chosen
        float top = -INFINITY;
#pragma unroll
        for (int q = 0; q < SL; ++q) {
            sc[q] = mine[q] >= 0 ? load1<F32>(A.x, t * A.ld + mine[q]) : -INFINITY;
            top = fmaxf(top, sc[q]);
        }
        top = lanes_max<L>(top);
#pragma unroll
        for (int q = 0; q < SL; ++q) {
            sc[q] = mine[q] >= 0 ? expf(sc[q] - top) : 0.f;
            sum += sc[q];
        }
    }
    float by = A.scale;
    if (A.renorm) {
        sum = lanes_sum<L>(sum);
        by = sum == 0.f ? 0.f : A.scale / sum;
    }
#pragma unroll
    for (int q = 0; q < SL; ++q) {
        const int i = q * L + l;
        if (there && i < A.k) {
            A.chosen[t * A.k + i] = mine[q];
            A.weights[t * A.k + i] = nan ? NAN : sc[q] * by;
            if (A.counts && mine[q] >= 0) atomicAdd(hist + mine[q], 1);
        }
    }
}

// Adds the CTA's counts to those of all CTAs; the last one hands them out and leaves zeros.
__device__ __forceinline__ void put_counts(const GateArgs &A, const int32_t *hist) {
    if (!A.counts) return;
    __syncthreads();
    if (gridDim.x == 1) {
        for (int e = threadIdx.x; e < A.E; e += kThreads) A.counts[e] = hist[e];
        return;
    }
    for (int e = threadIdx.x; e < A.E; e += kThreads)
        if (hist[e]) atomicAdd(A.ws + e, (uint32_t)hist[e]);
    __shared__ bool last;
    __threadfence();
    __syncthreads();
    if (threadIdx.x == 0) last = atomicInc(A.ws + A.E, gridDim.x - 1) == gridDim.x - 1;  // back at 0
    __syncthreads();
    if (!last) return;
    __threadfence();
    for (int e = threadIdx.x; e < A.E; e += kThreads) A.counts[e] = (int32_t)atomicExch(A.ws + e, 0u);
}

template <bool F32, int L, int N>
__global__ void __launch_bounds__(kThreads, 4) k_gate(const __grid_constant__ GateArgs A) {
    constexpr int TPW = 32 / L;     // tokens a warp takes at a time
    extern __shared__ float dyn[];  // shown values, where groups do not end with lanes
    __shared__ int32_t hist[kMaxExperts];
    for (int e = threadIdx.x; e < A.E; e += kThreads) hist[e] = 0;
    __syncthreads();
    for (int64_t w = int64_t(blockIdx.x) * kWarps + (threadIdx.x >> 5); w * TPW < A.tokens; w += int64_t(gridDim.x) * kWarps)
        route_tokens<F32, L, N>(A, w * TPW, hist, dyn);
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
__device__ __noinline__ void route_hard_token(const GateArgs &A, int64_t t, int32_t *hist) {
    route_tokens<F32, 32, N>(A, t, hist, nullptr);
}

// A warp to a token, for configs whose groups are whole lanes. Near ties aside, quick scores settle which groups are
// taken, and which experts may be among the top_k: at least k values are no less than the k-th of the lanes' largest, and
// few more; a lane to one of those, with its fp32 score, ranks it among the others. A token that this does not settle
// (near ties, a logit that is not finite, over 32 such experts) takes route_tokens.
// SCORE: kLogits (experts and groups by the logits alone), kSigmoid, kSoftmax (both: quick scores are needed).
enum { kLogits, kSigmoid, kSoftmax };
template <bool F32, int N, int SCORE>
__global__ void __launch_bounds__(kThreads, N == 16 ? 2 : 3) k_gate_wide(const __grid_constant__ GateArgs A) {
    __shared__ int32_t hist[kMaxExperts];
    __shared__ Cand cands[kWarps][32];
    const int lane = threadIdx.x & 31, e0 = lane * N;
    for (int e = threadIdx.x; e < A.E; e += kThreads) hist[e] = 0;
    __syncthreads();
    Cand *cand = cands[threadIdx.x >> 5];
    const uint32_t before = (1u << lane) - 1;
    const bool full = A.E == 32 * N, biased = SCORE == kSigmoid && A.bias;
    const int per = A.group_size / N, group = lane / per;  // (one group: unused)
    float bias[N], bias_max = 0.f;
#pragma unroll
    for (int j = 0; j < N; ++j) {
        bias[j] = biased && e0 + j < A.E ? A.bias[e0 + j] : 0.f;
        bias_max = fmaxf(bias_max, fabsf(bias[j]) < INFINITY ? fabsf(bias[j]) : 0.f);
        if (e0 + j < A.E && !choosable(bias[j])) bias[j] = -INFINITY;
    }
    // How far a quick choice may be from the fp32 one: the score's 2^-21 and the sum's rounding, with room to spare.
    const float off = 0x1p-20f * (2.f + lanes_max<32>(bias_max));
    // The top_groups best of the groups' scores `a` (in all lanes of a group); false where that hangs on less than `far` or a tie.
    auto take_groups = [&](float a, float far, bool &taken) {
        const uint32_t key = group < A.groups && choosable(a) ? order_key(a) : 0u;
        uint32_t left = key, least = 0;
        for (int g = 0; g < A.top_groups; ++g) {
            least = lanes_max<32>(left);
            if (left == least) left = 0;
        }
        const uint32_t next = lanes_max<32>(left);
        taken = least && key >= least;
        return __popc(__ballot_sync(kFullMask, taken && lane % per == 0)) == A.top_groups && (!next || key_value(least) - key_value(next) > far);
    };
    const uint32_t tokens = uint32_t(A.tokens), step = gridDim.x * kWarps;  // (t + step stays below 2^32)
    uint32_t t = blockIdx.x * kWarps + (threadIdx.x >> 5);
    float x[N];
    if (t < tokens) load_logits<F32, N>(A, t, true, e0, x);
    for (; t < tokens; t += step) {
        float next[N];  // the token after, under way
        if (t + step < tokens) load_logits<F32, N>(A, t + step, true, e0, next);
        bool fine = true;
        if (full) {
#pragma unroll
            for (int j = 0; j < N; ++j) fine = fine && fabsf(x[j]) < INFINITY;
        } else {
#pragma unroll
            for (int j = 0; j < N; ++j) fine = fine && (fabsf(x[j]) < INFINITY || e0 + j >= A.E);
        }
        bool easy = __all_sync(kFullMask, fine);
        float row_max = 0.f;
        if (SCORE == kSoftmax || (SCORE == kLogits && !A.sigmoid && !A.renorm)) {
            float m = x[0];
#pragma unroll
            for (int j = 1; j < N; ++j) m = fmaxf(m, x[j]);
            row_max = key_value(lanes_max<32>(order_key(m)));
        }
        float c[N];  // what experts are chosen by
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
                if (!full && e0 + j >= A.E) s = -INFINITY;
                a2 = fmaxf(fminf(a1, s), a2);
                a1 = fmaxf(a1, s);
                c[j] = biased ? s : x[j];
            }
            if (A.groups > 1) {
                for (int d = 1; d < per; d <<= 1) {
                    const float b1 = __shfl_xor_sync(kFullMask, a1, d), b2 = __shfl_xor_sync(kFullMask, a2, d);
                    merge_two(a1, a2, b1, b2);
                }
                const float a = A.group_top == 2 && choosable(a2) ? a1 + a2 : a1;
                easy = take_groups(a, 6.f * off, taken) && easy;
            }
        }
        float top = c[0];
#pragma unroll
        for (int j = 1; j < N; ++j) top = fmaxf(top, c[j]);
        uint32_t left = taken && choosable(top) ? order_key(top) : 0u, best = 0, first = 0;
        for (int i = 0; i < A.k; ++i) {
            best = lanes_max<32>(left);
            if (i == 0) first = best;
            if (left == best) left = 0;
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
            route_hard_token<F32, N>(A, t, hist);
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
            float by = A.scale;
            if (!A.sigmoid) {
                if (A.renorm) {
                    s = expf(own.x - key_value(first));  // the largest of the chosen
                } else {
                    float sum = 0.f;
#pragma unroll
                    for (int j = 0; j < N; ++j) sum += expf(x[j] - row_max);
                    s = expf(own.x - row_max) / lanes_sum<32>(sum);
                }
            }
            if (!is) s = 0.f;
            if (A.renorm) {
                const float sum = lanes_sum<32>(s);
                by = sum == 0.f ? 0.f : A.scale / sum;
            }
            if (rank < A.k) {
                const int64_t at = int64_t(t) * A.k + rank;
                A.chosen[at] = own.e;
                A.weights[at] = s * by;
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
        m = lanes_max<32>(m);
        if (m == -INFINITY) m = 0.f;
        float s = 0.f;
#pragma unroll
        for (int j = 0; j < N; ++j) s += p[j] = expf(p[j] - m);
        s = lanes_sum<32>(s);
        const float r = s == 0.f ? 0.f : 1.f / s;
#pragma unroll
        for (int j = 0; j < N; ++j) row[lane + 32 * j] = p[j] *= r;
        __syncwarp();
        const float pe = e >= 0 ? row[e] : 0.f;
        const float dot = lanes_sum<32>(e >= 0 ? g * pe : 0.f);
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

bool whole_lanes(const GateArgs &A, int N) { return A.groups == 1 || (A.group_size % N == 0 && ((A.group_size / N) & (A.group_size / N - 1)) == 0); }

template <bool F32, int L, int N>
cudaError_t launch_gate(const GateArgs &A, cudaStream_t s) {
    return ops_launch(false, k_gate<F32, L, N>, grid_for((A.tokens + 32 / L - 1) / (32 / L), 4), kThreads,
                      whole_lanes(A, N) ? 0 : kWarps * kMaxExperts * sizeof(float), s, A);
}

template <bool F32, int N>
cudaError_t launch_wide(const GateArgs &A, cudaStream_t s) {
    const bool shows = A.bias || (A.groups > 1 && A.group_top == 2);
    if (!whole_lanes(A, N) || (A.bias && !A.sigmoid) || (shows && !A.sigmoid && !A.renorm)) return launch_gate<F32, 32, N>(A, s);
    const uint32_t grid = grid_for(A.tokens, N == 16 ? 2 : 3);
    auto go = [&](auto k) { return ops_launch(false, k, grid, kThreads, 0, s, A); };
    return !shows ? go(k_gate_wide<F32, N, kLogits>) : A.sigmoid ? go(k_gate_wide<F32, N, kSigmoid>) : go(k_gate_wide<F32, N, kSoftmax>);
}

// Four logits a lane and as few lanes as hold a token; a whole warp for over 64 experts, and where groups are not whole lanes.
template <bool F32>
cudaError_t pick_gate(GateArgs &A, cudaStream_t s) {
    const int es = F32 ? 4 : 2, N = A.E <= 128 ? 4 : A.E <= 256 ? 8 : 16;
    const uintptr_t align = N * es < 16 ? N * es : 16;
    A.vec = A.E % N == 0 && A.ld * es % align == 0 && ((uintptr_t)A.x & (align - 1)) == 0;
    if (A.E <= 16 && whole_lanes(A, 4)) return launch_gate<F32, 4, 4>(A, s);
    if (A.E <= 32 && whole_lanes(A, 4)) return launch_gate<F32, 8, 4>(A, s);
    if (A.E <= 64 && whole_lanes(A, 4)) return launch_gate<F32, 16, 4>(A, s);
    if (A.E <= 128) return launch_wide<F32, 4>(A, s);
    if (A.E <= 256) return launch_wide<F32, 8>(A, s);
    return launch_wide<F32, 16>(A, s);
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
