// smoe_route_topk: the router for layers that serve k experts per token.  Scores s = softmax or sigmoid of the logits x . Wr^T, chosen
// by s + bias within the best groups, once among all experts (Eq. 1's choices and weights) and once among the resident ones (Masked
// Gating, SwapMoE Section 3.1).
//
// The product is smoe_route's (route_mfma.h); here is what follows it.  16 lanes hold a token's logits, 4 experts of every 64 a lane.  A
// round of the selection is the largest key among the 16 lanes and the lowest expert that holds it, rotations within the lanes; lane i keeps
// the i-th choice, reads its logit back from LDS and computes its weight.
//
// Which experts are chosen has to be right, and a logit in fp32 is off by some 1e-7 of |x| |w|: in a batch of 16384 tokens with 8 choices of
// 128 experts a few choices are nearer to each other than that.  So a selection also looks at the distances it decided by (between
// consecutive choices, the last one and the next best, the last kept group and the next); where one is within an estimate of the error, the token
// is put on a list, and a wave repeats it in 64 bits, products, scores and selection, from x and the router's rows in memory.
// Without a bias, and with single experts ranking the groups, the keys are the logits themselves, of which every score is a rising
// function.

#include <algorithm>
#include <cfloat>
#include <climits>
#include <cmath>
#include <type_traits>

#include "route_mfma.h"

struct smoe_topk_args : smoe_route_args {
    const float* bias;
    const float* wnorm;           // largest |w_e|
    double* logits;               // few tokens: [T, E]
    int k, sigmoid, groups, kept, best, renorm, by_logit, f32;
    int aligned;                  // a group is 4, 8, 16, 32 or 64 experts
    float scale, inv_per;         // 1 / experts of a group
    float err_norm, err_sum;      // estimated error of a logit in units of 2^-24: of |x| |w|, and of the sum of its slices' magnitudes
};

namespace {

__device__ __forceinline__ float sigmoid_of(float v) { return 1.0f / (1.0f + expf(-v)); }
// The same in a few instructions, for keys: the exponent is off by 1.5 2^-24 of its size (the constant and the product), the two instructions by a unit
// of 2^-23 each, the sum by half of one.
__device__ __forceinline__ float sigmoid_near(float v) {
    return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(v * -1.44269504f));
}
__device__ __forceinline__ float larger(float a, float b) { return fmaxf(a, b); }
__device__ __forceinline__ double larger(double a, double b) { return fmax(a, b); }
__device__ __forceinline__ int larger(int a, int b) { return max(a, b); }
__device__ __forceinline__ int smaller(int a, int b) { return min(a, b); }
__device__ __forceinline__ float smaller(float a, float b) { return fminf(a, b); }
__device__ __forceinline__ double smaller(double a, double b) { return fmin(a, b); }

// A lane's value from another of its row, by the control word of the instruction (0x120 + n: the row turned by n lanes), and the reductions of
// wave_ops.h in 64 bits.
template <int CTRL>
__device__ __forceinline__ int dpp(int v) { return __builtin_amdgcn_mov_dpp(v, CTRL, 0xf, 0xf, true); }
template <int CTRL>
__device__ __forceinline__ float dpp(float v) { return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), CTRL, 0xf, 0xf, true)); }
template <int CTRL>
__device__ __forceinline__ double dpp(double v) {
    return __hiloint2double(__builtin_amdgcn_mov_dpp(__double2hiint(v), CTRL, 0xf, 0xf, true),
                            __builtin_amdgcn_mov_dpp(__double2loint(v), CTRL, 0xf, 0xf, true));
}
// ... of integers each step is one instruction (a maximum of floats first quietens its operands, and takes three).
template <class T>
__device__ __forceinline__ T row_max(T v) {
    v = larger(v, dpp<0x128>(v));
    v = larger(v, dpp<0x124>(v));
    v = larger(v, dpp<0x122>(v));
    return larger(v, dpp<0x121>(v));
}
template <class T>
__device__ __forceinline__ T row_min(T v) {
    v = smaller(v, dpp<0x128>(v));
    v = smaller(v, dpp<0x124>(v));
    v = smaller(v, dpp<0x122>(v));
    return smaller(v, dpp<0x121>(v));
}
template <class T, int R>
__device__ __forceinline__ void row_max(T (&v)[R]) {       // step by step of all of them
#pragma unroll
    for (int r = 0; r < R; ++r) v[r] = larger(v[r], dpp<0x128>(v[r]));
#pragma unroll
    for (int r = 0; r < R; ++r) v[r] = larger(v[r], dpp<0x124>(v[r]));
#pragma unroll
    for (int r = 0; r < R; ++r) v[r] = larger(v[r], dpp<0x122>(v[r]));
#pragma unroll
    for (int r = 0; r < R; ++r) v[r] = larger(v[r], dpp<0x121>(v[r]));
}
template <int R>
__device__ __forceinline__ void row_min(int (&v)[R]) {
#pragma unroll
    for (int r = 0; r < R; ++r) v[r] = min(v[r], dpp<0x128>(v[r]));
#pragma unroll
    for (int r = 0; r < R; ++r) v[r] = min(v[r], dpp<0x124>(v[r]));
#pragma unroll
    for (int r = 0; r < R; ++r) v[r] = min(v[r], dpp<0x122>(v[r]));
#pragma unroll
    for (int r = 0; r < R; ++r) v[r] = min(v[r], dpp<0x121>(v[r]));
}
// Integers in the order of the floats, and back (of floats that are numbers).
__device__ __forceinline__ int ordered_bits(int i) { return i ^ (i >> 31 & 0x7fffffff); }
__device__ __forceinline__ int to_ordered(float v) { return ordered_bits(__float_as_int(v)); }
__device__ __forceinline__ float from_ordered(int i) { return __int_as_float(ordered_bits(i)); }
// The key of an expert whose logit is NaN: behind all numbers, in front of what cannot be had (-infinity).  Sums of two such keys are kept from
// becoming -infinity.
__device__ __forceinline__ float last_key(float) { return -FLT_MAX; }
__device__ __forceinline__ double last_key(double) { return -1e300; }
template <class T>
__device__ __forceinline__ T number_or_last(T v) { return v == v ? v : last_key(v); }

// What keys are compared as: floats as integers in their order, doubles as they are.
template <class T>
struct key_order {
    using type = T;
    static __device__ __forceinline__ T of(T v) { return v; }
    static __device__ __forceinline__ T value(T v) { return v; }
};
template <>
struct key_order<float> {
    using type = int;
    static __device__ __forceinline__ int of(float v) { return to_ordered(v); }
    static __device__ __forceinline__ float value(int v) { return from_ordered(v); }
};

template <class T>
__device__ __forceinline__ T row_sum(T v) {
    v += dpp<0x128>(v);
    v += dpp<0x124>(v);
    v += dpp<0x122>(v);
    return v + dpp<0x121>(v);
}

// e / (E / groups): e + 1/2 is at least 1/(2 per) from the next border, far more than the product's rounding
__device__ __forceinline__ int group_of(const smoe_topk_args& a, int e) { return (int)(((float)e + 0.5f) * a.inv_per); }

// How far keys may be off: by `base`, and by `rel` of themselves.  The second part is the rounding of a score's sum with its bias, so a bias that is large
// counts where its own key is compared and nowhere else.
struct key_error {
    float base, rel;
    float left_out;                                        // of every key: what a group of two has more of than a single expert
};
constexpr float HALF_STEP = 0x1p-24f;

// How far the rank of a group may be off, from its largest keys (best = 1: the first alone); 0 where the group has none.
__device__ __forceinline__ float rank_error(const smoe_topk_args& a, float m1, float m2, float rank, key_error err) {
    const float one = err.base + err.rel * fabsf(m1), two = one + err.base + err.rel * fabsf(m2) + (m1 + m2 != 0.f ? HALF_STEP * fabsf(rank) : 0.f);
    return rank == -INFINITY ? 0.f : a.best == 2 && m2 > -INFINITY ? two : one;
}

// The groups a token keeps, in its 16 lanes: the keys of all other experts become none.  Returns 2 where a group that is kept and one that is not may
// lie the other way round (fp32 keys; in 64 bits nothing is asked).
template <class T, int EC>
__device__ __forceinline__ int keep_groups(typename key_order<T>::type (&key)[EC][4], const smoe_topk_args& a, int sub, key_error err) {
    constexpr bool ASK = std::is_same<T, float>::value;
    using O = key_order<T>;
    using I = typename O::type;
    const I none = O::of(-INFINITY);
    int close = 0;
    if (a.groups > 1 && a.aligned) {
        // Groups of 4, 8, .. 64 experts: 1, 2, .. 16 neighbouring lanes of one of the lane's packs of four, so each lane finds the rank of its
        // own groups with the steps of one reduction, and counts the groups in front of each (16384 tokens, 8 groups of 16: 18 us
        // less than the walk over the groups below).
        I rank[EC];
        float off[EC];
        const int lanes = a.E / a.groups >> 2;
#pragma unroll
        for (int c = 0; c < EC; ++c) {
            const I hi0 = larger(key[c][0], key[c][1]), lo0 = smaller(key[c][0], key[c][1]);
            const I hi1 = larger(key[c][2], key[c][3]), lo1 = smaller(key[c][2], key[c][3]);
            I m1 = larger(hi0, hi1), m2 = larger(smaller(hi0, hi1), larger(lo0, lo1));
            auto merge = [&](I o1, I o2) {
                m2 = larger(smaller(m1, o1), larger(m2, o2));
                m1 = larger(m1, o1);
            };
            if (lanes >= 2) merge(dpp<0xB1>(m1), dpp<0xB1>(m2));
            if (lanes >= 4) merge(dpp<0x4E>(m1), dpp<0x4E>(m2));
            if (lanes >= 8) merge(dpp<0x141>(m1), dpp<0x141>(m2));   // the other quad of eight lanes
            if (lanes >= 16) merge(dpp<0x140>(m1), dpp<0x140>(m2));  // the other eight
            rank[c] = a.best == 2 && m2 > none ? O::of(larger(O::value(m1) + O::value(m2) + T(err.left_out), last_key(T(0)))) : m1;
            if constexpr (ASK) off[c] = rank_error(a, O::value(m1), O::value(m2), O::value(rank[c]), err);
        }
        int ahead[EC];
#pragma unroll
        for (int c = 0; c < EC; ++c) ahead[c] = 0;
        for (int s = 0; s < 16; s += lanes) {              // the row turned by s lanes: group (lane - s) / lanes of every pack
            const int at = ((threadIdx.x - s) & 15) | (threadIdx.x & 48);
#pragma unroll
            for (int o = 0; o < EC; ++o) {
                const I v = __shfl(rank[o], at);
#pragma unroll
                for (int c = 0; c < EC; ++c) {
                    const bool before = o < c || (o == c && ((at ^ threadIdx.x) & 15) && (at & 15) < (int)(threadIdx.x & 15));
                    ahead[c] += v > rank[c] || (v == rank[c] && before && (o < c || s)) ? 1 : 0;
                }
            }
        }
        float worst = INFINITY, next = -INFINITY;          // least that a kept group may have, most that another may
#pragma unroll
        for (int c = 0; c < EC; ++c) {
            if (64 * c >= a.E) continue;                   // uniform
            const bool in = 64 * c + 4 * sub < a.E, before = ahead[c] < a.kept;
            const bool keep = in && before && rank[c] > none;
            if constexpr (ASK) {
                worst = fminf(worst, in && before ? O::value(rank[c]) - off[c] : INFINITY);
                next = fmaxf(next, in && !before ? O::value(rank[c]) + off[c] : -INFINITY);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) key[c][j] = keep ? key[c][j] : none;
        }
        if constexpr (ASK) close = row_min(worst) < row_max(next) ? 2 : 0;
    } else if (a.groups > 1) {
        I rank = none;                                     // of group `sub`
        float off = 0.f;
        int gid[EC][4];
#pragma unroll
        for (int c = 0; c < EC; ++c)
#pragma unroll
            for (int j = 0; j < 4; ++j) gid[c][j] = group_of(a, 64 * c + 4 * sub + j);
        for (int g = 0; g < a.groups; ++g) {
            I m1 = none, m2 = none;                        // the two largest keys of the group
#pragma unroll
            for (int c = 0; c < EC; ++c)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const I v = gid[c][j] == g ? key[c][j] : none;
                    m2 = larger(m2, smaller(m1, v));
                    m1 = larger(m1, v);
                }
            auto merge = [&](I o1, I o2) {
                m2 = larger(smaller(m1, o1), larger(m2, o2));
                m1 = larger(m1, o1);
            };
            merge(dpp<0x128>(m1), dpp<0x128>(m2));
            merge(dpp<0x124>(m1), dpp<0x124>(m2));
            merge(dpp<0x122>(m1), dpp<0x122>(m2));
            merge(dpp<0x121>(m1), dpp<0x121>(m2));
            const I r = a.best == 2 && m2 > none ? O::of(larger(O::value(m1) + O::value(m2) + T(err.left_out), last_key(T(0)))) : m1;
            rank = g == sub ? r : rank;
            if constexpr (ASK) off = g == sub ? rank_error(a, O::value(m1), O::value(m2), O::value(r), err) : off;
        }
        unsigned kept = 0;
        I left = rank;
        for (int i = 0; i < a.kept; ++i) {
            const I most = row_max(left);
            const int w = row_min(left == most ? sub : 99);
            if (most > none) kept |= 1u << (w & 31);
            left = w == sub ? none : left;
        }
        if constexpr (ASK) {
            const bool mine = kept >> sub & 1u;
            close = row_min(mine ? O::value(rank) - off : INFINITY) < row_max(mine ? -INFINITY : O::value(rank) + off) ? 2 : 0;
        }
#pragma unroll
        for (int c = 0; c < EC; ++c)
#pragma unroll
            for (int j = 0; j < 4; ++j) key[c][j] = (kept >> (gid[c][j] & 31)) & 1u ? key[c][j] : none;
    }
    return close;
}

// The best experts by key of one token, in its 16 lanes, of R lists of keys at once (one's steps fill the other's waits): lane `sub` is left with
// choice number `sub` of each in `mine` (-1: none).  Returns whether two that follow each other may lie the other way round (fp32 keys).
template <class T, int EC, int R>
__device__ __forceinline__ int pick_row(typename key_order<T>::type (&key)[R][EC][4], const smoe_topk_args& a, int sub, key_error err, int (&mine)[R]) {
    constexpr bool ASK = std::is_same<T, float>::value;
    using O = key_order<T>;
    using I = typename O::type;
    const I none = O::of(-INFINITY);
    int close = 0;
    float last[R], reach[R];                               // the choice before, and both errors where the next is near it
#pragma unroll
    for (int r = 0; r < R; ++r) {
        mine[r] = -1;
        last[r] = INFINITY;
        reach[r] = 0.f;
    }
#pragma unroll 1
    for (int i = 0; i <= a.k; ++i) {                       // one round more than choices: the distance to the next best
        I m[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            m[r] = none;
#pragma unroll
            for (int c = 0; c < EC; ++c)
#pragma unroll
                for (int j = 0; j < 4; ++j) m[r] = larger(m[r], key[r][c][j]);
        }
        row_max(m);
        if constexpr (ASK)
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const float v = O::value(m[r]);
                close |= last[r] - v < reach[r] ? 1 : 0;   // (keys without errors: equal ones are a tie; from none to none: NaN)
                last[r] = v;
                reach[r] = 2.f * fmaf(err.rel, fabsf(v), err.base);
            }
        int at[R], e[R];                                   // the lane's first expert with that key; the row's first loses it
#pragma unroll
        for (int r = 0; r < R; ++r) {
            at[r] = INT_MAX;
#pragma unroll
            for (int c = EC - 1; c >= 0; --c)
#pragma unroll
                for (int j = 3; j >= 0; --j) at[r] = key[r][c][j] == m[r] ? 64 * c + j : at[r];
            e[r] = at[r] == INT_MAX ? at[r] : at[r] + 4 * sub;
        }
        int own[R];
#pragma unroll
        for (int r = 0; r < R; ++r) own[r] = e[r];
        row_min(e);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            mine[r] = m[r] > none && i == sub && i < a.k ? e[r] : mine[r];
            int gone = own[r] == e[r] ? at[r] : -1;
            asm("" : "+v"(gone));                          // one comparison a key below, not two and their conjunction
#pragma unroll
            for (int c = 0; c < EC; ++c)
#pragma unroll
                for (int j = 0; j < 4; ++j) key[r][c][j] = gone == 64 * c + j ? none : key[r][c][j];
        }
    }
    return close;
}

__device__ __forceinline__ float exp_of(float v) { return expf(v); }
__device__ __forceinline__ double exp_of(double v) { return exp(v); }

// What lane `sub` has chosen: weight and identity, among the resident experts with `served`, else among all.  score_at, logit_at: an expert's score and
// logit.  store: write the results to id and gate.
// Weights that are divided by their sum are taken in units of e^m, m the largest exponent among the chosen, which cancels: e^(l - m) for a softmax,
// e^(min(l, 0) - m) / (1 + e^-|l|) for a sigmoid.  The scores themselves may all be zero: those of residents more than 104 below the best of all experts are in
// fp32.
template <class T, class SCORE, class LOGIT>
__device__ __forceinline__ void store_choice(const smoe_topk_args& a, int mine, SCORE score_at, LOGIT logit_at, int sub, int tok, bool served, int32_t* id,
                                             float* gate, bool store) {
    const int e = min(max(mine, 0), a.E - 1);
    T w = 0;
    if (a.renorm) {
        const T l = mine >= 0 ? T(logit_at(e)) : T(-INFINITY), p = a.sigmoid ? smaller(l, T(0)) : l;
        const T m = row_max(p);
        if (mine >= 0) {
            w = exp_of(p - m);
            if (a.sigmoid) w /= 1 + exp_of(l < 0 ? l : -l);
        }
        const T sum = row_sum(w);                          // at least 1/2
        if (mine >= 0) w /= sum;
    } else if (mine >= 0) {
        w = score_at(e);
    }
    if (sub < a.k && store) {
        const size_t at = (size_t)tok * a.k + sub;
        id[at] = mine < 0 ? -1 : served ? a.e2s[e] : e;
        gate[at] = (float)(w * a.scale);
    }
}

// One token again in 64 bits, by one wave.  Only logits whose order is in question are computed again: those of experts whose keys are within
// the tolerance of another's, and those that rank a group near another where the groups are in question (`groups`).
// The others keep their fp32 logits, which are apart from whatever they are compared with.  Few tokens come here, and a workgroup that has one is
// the last to end, so what counts is the time of one pass: 27000 cycles with two logits to repeat (16384 tokens, 8 of 128 experts: 11 of 53 us), of
// which 1500 for the keys, 500 for the groups, 5300 for the distances, 3900 for the products and 14000 for the selection, whose code comes from memory
// for the first time.  Loads go together, 4 or 8 at a time (one at a time: 36000 cycles), but loops are not unrolled further.
template <int EC>
struct alignas(16) topk_exact {
    static constexpr int N = 64 * EC, WAVES = EC == 4 ? 6 : 8;   // waves that work on such tokens: what fits the LDS beside the logits
    double logit[N], score[N];                             // score: first the fp32 keys of all experts and of the resident ones
};

// Both selections of token tok by one wave from its logits in s.logit.
template <int EC>
__device__ __forceinline__ void select_exact(const smoe_topk_args& a, int tok, topk_exact<EC>& s) {
    const int lane = threadIdx.x & 63, sub = lane & 15;
    double top = 0, z = 0;                                 // scores: the largest logit, then the sum of the exponentials
    if (!a.sigmoid) {
        top = -INFINITY;
#pragma unroll 1
        for (int e = lane; e < a.E; e += 64) top = fmax(top, s.logit[e]);
#pragma unroll 1
        for (int o = 1; o < 64; o <<= 1) top = fmax(top, __shfl_xor(top, o));
    }
#pragma unroll 1
    for (int e = lane; e < 64 * EC; e += 64) {
        const double p = e >= a.E ? 0.0 : exp(a.sigmoid ? -s.logit[e] : s.logit[e] - top);
        s.score[e] = a.sigmoid ? 1.0 / (1.0 + p) : p;
        z += p;
    }
    if (!a.sigmoid) {
#pragma unroll 1
        for (int o = 1; o < 64; o <<= 1) z += __shfl_xor(z, o);
    }
    const double inv_z = a.sigmoid ? 1.0 : 1.0 / z;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    double key[1][EC][4];
    int sl[EC][4];
#pragma unroll
    for (int c = 0; c < EC; ++c)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int e = 64 * c + 4 * sub + j, ei = min(e, a.E - 1);
            key[0][c][j] = a.by_logit ? s.logit[ei] : s.score[ei] * inv_z + (a.bias ? (double)a.bias[ei] : 0.0);
            key[0][c][j] = e < a.E ? number_or_last(key[0][c][j]) : -INFINITY;
            sl[c][j] = e < a.E ? a.e2s[ei] : -1;
        }
    // the first 16 lanes select among all experts, the next 16 among the resident ones
    const bool served = lane & 16;
#pragma unroll
    for (int c = 0; c < EC; ++c)
#pragma unroll
        for (int j = 0; j < 4; ++j) key[0][c][j] = served && sl[c][j] < 0 ? -INFINITY : key[0][c][j];
    int mine[1];
    keep_groups<double, EC>(key[0], a, sub, key_error{});
    pick_row<double, EC, 1>(key, a, sub, key_error{}, mine);
    store_choice<double>(a, mine[0], [&](int e) { return s.score[e] * inv_z; }, [&](int e) { return s.logit[e]; }, sub, tok, served,
                         served ? a.slot : a.orig_expert, served ? a.gate : a.orig_gate, lane < 32);
}

// Whether another lane of the row holds a value that may be equal, each being off by at most `off`.
template <int N = 1>
__device__ __forceinline__ bool near_in_row(float v, float off) {
    bool near = fabsf(v - dpp<0x120 + N>(v)) <= off + dpp<0x120 + N>(off);
    if constexpr (N < 15) near |= near_in_row<N + 1>(v, off);
    return near;
}

template <int EC, class AT>
__device__ __forceinline__ void choose_exact(const smoe_topk_args& a, int tok, AT logit_at, float err, bool groups, topk_exact<EC>& s) {
    const int lane = threadIdx.x & 63, per = a.E / a.groups;
    float* fkey = (float*)s.score;
    float* rkey = fkey + 64 * EC;
#pragma unroll 1
    for (int e = lane; e < 64 * EC; e += 64) {
        const float l = e < a.E ? logit_at(e) : -INFINITY;
        const float key = a.by_logit || e >= a.E ? l : sigmoid_of(l) + (a.bias ? a.bias[e] : 0.f);
        s.logit[e] = l;
        fkey[e] = key;
        rkey[e] = e < a.E && a.e2s[e] >= 0 ? key : -INFINITY;
    }
    const key_error off = {a.by_logit ? err : 0.25f * err + 8 * HALF_STEP, a.by_logit ? 0.f : HALF_STEP, 0.f};
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); // lanes of a wave read what others wrote: its LDS accesses are in order
    // Groups whose rank is near another's, and the least key of those that make a group's rank (lane g: group g).
    bool near_group[2] = {false, false};
    float made_of[2];
    if (groups) {
#pragma unroll
        for (int res = 0; res < 2; ++res) {
            float m1 = -INFINITY, m2 = -INFINITY;
            const float* keys = res ? rkey : fkey;
#pragma unroll 1
            for (int f = 0; f < per; f += 4) {
                float v[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] = keys[min(min(lane, a.groups - 1) * per + f + i, a.E - 1)];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float u = lane < a.groups && f + i < per ? v[i] : -INFINITY;
                    m2 = fmaxf(m2, fminf(m1, u));
                    m1 = fmaxf(m1, u);
                }
            }
            made_of[res] = a.best == 2 ? m2 : m1;
            const float rank = a.best == 2 && m2 > -INFINITY ? fmaxf(m1 + m2, -FLT_MAX) : m1;
            near_group[res] = near_in_row(rank, rank_error(a, m1, m2, rank, off));   // (lanes behind the groups are infinitely far)
        }
    }
    unsigned again_of = 0;                                 // bit c: this lane's expert of chunk c
    float mine[EC], tol[EC];
    int near[EC];
#pragma unroll
    for (int c = 0; c < EC; ++c) {
        mine[c] = fkey[64 * c + lane];
        tol[c] = mine[c] > -INFINITY ? 2.f * fmaf(off.rel, fabsf(mine[c]), off.base) : 0.f;
        near[c] = 0;
    }
#pragma unroll 1
    for (int f = 0; f < a.E; f += 8) {                 // itself among them; past E: infinitely far
        const float4 lo = *(const float4*)(fkey + f), hi = *(const float4*)(fkey + f + 4);
        const float o[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int c = 0; c < EC; ++c) near[c] += fabsf(mine[c] - o[i]) <= tol[c];
    }
#pragma unroll
    for (int c = 0; c < EC; ++c) {
        const int e = 64 * c + lane, g = min(group_of(a, e), a.groups - 1);
        bool again = near[c] > 1;
        if (groups) {
            const bool in_all = __shfl((int)near_group[0], g), in_res = __shfl((int)near_group[1], g);
            const float least = __shfl(made_of[0], g), least_res = __shfl(made_of[1], g);
            again |= (in_all && mine[c] >= least) || (in_res && rkey[e] == mine[c] && mine[c] >= least_res);
        }
        again_of |= (again && e < a.E && mine[c] > -INFINITY ? 1u : 0u) << c;   // (what cannot be had is not asked for)
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    int* list = (int*)fkey;                                // the keys have been used up
    int n = 0;
#pragma unroll 1
    for (int c = 0; c < EC; ++c) {
        const bool again = again_of >> c & 1u;
        const unsigned long long m = __ballot(again);
        if (again) list[n + __popcll(m & ((1ull << lane) - 1ull))] = 64 * c + lane;
        n += __popcll(m);
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    // two experts at a time, 32 lanes each, four pieces of a row on their way together
#pragma unroll 1
    for (int i = lane >> 5; i < n + (lane >> 5); i += 2) {
        const int e = list[min(i, n - 1)];
        // the expert's row: the caller's, or out of the operand order that the product has just read (there it is in the L2), a
        // unit of 4 weights at a time: step c / 16, half c % 8 / 4, lane e % 32 + 32 (c % 16 / 8)
        const float4* w = a.f32 ? (const float4*)(a.wrow + (size_t)e * a.d) : (const float4*)a.wr + (size_t)(e >> 5) * (a.d >> 4) * 128 + (e & 31);
        double sum = 0;
#pragma unroll 1
        for (int c0 = (lane & 31) * 4; c0 < a.d; c0 += 512) {     // d_model is a multiple of 4
            float4 v[4], x[4];
            if (a.f32) {
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const int c = min(c0 + 128 * u, a.d - 4);
                    v[u] = w[c >> 2];
                    x[u] = *(const float4*)((const float*)a.x + (size_t)tok * a.d + c);
                }
            } else {
                uint2 p[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const int c = min(c0 + 128 * u, a.d - 4);
                    v[u] = w[(c >> 4) * 128 + (c >> 2 & 1) * 64 + (c >> 3 & 1) * 32];
                    p[u] = *(const uint2*)((const uint16_t*)a.x + (size_t)tok * a.d + c);
                }
#pragma unroll
                for (int u = 0; u < 4; ++u)
                    x[u] = make_float4(__uint_as_float(p[u].x << 16), __uint_as_float(p[u].x & 0xFFFF0000u), __uint_as_float(p[u].y << 16),
                                       __uint_as_float(p[u].y & 0xFFFF0000u));
            }
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                if (c0 + 128 * u >= a.d) v[u] = make_float4(0, 0, 0, 0);   // past the row
                sum = fma((double)x[u].x, (double)v[u].x, sum);
                sum = fma((double)x[u].y, (double)v[u].y, sum);
                sum = fma((double)x[u].z, (double)v[u].z, sum);
                sum = fma((double)x[u].w, (double)v[u].w, sum);
            }
        }
        sum = row_sum(sum);
        sum += __shfl_xor(sum, 16);
        if ((lane & 31) == 0) s.logit[e] = sum;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    select_exact<EC>(a, tok, s);
}

__device__ __forceinline__ float4 load_x4(const smoe_topk_args& a, size_t at) {
    if (a.f32) return *(const float4*)((const float*)a.x + at);
    const uint2 p = *(const uint2*)((const uint16_t*)a.x + at);
    return make_float4(__uint_as_float(p.x << 16), __uint_as_float(p.x & 0xFFFF0000u), __uint_as_float(p.y << 16), __uint_as_float(p.y & 0xFFFF0000u));
}

// Whether token tok's row of x is all zeros, by its 16 lanes.
__device__ __forceinline__ bool zero_row(const smoe_topk_args& a, int tok, int sub) {
    const uint4* row = (const uint4*)((const char*)a.x + (size_t)tok * a.d * (a.f32 ? 4 : 2));
    const uint32_t bits = a.f32 ? 0x7fffffffu : 0x7fff7fffu;   // -0 is a zero
    uint32_t any = 0;
    for (int c = sub; c < (a.f32 ? a.d >> 2 : a.d >> 3); c += 16) {
        const uint4 v = row[c];
        any |= (v.x | v.y | v.z | v.w) & bits;
    }
    return row_max(any ? 1 : 0) == 0;
}

// Where a bias meets the softmax every key holds the sum over all experts, and all logits are computed again: lane l's are those of the experts
// 64 c + l, over the columns 4 q0 .. 4 q1 - 1.
template <int EC>
__device__ __forceinline__ void all_logits(const smoe_topk_args& a, int tok, int q0, int q1, double (&sum)[EC]) {
    const int lane = threadIdx.x & 63;
    const float4* w[EC];
#pragma unroll
    for (int c = 0; c < EC; ++c) {
        const int e = min(64 * c + lane, a.E - 1);
        w[c] = a.f32 ? (const float4*)(a.wrow + (size_t)e * a.d) : (const float4*)a.wr + (size_t)(e >> 5) * (a.d >> 4) * 128 + (e & 31);
        sum[c] = 0;
    }
    constexpr int U = 4;                                   // on their way together
#pragma unroll 1
    for (int q = q0; q < q1; q += U) {
        float4 v[EC][U], x[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int qq = min(q + u, q1 - 1), at = a.f32 ? qq : (qq >> 2) * 128 + (qq & 1) * 64 + (qq >> 1 & 1) * 32;
            x[u] = load_x4(a, (size_t)tok * a.d + 4 * qq);
#pragma unroll
            for (int c = 0; c < EC; ++c) v[c][u] = w[c][at];
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (q + u >= q1) x[u] = make_float4(0, 0, 0, 0);   // past the columns
            const double x0 = x[u].x, x1 = x[u].y, x2 = x[u].z, x3 = x[u].w;
#pragma unroll
            for (int c = 0; c < EC; ++c) {
                sum[c] = fma(x0, (double)v[c][u].x, sum[c]);
                sum[c] = fma(x1, (double)v[c][u].y, sum[c]);
                sum[c] = fma(x2, (double)v[c][u].z, sum[c]);
                sum[c] = fma(x3, (double)v[c][u].w, sum[c]);
            }
        }
    }
}

}  // namespace

// What follows the product (found by the bodies of route_mfma.h through the type of the arguments).
template <int NEB, int TB>
__device__ __forceinline__ void smoe_route_finish(const int block, const smoe_topk_args& a,
                                                  smoe_f32x16 (&acc)[smoe_route_shape<NEB, TB>::NEBH][TB], float (&sq)[TB], float* smem) {
    using S = smoe_route_shape<NEB, TB>;
    constexpr int NS = S::NS, LDP = S::LDP, NTOK = S::NTOK, EC = smoe_route_chunks(NEB), EP = NEB * 32;
    float* part = smem;                                    // [NS][NTOK][LDP] partial logits
    float* sqp = smem + NS * NTOK * LDP;                   // [NS][2 halves][NTOK] partial sums of squares
    __shared__ int32_t s_n, s_close[NTOK];                 // tokens of the block to be repeated in 64 bits; bit 8: the groups too
    __shared__ float s_err[NTOK];
    using X = topk_exact<EC>;
    __shared__ X s_exact[X::WAVES];
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, sub = lane & 15;
    const int tw0 = block * NTOK;
    if (tid == 0) s_n = 0;
    int sl[EC][4];
    smoe_route_slots<NEB>(sl, a, sub);
    float bias[EC][4];
#pragma unroll
    for (int c = 0; c < EC; ++c)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int e = 64 * c + 4 * sub + j;
            bias[c][j] = a.bias && e < a.E ? a.bias[e] : 0.f;
        }
    const float wnorm = *a.wnorm;
    smoe_route_meet<NEB, TB>(a.E, acc, sq, part, sqp);

#pragma unroll 1
    for (int tb = 0; tb < TB; ++tb) {
        const int t = tb * SMOE_RT + wave * 4 + (lane >> 4), tok = tw0 + t;
        const float* row = part + t * LDP;
        float v[EC][4], big = 0.f;
#pragma unroll
        for (int c = 0; c < EC; ++c) {
            const float* col = row + min(64 * c + 4 * sub, EP - 4);
            float s[4] = {0.f, 0.f, 0.f, 0.f}, m[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int q = 0; q < NS; ++q) {                 // fixed order of the slices
                const float4 o = *(const float4*)(col + q * NTOK * LDP);
                const float p[4] = {o.x, o.y, o.z, o.w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    s[j] = q ? s[j] + p[j] : p[j];
                    m[j] += fabsf(p[j]);
                }
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const bool in = 64 * c + 4 * sub + j < a.E;
                v[c][j] = in ? s[j] : -INFINITY;
                big = fmaxf(big, in ? m[j] : 0.f);
            }
        }
        float ss = 0.f;
#pragma unroll
        for (int q = 0; q < 2 * NS; ++q) ss += sqp[t + q * NTOK];
        const float xnorm = sqrtf(ss);
        big = __int_as_float(row_max(__float_as_int(big)));
        float err = HALF_STEP * (a.err_norm * xnorm * wnorm + a.err_sum * big);
        // A row of zeros, as padding has them: its logits are zeros and its scores equal, both exactly, so its keys are the biases, without an error.  (16384
        // tokens, half of them zeros, 8 of 128 experts in groups: 51 us; with all their choices counted as close, and repeated in 64 bits, 1210.)
        const bool faint = ss < 0x1p-100f;
        bool zeros = false;
        if (__any(faint)) {
            int numbers = 1;
#pragma unroll
            for (int c = 0; c < EC; ++c)
#pragma unroll
                for (int j = 0; j < 4; ++j) numbers &= v[c][j] == v[c][j];
            zeros = zero_row(a, min(tok, a.T - 1), sub) && row_min(numbers);
            if (faint && !zeros) err = INFINITY;           // squares that underflow say nothing about the error: all in 64 bits
        }
        float top = -INFINITY, z = 1.f;
#pragma unroll
        for (int c = 0; c < EC; ++c)
#pragma unroll
            for (int j = 0; j < 4; ++j) top = fmaxf(top, v[c][j]);
        top = smoe_row_max(top);
        if (!a.sigmoid) {
            z = 0.f;
#pragma unroll
            for (int c = 0; c < EC; ++c)
#pragma unroll
                for (int j = 0; j < 4; ++j) z += expf(v[c][j] - top);
            z = smoe_row_sum(z);
        }
        const float inv_z = 1.f / z;
        auto logit_at = [&](int e) {
            float s = row[e];
#pragma unroll
            for (int q = 1; q < NS; ++q) s += row[q * NTOK * LDP + e];
            return s;
        };
        auto score_at = [&](int e) {
            const float l = logit_at(e);
            return a.sigmoid ? sigmoid_of(l) : expf(l - top) * inv_z;
        };
        key_error off = {err, 0.f, 0.f};
        if (!a.by_logit) {
            float most = 0.f;                              // largest score
#pragma unroll
            for (int c = 0; c < EC; ++c)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const bool in = 64 * c + 4 * sub + j < a.E;
                    const float s = a.sigmoid ? sigmoid_near(v[c][j]) : expf(v[c][j] - top) * inv_z;
                    v[c][j] = in ? s + bias[c][j] : -INFINITY;
                    most = fmaxf(most, in ? s : 0.f);
                }
            // a sigmoid is off by at most a quarter of its logit's error, a share of a softmax by at most twice its own size times that; and the
            // exponential and the quotient are rounded: units of 2^-24, 8 of them, and of the fast sigmoid s another
            // 1.5 (1 - s) |l|, where s (1 - s) |l| <= (|largest l| + 1/2) (largest s); and the sum with the bias, half a step of its own
            const float units = a.sigmoid ? 8.f + 2.f * fabsf(top) : 8.f;
            off.base = (a.sigmoid ? 0.25f : 2.f * inv_z) * err + HALF_STEP * units * __int_as_float(row_max(__float_as_int(most)));
            off.rel = HALF_STEP;
        }
        if (zeros) {
            off = {0.f, a.best == 2 ? HALF_STEP : 0.f, a.sigmoid ? 0.5f : inv_z};   // (the second for sums of two)
#pragma unroll
            for (int c = 0; c < EC; ++c)
#pragma unroll
                for (int j = 0; j < 4; ++j) v[c][j] = 64 * c + 4 * sub + j < a.E ? bias[c][j] + 0.f : -INFINITY;   // (-0 is no less than 0)
        }
#pragma unroll
        for (int c = 0; c < EC; ++c)
#pragma unroll
            for (int j = 0; j < 4; ++j) v[c][j] = number_or_last(v[c][j]);
        // both selections at once, or one after the other where the registers do not reach
        constexpr int R = EC <= 2 ? 2 : 1;
        int close = 0;
#pragma unroll 1
        for (int first = 0; first < 2; first += R) {
            int key[R][EC][4], mine[R];
#pragma unroll
            for (int r = 0; r < R; ++r) {
#pragma unroll
                for (int c = 0; c < EC; ++c)
#pragma unroll
                    for (int j = 0; j < 4; ++j) key[r][c][j] = to_ordered(first + r && sl[c][j] < 0 ? -INFINITY : v[c][j]);
                if (a.groups > 1) close |= keep_groups<float, EC>(key[r], a, sub, off);
            }
            close |= pick_row<float, EC, R>(key, a, sub, zeros ? key_error{} : off, mine);
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const bool served = first + r;
                store_choice<float>(a, mine[r], score_at, logit_at, sub, tok, served, served ? a.slot : a.orig_expert, served ? a.gate : a.orig_gate,
                                    tok < a.T);
            }
        }
        if (sub < a.k && tok < a.T) a.xnorm[(size_t)tok * a.k + sub] = xnorm;
        if (close && sub == 0 && tok < a.T) {
            const int i = atomicAdd(&s_n, 1);              // the order does not matter
            s_close[i] = t | (close & 2 ? 1 << 8 : 0);
            s_err[i] = err;
        }
    }
    __syncthreads();
    const int n = s_n;
    if (!a.sigmoid && !a.by_logit) {
        const int quads = a.d >> 2;
        double sum[EC];
        constexpr int W = X::WAVES;
        if (n <= 6) {
            // (uniform) The whole workgroup on one token after the other, a share of the columns each; then the selections, a wave each.  16384 tokens,
            // 8 of 128 experts with some workgroups of several such tokens: 88 us with this for at most 2 tokens, 70 for 6.
            const int share = (quads + W - 1) / W;
            for (int i = 0; i < n; ++i) {
                const int tok = tw0 + (__builtin_amdgcn_readfirstlane(s_close[i]) & 255);
                if (wave < W) {
                    all_logits<EC>(a, tok, min(wave * share, quads), min((wave + 1) * share, quads), sum);
#pragma unroll
                    for (int c = 0; c < EC; ++c) s_exact[wave].logit[64 * c + lane] = sum[c];
                }
                __syncthreads();
                if (wave == i)
#pragma unroll
                    for (int c = 0; c < EC; ++c) {
                        sum[c] = 0;
                        for (int w = 0; w < W; ++w) sum[c] += s_exact[w].logit[64 * c + lane];   // fixed order
                        s_exact[wave].score[64 * c + lane] = sum[c];
                    }
                __syncthreads();
            }
            if (wave >= n) return;
#pragma unroll
            for (int c = 0; c < EC; ++c) s_exact[wave].logit[64 * c + lane] = s_exact[wave].score[64 * c + lane];
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            select_exact<EC>(a, tw0 + (__builtin_amdgcn_readfirstlane(s_close[wave]) & 255), s_exact[wave]);
            return;
        }
        if (wave >= X::WAVES) return;
        for (int i = wave; i < n; i += X::WAVES) {         // a wave each
            const int tok = tw0 + (__builtin_amdgcn_readfirstlane(s_close[i]) & 255);
            all_logits<EC>(a, tok, 0, quads, sum);
#pragma unroll
            for (int c = 0; c < EC; ++c) s_exact[wave].logit[64 * c + lane] = sum[c];
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            select_exact<EC>(a, tok, s_exact[wave]);
        }
        return;
    }
    if (wave >= X::WAVES) return;
    for (int i = wave; i < n; i += X::WAVES) {             // a wave each
        const int word = __builtin_amdgcn_readfirstlane(s_close[i]), t = word & 255;
        const float* row = part + t * LDP;
        auto logit_at = [&](int e) {
            float s = row[e];
#pragma unroll
            for (int q = 1; q < NS; ++q) s += row[q * NTOK * LDP + e];
            return s;
        };
        choose_exact<EC>(a, tw0 + t, logit_at, s_err[i], word >> 8, s_exact[wave]);
    }
}

namespace {

template <int NEB, int TB, bool MULTI>
__global__ __launch_bounds__(512) void topk_mfma_kernel(const smoe_topk_args a) {
    extern __shared__ __align__(16) float smem[];
    smoe_route_mfma_body<NEB, TB, MULTI>(blockIdx.x, a, smem);
}

template <int NEB>
__global__ __launch_bounds__(512) void topk_f32_kernel(const smoe_topk_args a) {
    extern __shared__ __align__(16) float smem[];
    smoe_route_f32_body<NEB>(blockIdx.x, a, smem);
}

// Instances and their choice as in route.hip.
template <int NEB, int TB, bool MULTI>
int launch_multi(const smoe_topk_args& a, hipStream_t s) {
    using S = smoe_route_shape<NEB, TB>;
    static smoe_lds_raised raised;
    if (int rc = raised.ensure((const void*)topk_mfma_kernel<NEB, TB, MULTI>, S::lds_bytes(a.d), (int)S::lds_bytes(SMOE_ROUTE_KC))) return rc;
    constexpr int NTOK = SMOE_RT * TB;
    hipLaunchKernelGGL((topk_mfma_kernel<NEB, TB, MULTI>), dim3((a.T + NTOK - 1) / NTOK), dim3(512), S::lds_bytes(a.d), s, a);
    return smoe_check_hip(hipGetLastError(), "smoe_route_topk launch");
}

template <int NEB>
int launch(const smoe_topk_args& a, hipStream_t s) {
    if (a.f32) {
        const size_t lds = smoe_route_shape<NEB, 1>::lds_bytes(0);
        static smoe_lds_raised raised;
        if (int rc = raised.ensure((const void*)topk_f32_kernel<NEB>, lds, (int)lds)) return rc;
        hipLaunchKernelGGL(topk_f32_kernel<NEB>, dim3((a.T + SMOE_RT - 1) / SMOE_RT), dim3(512), lds, s, a);
        return smoe_check_hip(hipGetLastError(), "smoe_route_topk launch");
    }
    if constexpr (NEB <= 4) {
        if ((a.T + SMOE_RT - 1) / SMOE_RT > 256) {
            if constexpr (NEB <= 2) {
                if (a.d > SMOE_ROUTE_KC) return launch_multi<NEB, 2, true>(a, s);
            }
            return launch_multi<NEB, 2, false>(a, s);
        }
    }
    return launch_multi<NEB, 1, false>(a, s);
}

// Few tokens: a workgroup of the kernels above would read the whole router alone.  Here a wave takes the product of one expert with FEW_TOK tokens, in
// 64 bits (so that nothing has to be repeated), and a second launch selects, a wave a token.
constexpr int FEW_TOK = 4;

__global__ __launch_bounds__(256) void topk_logits_kernel(const smoe_topk_args a) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int e = blockIdx.x * 4 + wave, t0 = blockIdx.y * FEW_TOK;
    if (e >= a.E) return;
    double sum[FEW_TOK] = {};
#pragma unroll 2
    for (int c = lane * 4; c < a.d; c += 256) {            // d_model is a multiple of 4
        const float4 w = *(const float4*)(a.wrow + (size_t)e * a.d + c);
        const double w0 = w.x, w1 = w.y, w2 = w.z, w3 = w.w;
#pragma unroll
        for (int i = 0; i < FEW_TOK; ++i) {                // past the batch: the last token again, not written
            const float4 x = load_x4(a, (size_t)min(t0 + i, a.T - 1) * a.d + c);
            sum[i] = fma((double)x.x, w0, sum[i]);
            sum[i] = fma((double)x.y, w1, sum[i]);
            sum[i] = fma((double)x.z, w2, sum[i]);
            sum[i] = fma((double)x.w, w3, sum[i]);
        }
    }
#pragma unroll
    for (int i = 0; i < FEW_TOK; ++i) {
        double v = row_sum(sum[i]);
        v += __shfl_xor(v, 16);
        v += __shfl_xor(v, 32);
        if (lane == 0 && t0 + i < a.T) a.logits[(size_t)(t0 + i) * a.E + e] = v;
    }
}

template <int EC>
__global__ __launch_bounds__(64) void topk_select_kernel(const smoe_topk_args a) {
    __shared__ topk_exact<EC> s;
    const int lane = threadIdx.x, tok = blockIdx.x;
    for (int e = lane; e < 64 * EC; e += 64) s.logit[e] = e < a.E ? a.logits[(size_t)tok * a.E + e] : -INFINITY;
    float ss = 0.f;
    for (int c = lane * 4; c < a.d; c += 256) {
        const float4 x = load_x4(a, (size_t)tok * a.d + c);
        ss = fmaf(x.x, x.x, ss); ss = fmaf(x.y, x.y, ss); ss = fmaf(x.z, x.z, ss); ss = fmaf(x.w, x.w, ss);
    }
    ss = smoe_row_sum(ss);
    ss += __shfl_xor(ss, 16);
    ss += __shfl_xor(ss, 32);
    if (lane < a.k) a.xnorm[(size_t)tok * a.k + lane] = sqrtf(ss);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    select_exact<EC>(a, tok, s);
}

// Largest norm of the router's rows: a wave per row in turn, one workgroup (once per bind).
__global__ __launch_bounds__(1024) void router_norm_kernel(const float* __restrict__ w, int E, int d, float* __restrict__ out) {
    __shared__ float s_max[16];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    float big = 0.f;
    for (int e = wave; e < E; e += 16) {
        float ss = 0.f;
        for (int c = lane; c < d; c += 64) ss = fmaf(w[(size_t)e * d + c], w[(size_t)e * d + c], ss);
        for (int o = 32; o > 0; o >>= 1) ss += __shfl_xor(ss, o);
        big = fmaxf(big, ss);
    }
    if (lane == 0) s_max[wave] = big;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int i = 1; i < 16; ++i) big = fmaxf(big, s_max[i]);
        out[0] = sqrtf(big);
    }
}

// Whether T tokens take the launches for few tokens: where one workgroup's walk through the router takes longer than a second launch.  bf16 from
// 256 KB of router on, fp32 always (its matrix products are slow).  Measured with 2 choices (us, one launch / two): bf16, 64 experts of 768 columns,
// 1 token 8.9 / 9.0, 128 tokens 9.9 / 10.3; 64 of 1024 10.1 / 9.4 and 11.1 / 11.0; 128 of 512 11.4 / 9.6 and 12.5 / 11.6; 128 of 1024 14.7 / 10.9 and
// 15.9 / 13.7 (256 tokens: 16.0 / 17.4); 256 of 2048 40 / 16 and 42 / 28; fp32, 64 of 768 14.7 / 8.3 and 18.2 / 9.4, 512 tokens
// 18.5 / 13.3, 1024 18.5 / 18.2; 16 of 512 at 512 tokens 10.6 / 9.1, 128 of 1024 32 / 22, at 1024 32 to 39 / 35.
bool topk_few(const smoe_config& c, int T) { return T <= smoe_topk_few_tokens(c.dtype) && (c.dtype == SMOE_F32 || c.E * c.d_model >= 65536); }

}  // namespace

int smoe_launch_router_norm(const smoe_layer* L, hipStream_t s) {
    hipLaunchKernelGGL(router_norm_kernel, dim3(1), dim3(1024), 0, s, L->router_w, L->cfg.E, L->cfg.d_model, L->d_router_norm);
    return smoe_check_hip(hipGetLastError(), "smoe_route_topk: router norm launch");
}

int smoe_launch_route_topk(const smoe_layer* L, const smoe_topk_rule& rule, const float* bias, const void* x, int T, int32_t* orig_expert,
                           float* orig_gate, int32_t* slot, float* gate, float* xnorm, hipStream_t s) {
    const smoe_config& c = L->cfg;
    smoe_topk_args a{};
    a.x = x;
    a.wr = (const uint4*)L->d_router_split;
    a.wrow = L->router_w;
    a.e2s = L->d_expert_to_slot;
    a.T = T; a.d = c.d_model; a.E = c.E; a.K = c.K;
    a.orig_expert = orig_expert; a.orig_gate = orig_gate; a.slot = slot; a.gate = gate; a.xnorm = xnorm;
    a.bias = bias;
    a.wnorm = L->d_router_norm;
    a.k = rule.k; a.sigmoid = rule.score == SMOE_SCORE_SIGMOID;
    a.groups = rule.groups; a.kept = rule.groups_kept; a.best = rule.group_best;
    a.renorm = rule.renorm; a.scale = rule.scale;
    a.by_logit = !bias && (rule.groups == 1 || rule.group_best == 1);
    a.f32 = c.dtype == SMOE_F32;
    const int per = c.E / rule.groups;
    a.inv_per = 1.f / per;
    a.aligned = per >= 4 && per <= 64 && !(per & (per - 1));
    // The partial sums of a logit pass through n roundings.  Where x points nowhere in particular they are small, and the error measured at
    // most 1.0 |x| |w| 2^-24 (256 .. 16384 columns, up to 256 experts).  Where x follows a row of the router they grow to the logit's own size (seen in the
    // slices' sums also where these cancel), and it measured up to 1.8 + 0.08 n of it.  Where x follows a row for half of a slice and its negative for the other
    // half, they grow and vanish inside the slice, unseen: 2.3, 3.6 and 9.8 |x| |w| 2^-24 at 1024, 4096 and 16384 columns in bf16 (n = 48, 192, 768), 3.5, 5.6 and
    // 13.6 in fp32 (128, 512, 2048), at most 0.36 sqrt(n).  All kinds of rows measured at most 0.84 of the sum of both terms; it is an
    // estimate, not a bound, which would be n |x| |w| 2^-24.
    const int slices = c.E <= 32 ? 8 : 4;
    const int n = a.f32 ? 4 * (((c.d_model + 7) / 8 + slices - 1) / slices) : 3 * ((c.d_model / 16 + slices - 1) / slices);
    a.err_norm = std::max(1.f, 0.36f * std::sqrt((float)n));
    a.err_sum = 2.f + 0.1f * n;
    if (topk_few(c, T)) {
        a.logits = (double*)L->d_hidden;                   // scratch that the products after it fill
        hipLaunchKernelGGL(topk_logits_kernel, dim3((c.E + 3) / 4, (T + FEW_TOK - 1) / FEW_TOK), dim3(256), 0, s, a);
        if (int rc = smoe_check_hip(hipGetLastError(), "smoe_route_topk: logits launch")) return rc;
        const auto select = c.E <= 64 ? topk_select_kernel<1> : c.E <= 128 ? topk_select_kernel<2> : topk_select_kernel<4>;
        hipLaunchKernelGGL(select, dim3(T), dim3(64), 0, s, a);
        return smoe_check_hip(hipGetLastError(), "smoe_route_topk: selection launch");
    }
    if (c.E <= 32) return launch<1>(a, s);
    if (c.E <= 64) return launch<2>(a, s);
    if (c.E <= 128) return launch<4>(a, s);
    return launch<8>(a, s);
}
