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

#include <climits>

#include "route_mfma.h"

struct smoe_topk_args : smoe_route_args {
    const float* bias;
    const float* wnorm;           // largest |w_e|
    double* logits;               // few tokens: [T, E]
    int k, sigmoid, groups, kept, best, renorm, by_logit, f32;
    int aligned;                  // a group is 4, 8, 16, 32 or 64 experts
    float scale;
    float err_norm, err_sum;      // estimated error of a logit in units of 2^-24: of |x| |w|, and of the sum of its slices' magnitudes
};

namespace {

__device__ __forceinline__ float sigmoid_of(float v) { return 1.0f / (1.0f + expf(-v)); }
__device__ __forceinline__ float larger(float a, float b) { return fmaxf(a, b); }
__device__ __forceinline__ double larger(double a, double b) { return fmax(a, b); }
__device__ __forceinline__ float smaller(float a, float b) { return fminf(a, b); }
__device__ __forceinline__ double smaller(double a, double b) { return fmin(a, b); }

// The rotations and reductions of wave_ops.h in 64 bits.
template <int N>
__device__ __forceinline__ float row_ror(float v) { return smoe_row_ror<N>(v); }
template <int N>
__device__ __forceinline__ double row_ror(double v) {
    return __hiloint2double(smoe_row_ror<N>(__double2hiint(v)), smoe_row_ror<N>(__double2loint(v)));
}
template <int CTRL>
__device__ __forceinline__ float dpp(float v) { return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), CTRL, 0xf, 0xf, true)); }
template <int CTRL>
__device__ __forceinline__ double dpp(double v) {
    return __hiloint2double(__builtin_amdgcn_mov_dpp(__double2hiint(v), CTRL, 0xf, 0xf, true),
                            __builtin_amdgcn_mov_dpp(__double2loint(v), CTRL, 0xf, 0xf, true));
}
template <class T>
__device__ __forceinline__ T row_max(T v) {
    v = larger(v, row_ror<8>(v));
    v = larger(v, row_ror<4>(v));
    v = larger(v, row_ror<2>(v));
    return larger(v, row_ror<1>(v));
}
template <class T>
__device__ __forceinline__ T row_sum(T v) {
    v += row_ror<8>(v);
    v += row_ror<4>(v);
    v += row_ror<2>(v);
    return v + row_ror<1>(v);
}

// The best experts by key of one token, in its 16 lanes: lane `sub` is left with choice number `sub` in `mine` (-1: none).  Returns what was
// decided by a distance of at most tol (twice that between sums of two): 1 the choices, 2 the groups.  gid: group of each of the lane's experts.
template <class T, int EC>
__device__ __forceinline__ int pick_row(T (&key)[EC][4], const int (&gid)[EC][4], const smoe_topk_args& a, int sub, T tol, int& mine) {
    const T none = -INFINITY;
    int close = 0;
    if (a.groups > 1 && a.aligned) {
        // Groups of 4, 8, .. 64 experts: 1, 2, .. 16 neighbouring lanes of one of the lane's packs of four, so each lane finds the rank of its
        // own groups with the steps of one reduction, and counts the groups in front of each (16384 tokens, 8 groups of 16: 18 us
        // less than the walk over the groups below).
        T rank[EC];
        const int lanes = a.E / a.groups >> 2;
#pragma unroll
        for (int c = 0; c < EC; ++c) {
            const T hi0 = larger(key[c][0], key[c][1]), lo0 = smaller(key[c][0], key[c][1]);
            const T hi1 = larger(key[c][2], key[c][3]), lo1 = smaller(key[c][2], key[c][3]);
            T m1 = larger(hi0, hi1), m2 = larger(smaller(hi0, hi1), larger(lo0, lo1));
            auto merge = [&](T o1, T o2) {
                m2 = larger(smaller(m1, o1), larger(m2, o2));
                m1 = larger(m1, o1);
            };
            if (lanes >= 2) merge(dpp<0xB1>(m1), dpp<0xB1>(m2));
            if (lanes >= 4) merge(dpp<0x4E>(m1), dpp<0x4E>(m2));
            if (lanes >= 8) merge(dpp<0x141>(m1), dpp<0x141>(m2));   // the other quad of eight lanes
            if (lanes >= 16) merge(dpp<0x140>(m1), dpp<0x140>(m2));  // the other eight
            rank[c] = a.best == 2 && m2 > none ? m1 + m2 : m1;
        }
        int ahead[EC];
#pragma unroll
        for (int c = 0; c < EC; ++c) ahead[c] = 0;
        for (int s = 0; s < 16; s += lanes) {              // the row turned by s lanes: group (lane - s) / lanes of every pack
            const int at = ((threadIdx.x - s) & 15) | (threadIdx.x & 48);
#pragma unroll
            for (int o = 0; o < EC; ++o) {
                const T v = __shfl(rank[o], at);
#pragma unroll
                for (int c = 0; c < EC; ++c) {
                    const bool before = o < c || (o == c && ((at ^ threadIdx.x) & 15) && (at & 15) < (int)(threadIdx.x & 15));
                    ahead[c] += v > rank[c] || (v == rank[c] && before && (o < c || s)) ? 1 : 0;
                }
            }
        }
        T worst = INFINITY, next = none;
#pragma unroll
        for (int c = 0; c < EC; ++c) {
            if (64 * c >= a.E) continue;                   // uniform
            const bool in = 64 * c + 4 * sub < a.E;
            const bool keep = in && ahead[c] < a.kept && rank[c] > none;
            worst = smaller(worst, in && ahead[c] < a.kept ? rank[c] : T(INFINITY));
            next = larger(next, in && ahead[c] >= a.kept ? rank[c] : none);
#pragma unroll
            for (int j = 0; j < 4; ++j) key[c][j] = keep ? key[c][j] : none;
        }
        close = -row_max(-worst) - row_max(next) <= (a.best == 2 ? 2 * tol : tol) ? 2 : 0;   // (two empty groups: NaN, not close)
    } else if (a.groups > 1) {
        T rank = none;                                     // of group `sub`
        for (int g = 0; g < a.groups; ++g) {
            T m1 = none, m2 = none;                        // the two largest keys of the group
#pragma unroll
            for (int c = 0; c < EC; ++c)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const T v = gid[c][j] == g ? key[c][j] : none;
                    m2 = larger(m2, smaller(m1, v));
                    m1 = larger(m1, v);
                }
            auto merge = [&](T o1, T o2) {
                m2 = larger(smaller(m1, o1), larger(m2, o2));
                m1 = larger(m1, o1);
            };
            merge(row_ror<8>(m1), row_ror<8>(m2));
            merge(row_ror<4>(m1), row_ror<4>(m2));
            merge(row_ror<2>(m1), row_ror<2>(m2));
            merge(row_ror<1>(m1), row_ror<1>(m2));
            const T r = a.best == 2 && m2 > none ? m1 + m2 : m1;
            rank = g == sub ? r : rank;
        }
        unsigned kept = 0;
        T last = INFINITY;
        for (int i = 0; i < a.kept; ++i) {
            last = row_max(rank);
            const int w = smoe_row_min(rank == last ? sub : 99);
            if (last > none) kept |= 1u << (w & 31);
            rank = w == sub ? none : rank;
        }
        close = last - row_max(rank) <= (a.best == 2 ? 2 * tol : tol) ? 2 : 0;
#pragma unroll
        for (int c = 0; c < EC; ++c)
#pragma unroll
            for (int j = 0; j < 4; ++j) key[c][j] = (kept >> (gid[c][j] & 31)) & 1u ? key[c][j] : none;
    }
    mine = -1;
    T last = INFINITY;
    for (int i = 0; i <= a.k; ++i) {                       // one round more than choices: the distance to the next best
        T m = none;
#pragma unroll
        for (int c = 0; c < EC; ++c)
#pragma unroll
            for (int j = 0; j < 4; ++j) m = larger(m, key[c][j]);
        m = row_max(m);
        close |= last - m <= tol ? 1 : 0;
        last = m;
        if (i == a.k) break;                               // uniform
        int e = INT_MAX;
#pragma unroll
        for (int c = EC - 1; c >= 0; --c)
#pragma unroll
            for (int j = 3; j >= 0; --j) e = key[c][j] == m ? 64 * c + 4 * sub + j : e;
        e = smoe_row_min(e);
        mine = m > none && i == sub ? e : mine;
#pragma unroll
        for (int c = 0; c < EC; ++c)
#pragma unroll
            for (int j = 0; j < 4; ++j) key[c][j] = 64 * c + 4 * sub + j == e ? none : key[c][j];
    }
    return close;
}

// A selection of token tok in its 16 lanes: among the resident experts with `served`, else among all.  score_at: an expert's score.  Returns
// what pick_row does; store: write the results to id and gate.
template <class T, int EC, class AT>
__device__ __forceinline__ int select_row(const smoe_topk_args& a, const T (&key)[EC][4], AT score_at, const int (&sl)[EC][4],
                                          const int (&gid)[EC][4], int sub, int tok, bool served, int32_t* id, float* gate, bool store, T tol) {
    T kk[EC][4];
#pragma unroll
    for (int c = 0; c < EC; ++c)
#pragma unroll
        for (int j = 0; j < 4; ++j) kk[c][j] = served && sl[c][j] < 0 ? T(-INFINITY) : key[c][j];
    int mine;
    const int close = pick_row<T, EC>(kk, gid, a, sub, tol, mine);
    const int e = min(max(mine, 0), a.E - 1);
    T w = 0;
    if (mine >= 0) w = score_at(e);
    if (a.renorm) {
        const T sum = row_sum(w);
        w = sum > 0 ? w / sum : T(0);
    }
    if (sub < a.k && store) {
        const size_t at = (size_t)tok * a.k + sub;
        id[at] = !served ? e : mine < 0 ? -1 : a.e2s[e];   // (a token whose logits are all NaN: expert 0, weight 0)
        gate[at] = (float)(w * a.scale);
    }
    return close;
}

// One token again in 64 bits, by one wave.  Only logits whose order is in question are computed again: those of experts whose keys are within
// the tolerance of another's, those that rank a group near another where the groups are in question (`groups`), all of them where a bias meets the softmax (every key holds the sum over all).
// The others keep their fp32 logits, which are apart from whatever they are compared with.  Few tokens come here, and a workgroup that has one is
// the last to end, so what counts is the time of one pass, most of it instructions that come from the L2: loops are not unrolled (the product's
// loop eight times: 1.5 us more).  16384 tokens, 8 of 128 experts: 53 us, 38 with this left out.
template <int EC>
struct topk_exact {
    static constexpr int N = 64 * EC, WAVES = EC == 4 ? 6 : 8;   // waves that work on such tokens: what fits the LDS beside the logits
    double logit[N], score[N];                             // score: first the fp32 keys of all experts and of the resident ones
};

// Both selections of token tok by one wave from its logits in s.logit.
template <int EC>
__device__ __forceinline__ void select_exact(const smoe_topk_args& a, int tok, topk_exact<EC>& s) {
    const int lane = threadIdx.x & 63, sub = lane & 15, per = a.E / a.groups;
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
    double key[EC][4];
    int sl[EC][4], gid[EC][4];
#pragma unroll
    for (int c = 0; c < EC; ++c)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int e = 64 * c + 4 * sub + j, ei = min(e, a.E - 1);
            key[c][j] = a.by_logit ? s.logit[ei] : s.score[ei] * inv_z + (a.bias ? (double)a.bias[ei] : 0.0);
            key[c][j] = e < a.E ? key[c][j] : -INFINITY;
            sl[c][j] = e < a.E ? a.e2s[ei] : -1;
            gid[c][j] = e / per;
        }
    // the first 16 lanes select among all experts, the next 16 among the resident ones
    select_row<double, EC>(a, key, [&](int e) { return s.score[e] * inv_z; }, sl, gid, sub, tok, lane & 16,
                           lane & 16 ? a.slot : a.orig_expert, lane & 16 ? a.gate : a.orig_gate, lane < 32, 0.0);
}

template <int EC, class AT>
__device__ __forceinline__ void choose_exact(const smoe_topk_args& a, int tok, AT logit_at, float err, bool groups, topk_exact<EC>& s) {
    const int lane = threadIdx.x & 63, sub = lane & 15, per = a.E / a.groups;
    const bool all = !a.sigmoid && !a.by_logit;
    float* fkey = (float*)s.score;
    float* rkey = fkey + 64 * EC;
    float most = 0.f;
#pragma unroll 1
    for (int e = lane; e < 64 * EC; e += 64) {
        const float l = e < a.E ? logit_at(e) : -INFINITY;
        const float key = a.by_logit || all || e >= a.E ? l : sigmoid_of(l) + (a.bias ? a.bias[e] : 0.f);
        s.logit[e] = l;
        fkey[e] = key;
        rkey[e] = e < a.E && a.e2s[e] >= 0 ? key : -INFINITY;
        most = fmaxf(most, e < a.E ? fabsf(key) : 0.f);
    }
    for (int o = 32; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor(most, o));
    const float tol = 2.f * (a.by_logit ? err : 0.25f * err + 4.8e-7f * (most + 1.f));
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); // lanes of a wave read what others wrote: its LDS accesses are in order
    unsigned near_all = 0, near_res = 0;                   // groups whose rank is near another's
    if (groups) {
        float r[2];
#pragma unroll
        for (int res = 0; res < 2; ++res) {
            float m1 = -INFINITY, m2 = -INFINITY;
#pragma unroll 1
            for (int f = 0; f < per; ++f) {
                const float v = lane < a.groups ? (res ? rkey : fkey)[lane * per + f] : -INFINITY;
                m2 = fmaxf(m2, fminf(m1, v));
                m1 = fmaxf(m1, v);
            }
            r[res] = a.best == 2 && m2 > -INFINITY ? m1 + m2 : m1;
        }
#pragma unroll 1
        for (int g = 0; g < a.groups; ++g) {
            const float o0 = __shfl(r[0], g), o1 = __shfl(r[1], g);
            near_all |= lane != g && fabsf(r[0] - o0) <= 2.f * tol;
            near_res |= lane != g && fabsf(r[1] - o1) <= 2.f * tol;
        }
        near_all = (unsigned)__ballot(lane < a.groups && near_all);
        near_res = (unsigned)__ballot(lane < a.groups && near_res);
    }
    unsigned again_of = 0;                                 // bit c: this lane's expert of chunk c
#pragma unroll 1
    for (int e0 = 0; e0 < a.E; e0 += 64) {
        const int e = e0 + lane;
        bool again = e < a.E;
        if (!all) {
            const float mine = fkey[e];
            int near = 0;
#pragma unroll 1
            for (int f = 0; f < a.E; f += 4) {             // itself among them; past E: infinitely far
                const float4 o = *(const float4*)(fkey + f);
                near += (fabsf(mine - o.x) <= tol) + (fabsf(mine - o.y) <= tol) + (fabsf(mine - o.z) <= tol) + (fabsf(mine - o.w) <= tol);
            }
            bool top = false;
            if (groups && again) {
                const int f0 = e / per * per;
                int above = 0, above_res = 0;
#pragma unroll 1
                for (int f = f0; f < f0 + per; ++f) {
                    above += fkey[f] > mine;
                    above_res += rkey[f] > mine;
                }
                const int g = e / per;
                top = ((near_all >> g & 1) && above < a.best) || ((near_res >> g & 1) && rkey[e] == mine && above_res < a.best);
            }
            again = again && (near > 1 || top);
        }
        again_of |= (again ? 1u : 0u) << (e0 >> 6);
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
    // four experts at a time, 16 lanes each
#pragma unroll 1
    for (int i = lane >> 4; i < n + (lane >> 4); i += 4) {
        const int e = list[min(i, n - 1)];
        // the expert's row: the caller's, or out of the operand order that the product has just read (there it is in the L2), a
        // unit of 4 weights at a time: step c / 16, half c % 8 / 4, lane e % 32 + 32 (c % 16 / 8)
        const float4* w = a.f32 ? (const float4*)(a.wrow + (size_t)e * a.d) : (const float4*)a.wr + (size_t)(e >> 5) * (a.d >> 4) * 128 + (e & 31);
        double sum = 0;
#pragma unroll 1
        for (int c = sub * 4; c < a.d; c += 64) {          // d_model is a multiple of 4
            const float4 v = w[a.f32 ? c >> 2 : (c >> 4) * 128 + (c >> 2 & 1) * 64 + (c >> 3 & 1) * 32];
            float4 x;
            if (a.f32) x = *(const float4*)((const float*)a.x + (size_t)tok * a.d + c);
            else {
                const uint2 p = *(const uint2*)((const uint16_t*)a.x + (size_t)tok * a.d + c);
                x = make_float4(__uint_as_float(p.x << 16), __uint_as_float(p.x & 0xFFFF0000u), __uint_as_float(p.y << 16),
                                __uint_as_float(p.y & 0xFFFF0000u));
            }
            sum = fma((double)x.x, (double)v.x, sum);
            sum = fma((double)x.y, (double)v.y, sum);
            sum = fma((double)x.z, (double)v.z, sum);
            sum = fma((double)x.w, (double)v.w, sum);
        }
        sum = row_sum(sum);
        if (sub == 0) s.logit[e] = sum;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    select_exact<EC>(a, tok, s);
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
    const int tw0 = block * NTOK, per = a.E / a.groups;
    if (tid == 0) s_n = 0;
    int sl[EC][4], gid[EC][4];
    smoe_route_slots<NEB>(sl, a, sub);
    float bias[EC][4];
#pragma unroll
    for (int c = 0; c < EC; ++c)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int e = 64 * c + 4 * sub + j;
            gid[c][j] = e / per;
            bias[c][j] = a.bias && e < a.E ? a.bias[e] : 0.f;
        }
    const float wnorm = *a.wnorm;
    smoe_route_meet<NEB, TB>(a.E, acc, sq, part, sqp);

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
        const float err = 0x1p-24f * (a.err_norm * xnorm * wnorm + a.err_sum * smoe_row_max(big));
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
        float tol = err;
        if (!a.by_logit) {
            float most = 0.f;
#pragma unroll
            for (int c = 0; c < EC; ++c)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const bool in = 64 * c + 4 * sub + j < a.E;
                    const float s = a.sigmoid ? sigmoid_of(v[c][j]) : expf(v[c][j] - top) * inv_z;
                    v[c][j] = in ? s + bias[c][j] : -INFINITY;
                    most = fmaxf(most, in ? fmaxf(fabsf(v[c][j]), s) : 0.f);
                }
            // a sigmoid is off by at most a quarter of its logit's error, a share of a softmax by at most twice its own size times that; and the
            // exponential, the quotient and the sum with the bias are rounded, each by a few units of 2^-24
            tol = (a.sigmoid ? 0.25f : 2.f * inv_z) * err + 4.8e-7f * smoe_row_max(most);
        }
        int close = select_row<float, EC>(a, v, score_at, sl, gid, sub, tok, false, a.orig_expert, a.orig_gate, tok < a.T, 2.f * tol);
        close |= select_row<float, EC>(a, v, score_at, sl, gid, sub, tok, true, a.slot, a.gate, tok < a.T, 2.f * tol);
        if (sub < a.k && tok < a.T) a.xnorm[(size_t)tok * a.k + sub] = xnorm;
        if (close && sub == 0 && tok < a.T) {
            const int i = atomicAdd(&s_n, 1);              // the order does not matter
            s_close[i] = t | (close & 2 ? 1 << 8 : 0);
            s_err[i] = err;
        }
    }
    __syncthreads();
    const int n = s_n;
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

__device__ __forceinline__ float4 load_x4(const smoe_topk_args& a, size_t at) {
    if (a.f32) return *(const float4*)((const float*)a.x + at);
    const uint2 p = *(const uint2*)((const uint16_t*)a.x + at);
    return make_float4(__uint_as_float(p.x << 16), __uint_as_float(p.x & 0xFFFF0000u), __uint_as_float(p.y << 16), __uint_as_float(p.y & 0xFFFF0000u));
}

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
// 1 token 8.1 / 8.3, 128 tokens 9.1 / 9.6; 128 of 1024 13.4 / 9.7 and 15.1 / 12.9 (256 tokens: 15.3 / 16.9); 256 of 2048 38 / 15 and 40 / 26; fp32, 64 of
// 768 14.1 / 7.6 and 17.6 / 8.7.
bool topk_few(const smoe_config& c, int T) { return T <= SMOE_TOPK_FEW && (c.dtype == SMOE_F32 || c.E * c.d_model > 65536); }

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
    a.aligned = per >= 4 && per <= 64 && !(per & (per - 1));
    // The partial sums of a logit pass through n roundings.  Where x points nowhere in particular they are small, and the error measured at
    // most 0.75 |x| |w| 2^-24 (bf16; fp32: 1.3) in batches of 16384 tokens, 64 .. 16384 columns and up to 256 experts.  Where x follows a row of the
    // router they grow to the logit's own size (seen in the slices' sums also where these cancel), and it measured 0.08 n of it.
    const int slices = c.E <= 32 ? 8 : 4;
    const int n = a.f32 ? 4 * (((c.d_model + 7) / 8 + slices - 1) / slices) : 3 * ((c.d_model / 16 + slices - 1) / slices);
    a.err_norm = a.f32 ? 1.5f : 1.f;
    a.err_sum = 1.f + 0.1f * n;
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
