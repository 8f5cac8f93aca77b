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
// is put on a list, and the workgroup repeats it in 64 bits, product, scores and selection, from x and the router's rows in memory.
// Without a bias, and with single experts ranking the groups, the keys are the logits themselves, of which every score is a rising
// function.

#include <climits>

#include "route_mfma.h"

struct smoe_topk_args : smoe_route_args {
    const float* bias;
    const float* wnorm;           // largest |w_e|
    int k, sigmoid, groups, kept, best, renorm, by_logit, f32;
    float scale, err;             // err: estimated error of a logit, in units of |x| |w| 2^-24
};

namespace {
__device__ __forceinline__ float sigmoid_of(float v) { return 1.0f / (1.0f + expf(-v)); }
__device__ __forceinline__ double sigmoid_of(double v) { return 1.0 / (1.0 + exp(-v)); }

// The best experts by key of one token, in its 16 lanes: lane `sub` is left with the choice number `sub` (-1: none).  Returns whether a
// distance that decided something is at most tol (keys) or rtol (ranks of groups).  gid: group of each of the lane's experts.
template <int EC>
__device__ __forceinline__ bool pick_row(float (&key)[EC][4], const int (&gid)[EC][4], const smoe_topk_args& a, int sub, float tol, int& mine) {
    bool close = false;
    if (a.groups > 1) {
        float rank = -INFINITY;                            // of group `sub`
        for (int g = 0; g < a.groups; ++g) {
            float m1 = -INFINITY, m2 = -INFINITY;          // the two largest keys of the group
#pragma unroll
            for (int c = 0; c < EC; ++c)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float v = gid[c][j] == g ? key[c][j] : -INFINITY;
                    m2 = fmaxf(m2, fminf(m1, v));
                    m1 = fmaxf(m1, v);
                }
            auto merge = [&](float o1, float o2) {
                m2 = fmaxf(fminf(m1, o1), fmaxf(m2, o2));
                m1 = fmaxf(m1, o1);
            };
            merge(smoe_row_ror<8>(m1), smoe_row_ror<8>(m2));
            merge(smoe_row_ror<4>(m1), smoe_row_ror<4>(m2));
            merge(smoe_row_ror<2>(m1), smoe_row_ror<2>(m2));
            merge(smoe_row_ror<1>(m1), smoe_row_ror<1>(m2));
            const float r = a.best == 2 && m2 > -INFINITY ? m1 + m2 : m1;
            rank = g == sub ? r : rank;
        }
        unsigned kept = 0;
        float last = INFINITY;
        for (int i = 0; i < a.kept; ++i) {
            last = smoe_row_max(rank);
            const int w = smoe_row_min(rank == last ? sub : 99);
            if (last > -INFINITY) kept |= 1u << (w & 31);
            rank = w == sub ? -INFINITY : rank;
        }
        const float next = smoe_row_max(rank);
        close = last - next <= (a.best == 2 ? 2.f * tol : tol);     // (two empty groups: NaN, not close)
#pragma unroll
        for (int c = 0; c < EC; ++c)
#pragma unroll
            for (int j = 0; j < 4; ++j) key[c][j] = (kept >> (gid[c][j] & 31)) & 1u ? key[c][j] : -INFINITY;
    }
    mine = -1;
    float last = INFINITY;
    for (int i = 0; i <= a.k; ++i) {                       // one round more than choices: the distance to the next best
        float m = -INFINITY;
#pragma unroll
        for (int c = 0; c < EC; ++c)
#pragma unroll
            for (int j = 0; j < 4; ++j) m = fmaxf(m, key[c][j]);
        m = smoe_row_max(m);
        close |= last - m <= tol;
        last = m;
        if (i == a.k) break;                               // uniform
        int e = INT_MAX;
#pragma unroll
        for (int c = EC - 1; c >= 0; --c)
#pragma unroll
            for (int j = 3; j >= 0; --j) e = key[c][j] == m ? 64 * c + 4 * sub + j : e;
        e = smoe_row_min(e);
        if (m > -INFINITY) mine = i == sub ? e : mine;
#pragma unroll
        for (int c = 0; c < EC; ++c)
#pragma unroll
            for (int j = 0; j < 4; ++j) key[c][j] = 64 * c + 4 * sub + j == e ? -INFINITY : key[c][j];
    }
    return close;
}

// Weights of the choices in the 16 lanes (w: this lane's score, 0 where it has no choice).
__device__ __forceinline__ float weigh(float w, const smoe_topk_args& a) {
    if (a.renorm) {
        const float sum = smoe_row_sum(w);
        w = sum > 0.f ? w / sum : 0.f;
    }
    return w * a.scale;
}

__device__ __forceinline__ double wave_max(double v) {
    for (int o = 32; o > 0; o >>= 1) v = fmax(v, __shfl_xor(v, o));
    return v;
}
__device__ __forceinline__ double wave_sum(double v) {
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
    return v;
}
__device__ __forceinline__ int wave_min(int v) {
    for (int o = 32; o > 0; o >>= 1) v = min(v, __shfl_xor(v, o));
    return v;
}

// The selection of one token again, by one wave, from its logits in 64 bits; experts lane, lane + 64, ...
__device__ void pick_exact(const double* logit, const smoe_topk_args& a, bool served, int tok) {
    const int lane = threadIdx.x & 63;
    double v[4], s[4], key[4], top = -INFINITY;
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        const int e = lane + 64 * c;
        v[c] = e < a.E ? logit[e] : -INFINITY;
        top = fmax(top, v[c]);
    }
    top = wave_max(top);
    double z = 0;
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        s[c] = lane + 64 * c >= a.E ? 0.0 : a.sigmoid ? sigmoid_of(v[c]) : exp(v[c] - top);
        z += s[c];
    }
    z = a.sigmoid ? 1.0 : wave_sum(z);
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        const int e = lane + 64 * c;
        s[c] /= z;
        const bool ok = e < a.E && (!served || a.e2s[e < a.E ? e : 0] >= 0);
        key[c] = !ok ? -INFINITY : a.by_logit ? v[c] : s[c] + (a.bias ? (double)a.bias[e] : 0.0);
    }
    const int per = a.E / a.groups;
    if (a.groups > 1) {
        double rank = -INFINITY;                           // of group `lane`
        for (int g = 0; g < a.groups; ++g) {
            double m1 = -INFINITY;
#pragma unroll
            for (int c = 0; c < 4; ++c) m1 = fmax(m1, (lane + 64 * c) / per == g ? key[c] : -INFINITY);
            m1 = wave_max(m1);
            int first = INT_MAX;                           // one expert that holds it is left out of the second
#pragma unroll
            for (int c = 0; c < 4; ++c) first = min(first, (lane + 64 * c) / per == g && key[c] == m1 ? lane + 64 * c : INT_MAX);
            first = wave_min(first);
            double m2 = -INFINITY;
#pragma unroll
            for (int c = 0; c < 4; ++c) m2 = fmax(m2, (lane + 64 * c) / per == g && lane + 64 * c != first ? key[c] : -INFINITY);
            m2 = wave_max(m2);
            const double r = a.best == 2 && m2 > -INFINITY ? m1 + m2 : m1;
            rank = g == lane ? r : rank;
        }
        unsigned kept = 0;
        for (int i = 0; i < a.kept; ++i) {
            const double m = wave_max(rank);
            const int w = wave_min(rank == m ? lane : 99);
            if (m > -INFINITY) kept |= 1u << (w & 31);
            rank = w == lane ? -INFINITY : rank;
        }
#pragma unroll
        for (int c = 0; c < 4; ++c) key[c] = (kept >> (((lane + 64 * c) / per) & 31)) & 1u ? key[c] : -INFINITY;
    }
    int mine = -1;
    double w = 0;
    for (int i = 0; i < a.k; ++i) {
        double m = -INFINITY;
#pragma unroll
        for (int c = 0; c < 4; ++c) m = fmax(m, key[c]);
        m = wave_max(m);
        int e = INT_MAX;
#pragma unroll
        for (int c = 3; c >= 0; --c) e = key[c] == m ? lane + 64 * c : e;
        e = wave_min(e);
        double sc = 0;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            sc = fmax(sc, lane + 64 * c == e ? s[c] : 0.0);
            key[c] = lane + 64 * c == e ? -INFINITY : key[c];
        }
        sc = wave_max(sc);
        if (m > -INFINITY && lane == i) { mine = e; w = sc; }
    }
    const double sum = wave_sum(w);
    if (a.renorm) w = sum > 0 ? w / sum : 0;
    if (lane < a.k) {
        const size_t at = (size_t)tok * a.k + lane;
        if (served) {
            a.slot[at] = mine < 0 ? -1 : a.e2s[mine];
            a.gate[at] = (float)(w * a.scale);
        } else {
            a.orig_expert[at] = max(mine, 0);
            a.orig_gate[at] = (float)(w * a.scale);
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
    __shared__ int32_t s_n, s_close[NTOK];                 // tokens to be repeated in 64 bits
    __shared__ double s_logit[256];
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
            gid[c][j] = a.groups > 1 ? e / per : 0;
            bias[c][j] = a.bias && e < a.E ? a.bias[e] : 0.f;
        }
    const float wnorm = *a.wnorm;
    smoe_route_meet<NEB, TB>(a.E, acc, sq, part, sqp);

#pragma unroll
    for (int tb = 0; tb < TB; ++tb) {
        const int t = tb * SMOE_RT + wave * 4 + (lane >> 4), tok = tw0 + t;
        const float* row = part + t * LDP;
        auto logit_at = [&](int e) {                       // fixed order of the slices
            float s = row[e];
#pragma unroll
            for (int q = 1; q < NS; ++q) s += row[q * NTOK * LDP + e];
            return s;
        };
        float v[EC][4], top = -INFINITY, big = 0.f;
#pragma unroll
        for (int c = 0; c < EC; ++c) {
            const float* col = row + min(64 * c + 4 * sub, EP - 4);
            float4 s = *(const float4*)col;
#pragma unroll
            for (int q = 1; q < NS; ++q) {
                const float4 o = *(const float4*)(col + q * NTOK * LDP);
                s.x += o.x; s.y += o.y; s.z += o.z; s.w += o.w;
            }
            v[c][0] = s.x; v[c][1] = s.y; v[c][2] = s.z; v[c][3] = s.w;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const bool in = 64 * c + 4 * sub + j < a.E;
                v[c][j] = in ? v[c][j] : -INFINITY;
                top = fmaxf(top, v[c][j]);
                big = fmaxf(big, in ? fabsf(v[c][j]) : 0.f);
            }
        }
        top = smoe_row_max(top);
        big = smoe_row_max(big);
        float ss = 0.f;
#pragma unroll
        for (int q = 0; q < 2 * NS; ++q) ss += sqp[t + q * NTOK];
        const float xnorm = sqrtf(ss);
        // error of a logit: roundings of partial sums, which are some |x| |w| / sqrt(d) for tokens that point nowhere in particular and grow to
        // the logit's own size for those that do (a.err counts the former, 16 roundings' worth of the largest logit the latter)
        float tol = 5.96e-8f * (a.err * xnorm * wnorm + 16.f * big);
        float z = 1.f;
        if (!a.sigmoid) {
            z = 0.f;
#pragma unroll
            for (int c = 0; c < EC; ++c)
#pragma unroll
                for (int j = 0; j < 4; ++j) z += expf(v[c][j] - top);
            z = smoe_row_sum(z);
        }
        const float inv_z = 1.f / z;
        float key[EC][4];
#pragma unroll
        for (int c = 0; c < EC; ++c)
#pragma unroll
            for (int j = 0; j < 4; ++j) key[c][j] = v[c][j];
        if (!a.by_logit) {
            float most = 0.f;
#pragma unroll
            for (int c = 0; c < EC; ++c)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const bool in = 64 * c + 4 * sub + j < a.E;
                    const float s = a.sigmoid ? sigmoid_of(v[c][j]) : expf(v[c][j] - top) * inv_z;
                    key[c][j] = in ? s + bias[c][j] : -INFINITY;
                    most = fmaxf(most, in ? fmaxf(fabsf(key[c][j]), s) : 0.f);
                }
            most = smoe_row_max(most);
            // a sigmoid is at most a quarter as far off as its logit, a share of a softmax at most twice its own size times that; and the
            // exponential, the quotient and the sum with the bias are rounded
            tol = (a.sigmoid ? 0.25f : 2.f * inv_z) * tol + 4.8e-7f * most;
        }
        bool close = false;
#pragma unroll
        for (int served = 0; served < 2; ++served) {
            float kk[EC][4];
#pragma unroll
            for (int c = 0; c < EC; ++c)
#pragma unroll
                for (int j = 0; j < 4; ++j) kk[c][j] = served && sl[c][j] < 0 ? -INFINITY : key[c][j];
            int mine;
            close |= pick_row<EC>(kk, gid, a, sub, 2.f * tol, mine);
            float w = 0.f;
            const int e = min(max(mine, 0), a.E - 1);
            if (mine >= 0) {
                const float l = logit_at(e);
                w = a.sigmoid ? sigmoid_of(l) : expf(l - top) * inv_z;
            }
            w = weigh(w, a);
            if (sub < a.k && tok < a.T) {
                const size_t at = (size_t)tok * a.k + sub;
                if (served) {
                    a.slot[at] = mine < 0 ? -1 : a.e2s[e];
                    a.gate[at] = w;
                } else {                                   // (a token whose logits are all NaN: expert 0, weight 0)
                    a.orig_expert[at] = e;
                    a.orig_gate[at] = w;
                    a.xnorm[at] = xnorm;
                }
            }
        }
        if (close && sub == 0 && tok < a.T) s_close[atomicAdd(&s_n, 1)] = tok;   // the order does not matter
    }
    __syncthreads();
    for (int i = 0; i < s_n; ++i) {
        const int tok = s_close[i];
        for (int e = wave; e < a.E; e += 8) {
            double sum = 0;
            const float* w = a.wrow + (size_t)e * a.d;
            for (int c = lane; c < a.d; c += 64) {
                const float xv = a.f32 ? ((const float*)a.x)[(size_t)tok * a.d + c]
                                       : __uint_as_float((uint32_t)((const uint16_t*)a.x)[(size_t)tok * a.d + c] << 16);
                sum = fma((double)xv, (double)w[c], sum);
            }
            sum = wave_sum(sum);
            if (lane == 0) s_logit[e] = sum;
        }
        __syncthreads();
        if (wave < 2) pick_exact(s_logit, a, wave == 1, tok);
        __syncthreads();
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
    a.err = 4.f;
    if (c.E <= 32) return launch<1>(a, s);
    if (c.E <= 64) return launch<2>(a, s);
    if (c.E <= 128) return launch<4>(a, s);
    return launch<8>(a, s);
}
