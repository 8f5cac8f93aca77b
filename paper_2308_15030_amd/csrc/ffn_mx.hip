// smoe_expert_ffn_mx: the experts' two products y = ReLU(x W1_k) W2_k (SwapMoE, Background section: E_i(x)) on 8-bit values with
// scales (mx.h), for the sorted (token, choice) pairs of a batch; and the loads of experts into 8-bit slots.
//
// The weights are the instruction's first operand and the tokens its second, so a lane of the accumulator holds one token and, of a
// block of 32 features, 8 q + 4 (lane / 32) + i for q, i < 4.  The hidden activations are rounded to 8 bits between the products: a
// block of 32 features of a token lies in two lanes, so its scale takes one exchange, and the block of 32 tokens x 32 features
// that a wave holds is then one contiguous kilobyte of the second product's operand order.
//
// Two forms of each product:
//   stream_mx_kernel   few rows a slot: what bounds it is the bytes of the weights.  A wave takes one block of 32 features and a
//                      share of the reduction, several loads ahead, straight into registers.
//   tile_mx_kernel     many rows a slot: the matrix cores bound it.  Weights go straight into registers (no other wave of the
//                      workgroup needs them), the token tile is staged through LDS.

#include <algorithm>
#include <cstdio>
#include <string>
#include <type_traits>

#include "mx.h"
#include "wave_ops.h"

namespace {

typedef smoe_mx_acc f32x16;
constexpr int MAX_SLOTS = 256;            // K <= E <= 256 by the C ABI

struct MxArgs {
    const uint8_t* x;                     // first product: q [tokens, R]; second: hidden, operand order
    const uint8_t* xs;                    // their scales: [tokens, pitch], or operand order
    int pitch;
    const int32_t* perm;                  // pair of each sorted row, or NULL (row r is token r)
    int k, tokens;
    const uint8_t* w;                     // slot array
    size_t wstride;                       // bytes of a slot
    const int32_t* phys;
    const int32_t* offsets;
    int nslots, rows, R, N;
    uint8_t* h;                           // first product's output, operand order
    uint8_t* hs;
    uint16_t* y;                          // second product's output [rows, N]
};

// Row tiles of all slots form one list in slot order; segments are re-based to multiples of 32 rows in the hidden activations.
struct SlotMap {
    int first[MAX_SLOTS + 1];             // row tiles before slot k
    int pad[MAX_SLOTS];                   // 32-row blocks before slot k
    int a[MAX_SLOTS], b[MAX_SLOTS];       // clamped segment bounds
};

// Called by every thread of the workgroup; ends with a barrier.
__device__ __forceinline__ void build_slot_map(SlotMap& m, const int32_t* __restrict__ offsets, int nslots, int rows, int bt) {
    if (threadIdx.x < 64) {
        const int lane = threadIdx.x;
        int tiles_before = 0, pad_before = 0;
        for (int base = 0; base < nslots; base += 64) {
            const int k = base + lane;
            int a = 0, b = 0, tiles = 0, pad = 0;
            if (k < nslots) {
                a = min(max(offsets[k], 0), rows);             // clamps guard misuse
                b = max(min(max(offsets[k + 1], 0), rows), a);
                tiles = (b - a + bt - 1) / bt;
                pad = (b - a + 31) >> 5;
            }
            const int tin = smoe_wave_incl_scan(tiles), pin = smoe_wave_incl_scan(pad);
            if (k < nslots) {
                m.first[k] = tiles_before + tin - tiles;
                m.pad[k] = pad_before + pin - pad;
                m.a[k] = a;
                m.b[k] = b;
            }
            tiles_before += __builtin_amdgcn_readlane(tin, 63);
            pad_before += __builtin_amdgcn_readlane(pin, 63);
        }
        if (lane == 0) m.first[nslots] = tiles_before;
    }
    __syncthreads();
}

// The last slot whose first row tile is <= mt (empty slots repeat the next one's).
__device__ __forceinline__ int slot_of_tile(const SlotMap& m, int nslots, int mt) {
    const int lane = threadIdx.x & 63;
    int nle = 0;
    for (int base = 0; base < nslots; base += 64) {
        const int k = base + lane;
        nle += __popcll(__ballot(k < nslots && m.first[k] <= mt));
    }
    return __builtin_amdgcn_readfirstlane(nle - 1);
}

__device__ __forceinline__ int token_of_row(const MxArgs& g, int row) {
    if (!g.perm) return min(row, g.tokens - 1);
    return min(max(g.perm[row] / g.k, 0), g.tokens - 1);       // in range by construction; clamps guard misuse
}

// First product, one block of 32 features x 32 tokens: ReLU, scale, 8 bits, into block `rb` (32 rows) and feature block fb of the hidden
// activations.  Feature block fb is half fb % 2 of step fb / 2; behind an odd number of blocks the other half of the last step is zeroed.
__device__ __forceinline__ void store_hidden(const MxArgs& g, f32x16& acc, int rb, int fb) {
    const int lane = threadIdx.x & 63, nfb = g.N >> 5;
    float amax = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        acc[i] = fmaxf(acc[i], 0.f);
        amax = fmaxf(amax, acc[i]);
    }
    uint32_t lo = __float_as_uint(amax), hi = lo;
    smoe_swap_halves(lo, hi);
    amax = fmaxf(__uint_as_float(lo), __uint_as_float(hi));
    const uint32_t sc = smoe_mx_scale(amax);
    const float inv = smoe_mx_inverse(sc);
    uint32_t q[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        q[i] = smoe_mx_pack(acc[4 * i] * inv, acc[4 * i + 1] * inv, acc[4 * i + 2] * inv, acc[4 * i + 3] * inv);
    smoe_swap_halves(q[0], q[2]);                              // lower lanes: features 0 .. 15, upper: 16 .. 31
    smoe_swap_halves(q[1], q[3]);
    const int step = fb >> 1;
    uint4* dst = (uint4*)(g.h + (size_t)rb * smoe_mx_row_bytes(g.N) + (size_t)step * 2048) + (fb & 1) * 64 + lane;
    uint8_t* sdst = g.hs + (size_t)rb * smoe_mx_row_scales(g.N) + (size_t)(step >> 2) * 256 + (step & 3) + (lane & 31) * 4;
    *dst = make_uint4(q[0], q[2], q[1], q[3]);
    if (lane < 32) sdst[(fb & 1) * 128] = (uint8_t)sc;
    if (fb == nfb - 1 && !(fb & 1)) {
        dst[64] = make_uint4(0, 0, 0, 0);
        if (lane < 32) sdst[128] = 1;
    }
}

// Second product, one block: row `row` of the lane's token gets 32 features from n0 on, rounded once to bf16.
__device__ __forceinline__ void store_rows(const MxArgs& g, const f32x16& acc, int row, bool live, int n0) {
    const int lane = threadIdx.x & 63;
    uint32_t p[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) p[i] = smoe_pack_bf16(acc[2 * i], acc[2 * i + 1]);
#pragma unroll
    for (int i = 0; i < 4; ++i) smoe_swap_halves(p[i], p[i + 4]);   // lower lanes: features 0 .. 15, upper: 16 .. 31
    if (live) {
        uint4* dst = (uint4*)(g.y + (size_t)row * g.N + n0 + 16 * (lane >> 5));
        dst[0] = make_uint4(p[0], p[1], p[4], p[5]);
        dst[1] = make_uint4(p[2], p[3], p[6], p[7]);
    }
}

// The four scale bytes of a group of four steps that belong to this lane's half, of a token's row of scale bytes.
__device__ __forceinline__ uint32_t row_scales(const uint8_t* row, int group, int blocks) {
    const uint2 v = *(const uint2*)(row + group * 8);
    const int left = blocks - group * 8;                       // bytes behind the row's last block are not used: whatever lies there
    uint32_t s = __builtin_amdgcn_perm(v.y, v.x, (threadIdx.x & 32) ? 0x07050301u : 0x06040200u);
    const int mine = (left + ((threadIdx.x & 32) ? 0 : 1)) >> 1;   // blocks of this half
    if (mine < 4) s &= mine > 0 ? (1u << (8 * mine)) - 1u : 0u;
    return s;
}

// ------------------------------------------------------------------ few rows a slot
// One item = 32 rows of a slot x (4 / SPLIT) feature blocks; the SPLIT waves of a feature block take a share of the reduction
// each and meet in LDS.
template <bool FIRST, int SPLIT>
__global__ __launch_bounds__(256) void stream_mx_kernel(const MxArgs g) {
    __shared__ SlotMap m;
    __shared__ float part[4][16][64];
    build_slot_map(m, g.offsets, g.nslots, g.rows, 32);
    constexpr int PER = 4 / SPLIT;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
    const int nfb = g.N >> 5, ftiles = (nfb + PER - 1) / PER;
    const int mt = blockIdx.x / ftiles, ft = blockIdx.x - mt * ftiles;
    if (mt >= m.first[g.nslots]) return;
    const int slot = slot_of_tile(m, g.nslots, mt);
    const int within = mt - m.first[slot], m0 = m.a[slot] + 32 * within, m_end = m.b[slot], rb = m.pad[slot] + within;
    const int fb = ft * PER + wave / SPLIT, part_of = wave % SPLIT;
    const bool on = fb < nfb;
    const int steps = smoe_mx_steps(g.R), blocks = g.R >> 5;
    const int groups = smoe_mx_groups(g.R), gper = (groups + SPLIT - 1) / SPLIT;   // shares are whole groups of four steps
    const int lo = min(part_of * gper * 4, steps), hi = min(lo + gper * 4, steps);
    f32x16 acc;
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[i] = 0.f;
    if (on && lo < hi) {
        const uint8_t* wslot = g.w + (size_t)g.phys[slot] * g.wstride;
        const uint4* wp = (const uint4*)(wslot + (size_t)fb * smoe_mx_row_bytes(g.R)) + lane;
        const uint32_t* wsp = (const uint32_t*)(wslot + (size_t)nfb * smoe_mx_row_bytes(g.R) + (size_t)fb * smoe_mx_row_scales(g.R)) + lane;
        const uint8_t *xrow, *xsrow;
        if (FIRST) {
            const int t = token_of_row(g, min(m0 + (lane & 31), m_end - 1));
            xrow = g.x + (size_t)t * g.R + 16 * (lane >> 5);
            xsrow = g.xs + (size_t)t * g.pitch;
        } else {
            xrow = g.x + (size_t)rb * smoe_mx_row_bytes(g.R) + lane * 16;
            xsrow = g.xs + (size_t)rb * smoe_mx_row_scales(g.R) + lane * 4;
        }
        for (int s0 = lo; s0 < hi; s0 += 4) {
            uint4 w[4][2], x[4][2];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int s = min(s0 + i, steps - 1);
                w[i][0] = smoe_load_stream(wp + (size_t)s * 128);
                w[i][1] = smoe_load_stream(wp + (size_t)s * 128 + 64);
                if (FIRST) {
                    const bool second = s * 64 + 32 < g.R;         // the last step may be half a step
                    x[i][0] = *(const uint4*)(xrow + s * 64);
                    x[i][1] = *(const uint4*)(xrow + s * 64 + (second ? 32 : 0));
                    if (!second) x[i][1] = make_uint4(0, 0, 0, 0);
                } else {
                    x[i][0] = *(const uint4*)(xrow + (size_t)s * 2048);
                    x[i][1] = *(const uint4*)(xrow + (size_t)s * 2048 + 1024);
                }
            }
            const uint32_t ws = wsp[(s0 >> 2) * 64];
            const uint32_t xs = FIRST ? row_scales(xsrow, s0 >> 2, blocks) : *(const uint32_t*)(xsrow + (s0 >> 2) * 256);
            smoe_mx_mfma<0>(acc, w[0], x[0], ws, xs);
            if (s0 + 1 < hi) smoe_mx_mfma<1>(acc, w[1], x[1], ws, xs);
            if (s0 + 2 < hi) smoe_mx_mfma<2>(acc, w[2], x[2], ws, xs);
            if (s0 + 3 < hi) smoe_mx_mfma<3>(acc, w[3], x[3], ws, xs);
        }
    }
    if (SPLIT > 1) {
        if (part_of)
#pragma unroll
            for (int i = 0; i < 16; ++i) part[wave][i][lane] = acc[i];
        __syncthreads();
        if (part_of) return;
#pragma unroll
        for (int q = 1; q < SPLIT; ++q)                        // in order of the reduction
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[i] += part[wave + q][i][lane];
    }
    if (!on) return;
    if (FIRST) store_hidden(g, acc, rb, fb);
    else store_rows(g, acc, m0 + (lane & 31), m0 + (lane & 31) < m_end, fb * 32);
}

// ------------------------------------------------------------------ loads of experts
// One workgroup takes 64 reduction rows x 128 feature columns of a bank matrix [R, N] (bf16): rows are read with 16-byte pieces, turned
// through LDS; wave w makes the operand block of the columns 32 w .. 32 w + 31.
constexpr int MX_PACK_COLS = 128;
constexpr int MX_PACK_LD = MX_PACK_COLS + 2;

__device__ __forceinline__ void pack_mx_tile(const uint16_t* __restrict__ src, int R, int N, uint8_t* __restrict__ dst, int tile, uint16_t* lds) {
    const int ctiles = (N + MX_PACK_COLS - 1) / MX_PACK_COLS;
    const int step = tile / ctiles, ct = tile - step * ctiles, n0 = ct * MX_PACK_COLS, tid = threadIdx.x;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int idx = tid + i * 256, r = idx >> 4, col = n0 + (idx & 15) * 8, row = step * 64 + r;
        uint4 v = make_uint4(0, 0, 0, 0);                      // rows past the matrix: zeros
        if (col < N && row < R) v = *(const uint4*)(src + (size_t)row * N + col);
        uint32_t* d = (uint32_t*)&lds[r * MX_PACK_LD + (idx & 15) * 8];
        d[0] = v.x; d[1] = v.y; d[2] = v.z; d[3] = v.w;
    }
    __syncthreads();
    const int wave = tid >> 6, lane = tid & 63, nb = ct * (MX_PACK_COLS / 32) + wave, nfb = N >> 5;
    if (nb < nfb) {
        const int c = wave * 32 + (lane & 31), h = lane >> 5;
        auto at = [&](int r) { return __uint_as_float((uint32_t)lds[r * MX_PACK_LD + c] << 16); };
        float amax = 0.f;
        for (int i = 0; i < 32; ++i) amax = fmaxf(amax, fabsf(at(32 * h + i)));
        uint32_t s0 = smoe_mx_scale(amax), s1 = s0;
        const uint32_t own = s0;
        smoe_swap_halves(s0, s1);                              // the scales of both blocks of the column
        uint4* out = (uint4*)(dst + (size_t)nb * smoe_mx_row_bytes(R) + (size_t)step * 2048) + lane;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const float inv = smoe_mx_inverse(half ? s1 : s0);
            const int r0 = 32 * half + 16 * h;
            uint32_t q[4];
#pragma unroll
            for (int i = 0; i < 4; ++i)
                q[i] = smoe_mx_pack(at(r0 + 4 * i) * inv, at(r0 + 4 * i + 1) * inv, at(r0 + 4 * i + 2) * inv, at(r0 + 4 * i + 3) * inv);
            out[half * 64] = make_uint4(q[0], q[1], q[2], q[3]);
        }
        uint8_t* sc = dst + (size_t)nfb * smoe_mx_row_bytes(R) + (size_t)nb * smoe_mx_row_scales(R) + (size_t)(step >> 2) * 256 + lane * 4;
        sc[step & 3] = (uint8_t)own;
        if (step == smoe_mx_steps(R) - 1)
            for (int i = (step & 3) + 1; i < 4; ++i) sc[i] = 1;    // steps that do not exist
    }
}

// As pack_bf16_kernel of resident.hip: both matrices of one expert and, with map_slot >= 0, the maps.
template <bool WALK>
__global__ __launch_bounds__(256) void pack_mx_kernel(const uint16_t* __restrict__ w1, const uint16_t* __restrict__ w2, int d_model, int d_ff,
                                                      uint8_t* __restrict__ dst1, uint8_t* __restrict__ dst2, int nblk1, int nblk, int32_t* e2s,
                                                      int32_t* s2e, int32_t* phys, int map_slot, int expert, int old_expert, int p) {
    __shared__ __align__(16) uint16_t lds[64 * MX_PACK_LD];
    int t = blockIdx.x;                                        // the grid has no more workgroups than there are tiles
    do {
        if (t < nblk1) pack_mx_tile(w1, d_model, d_ff, dst1, t, lds);
        else pack_mx_tile(w2, d_ff, d_model, dst2, t - nblk1, lds);
        if (WALK) __syncthreads();                             // the tile buffer is reused
        t += gridDim.x;
    } while (WALK && t < nblk);
    if (map_slot >= 0 && blockIdx.x == 0 && threadIdx.x == 0) {
        if (old_expert >= 0) e2s[old_expert] = -1;
        e2s[expert] = map_slot;
        s2e[map_slot] = expert;
        phys[map_slot] = p;
    }
}

template <bool FIRST>
int launch_product(const MxArgs& g, hipStream_t s) {
    constexpr int SPLIT = 4;
    const int nfb = g.N >> 5, per = 4 / SPLIT, ftiles = (nfb + per - 1) / per;
    const size_t tiles = (size_t)(g.rows / 32 + std::min(g.nslots, g.rows));   // an upper bound of the sum of ceil(len / 32)
    hipLaunchKernelGGL((stream_mx_kernel<FIRST, SPLIT>), dim3((unsigned)(tiles * ftiles)), dim3(256), 0, s, g);
    return smoe_check_hip(hipGetLastError(), FIRST ? "smoe_expert_ffn_mx: first product launch" : "smoe_expert_ffn_mx: second product launch");
}

}  // namespace

int smoe_launch_pack_mx(const smoe_layer* L, int slot, const void* w1_src, const void* w2_src, hipStream_t s, int map_slot, int expert,
                        int old_expert) {
    const smoe_config& c = L->cfg;
    const int nblk1 = smoe_mx_steps(c.d_model) * ((c.d_ff + MX_PACK_COLS - 1) / MX_PACK_COLS);
    const int nblk2 = smoe_mx_steps(c.d_ff) * ((c.d_model + MX_PACK_COLS - 1) / MX_PACK_COLS);
    const size_t stride = smoe_slot_bytes(c);
    const int nblk = nblk1 + nblk2;
    hipLaunchKernelGGL(L->load_from_host ? pack_mx_kernel<true> : pack_mx_kernel<false>,
                       dim3((unsigned)(L->load_from_host ? std::min(nblk, SMOE_PACK_HOST_WGS) : nblk)), dim3(256), 0, s, (const uint16_t*)w1_src,
                       (const uint16_t*)w2_src, c.d_model, c.d_ff, (uint8_t*)L->slot_w1 + (size_t)slot * stride,
                       (uint8_t*)L->slot_w2 + (size_t)slot * stride, nblk1, nblk, L->d_expert_to_slot, L->d_slot_to_expert, L->d_phys, map_slot,
                       expert, old_expert, slot);
    return smoe_check_hip(hipGetLastError(), "expert load launch");
}

int smoe_launch_ffn_mx(const smoe_layer* L, const void* q, const void* q_scale, const int32_t* perm, int k, const int32_t* offsets, int T,
                       void* y_perm, hipStream_t s) {
    const smoe_config& c = L->cfg;
    uint8_t* h = (uint8_t*)L->d_hidden;
    uint8_t* hs = h + smoe_mx_hidden_blocks(c) * smoe_mx_row_bytes(c.d_ff);
    MxArgs g{};
    g.x = (const uint8_t*)q;
    g.xs = (const uint8_t*)q_scale;
    g.pitch = (int)smoe_scale_pitch(c.d_model);
    g.perm = perm;
    g.k = k;
    g.tokens = T;
    g.w = (const uint8_t*)L->slot_w1;
    g.wstride = smoe_slot_bytes(c);
    g.phys = L->d_phys;
    g.offsets = offsets;
    g.nslots = c.K;
    g.rows = T * k;
    g.R = c.d_model;
    g.N = c.d_ff;
    g.h = h;
    g.hs = hs;
    g.y = (uint16_t*)y_perm;
    int rc = launch_product<true>(g, s);
    if (rc) return rc;
    g.x = h;
    g.xs = hs;
    g.w = (const uint8_t*)L->slot_w2;
    g.R = c.d_ff;
    g.N = c.d_model;
    return launch_product<false>(g, s);
}
