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
//   tile_mx_kernel     many rows a slot: what bounds it is the way of the operands through LDS next to the matrix cores.  Both are staged
//                      there, 16384 rows of 1024 x 4096: 1440 TFLOP/s.

#include <algorithm>
#include <climits>
#include <cstdio>
#include <string>
#include <type_traits>

#include "mx.h"
#include "wave_ops.h"

namespace {

typedef smoe_mx_acc f32x16;

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
    int nslots, rows, R, N, cus;
    bool past;                            // weights come from memory (smoe_weights_outgrow_cache)
    uint8_t* h;                           // first product's output, operand order
    uint8_t* hs;
    uint16_t* y;                          // second product's output [rows, N]
};

__device__ __forceinline__ int uni(int v) { return __builtin_amdgcn_readfirstlane(v); }

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
        acc[i] = __builtin_elementwise_maximum(acc[i], 0.f);   // (keeps a NaN, as fmaxf does not)
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

// The four scale bytes of a group of four steps that belong to this lane's half, of the group's eight in a row of scale bytes; `left`: blocks
// of the row from the group on.  Bytes behind the row's last block are not used, whatever lies there.
__device__ __forceinline__ uint32_t half_scales(uint2 v, int left) {
    uint32_t s = __builtin_amdgcn_perm(v.y, v.x, (threadIdx.x & 32) ? 0x07050301u : 0x06040200u);
    const int mine = (left + ((threadIdx.x & 32) ? 0 : 1)) >> 1;   // blocks of this half
    if (mine < 4) s &= mine > 0 ? (1u << (8 * mine)) - 1u : 0u;
    return s;
}

// ------------------------------------------------------------------ few rows a slot
// One item = 32 rows of a slot x one feature block; the NW waves of a workgroup take a share of the reduction each and meet in LDS.  A wave asks for
// BATCH steps at a time, one batch ahead of the products.  NT: the weights come from memory, not from the Infinity Cache, and are kept out of the
// caches (smoe_weights_outgrow_cache).
template <bool NT>
__device__ __forceinline__ uint4 load_weights(const uint4* p) { return NT ? smoe_load_stream(p) : *p; }

template <bool FIRST, int NW, int BATCH, bool NT>
__global__ __launch_bounds__(64 * NW) void stream_mx_kernel(const MxArgs g) {
    __shared__ float part[NW > 1 ? NW - 1 : 1][16][64];
    const int wave = uni(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int nfb = g.N >> 5, item = blockIdx.x / nfb, fb = blockIdx.x - item * nfb;
    // the item's slot and rows, worked out by every wave for itself: 32-row tiles of all slots in slot order
    int m0 = 0, m_end = 0, rb = 0, phys = -1;
    for (int base = 0, before = 0; base < g.nslots; base += 64) {
        const int k = base + lane;
        int a = 0, b = 0, p = 0;
        if (k < g.nslots) {
            p = g.phys[k];
            a = min(max(g.offsets[k], 0), g.rows);         // clamps guard misuse
            b = max(min(max(g.offsets[k + 1], 0), g.rows), a);
        }
        const int n = (b - a + 31) >> 5, incl = smoe_wave_incl_scan(n), all = __builtin_amdgcn_readlane(incl, 63);
        if (item < before + all) {                         // uniform: the slot is among these 64
            const int l = __popcll(__ballot(before + incl <= item));   // slots that end in front of the item
            const int within = item - before - __builtin_amdgcn_readlane(incl - n, l);
            m0 = __builtin_amdgcn_readlane(a, l) + 32 * within;
            m_end = __builtin_amdgcn_readlane(b, l);
            phys = __builtin_amdgcn_readlane(p, l);
            rb = item;
            break;
        }
        before += all;
    }
    if (phys < 0) return;
    const int steps = smoe_mx_steps(g.R), blocks = g.R >> 5, share = (steps + NW - 1) / NW;
    const int lo = min(wave * share, steps), hi = min(lo + share, steps);
    f32x16 acc;
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[i] = 0.f;
    if (lo < hi) {
        const uint8_t* wslot = g.w + (size_t)phys * g.wstride;
        const uint4* wp = (const uint4*)(wslot + (size_t)fb * smoe_mx_row_bytes(g.R)) + lane;
        const uint8_t* wsp = wslot + (size_t)nfb * smoe_mx_row_bytes(g.R) + (size_t)fb * smoe_mx_row_scales(g.R) + lane * 4;
        uint4 w[2][BATCH][2], x[2][BATCH][2];
        uint32_t ws[2][BATCH], xs[2][BATCH];
        auto ask_w = [&](auto sc, int s0) {                // past the share: its last step again, not multiplied
            constexpr int z = decltype(sc)::value;
#pragma unroll
            for (int i = 0; i < BATCH; ++i) {
                const int s = min(s0 + i, hi - 1);
                w[z][i][0] = load_weights<NT>(wp + (size_t)s * 128);
                w[z][i][1] = load_weights<NT>(wp + (size_t)s * 128 + 64);
                ws[z][i] = wsp[(s >> 2) * 256 + (s & 3)];
            }
        };
        ask_w(std::integral_constant<int, 0>{}, lo);       // on their way while the token of the row is looked up
        const uint8_t *xrow, *xsrow;
        if (FIRST) {
            const int t = token_of_row(g, min(m0 + (lane & 31), m_end - 1));
            xrow = g.x + (size_t)t * g.R + 16 * (lane >> 5);
            xsrow = g.xs + (size_t)t * g.pitch + (lane >> 5);
        } else {
            xrow = g.x + (size_t)rb * smoe_mx_row_bytes(g.R) + lane * 16;
            xsrow = g.xs + (size_t)rb * smoe_mx_row_scales(g.R) + lane * 4;
        }
        auto ask_x = [&](auto sc, int s0) {
            constexpr int z = decltype(sc)::value;
#pragma unroll
            for (int i = 0; i < BATCH; ++i) {
                const int s = min(s0 + i, hi - 1);
                if (FIRST) {                               // the last step may be half a step: nothing behind it is used
                    const bool second = s * 64 + 32 < g.R;
                    x[z][i][0] = *(const uint4*)(xrow + s * 64);
                    x[z][i][1] = *(const uint4*)(xrow + s * 64 + (second ? 32 : 0));
                    if (!second) x[z][i][1] = make_uint4(0, 0, 0, 0);
                    const uint32_t v = xsrow[s * 2];
                    xs[z][i] = 2 * s + (lane >> 5) < blocks ? v : 0;
                } else {
                    x[z][i][0] = *(const uint4*)(xrow + (size_t)s * 2048);
                    x[z][i][1] = *(const uint4*)(xrow + (size_t)s * 2048 + 1024);
                    xs[z][i] = xsrow[(s >> 2) * 256 + (s & 3)];
                }
            }
        };
        auto multiply = [&](auto sc, int s0) {
            constexpr int z = decltype(sc)::value;
#pragma unroll
            for (int i = 0; i < BATCH; ++i)
                if (s0 + i < hi) smoe_mx_mfma<0>(acc, w[z][i], x[z][i], ws[z][i], xs[z][i]);
        };
        ask_x(std::integral_constant<int, 0>{}, lo);
        for (int s0 = lo; s0 < hi; s0 += 2 * BATCH) {
            if (s0 + BATCH < hi) {
                ask_w(std::integral_constant<int, 1>{}, s0 + BATCH);
                ask_x(std::integral_constant<int, 1>{}, s0 + BATCH);
            }
            __builtin_amdgcn_sched_barrier(0);             // the next batch is on its way
            multiply(std::integral_constant<int, 0>{}, s0);
            if (s0 + BATCH >= hi) break;
            if (s0 + 2 * BATCH < hi) {
                ask_w(std::integral_constant<int, 0>{}, s0 + 2 * BATCH);
                ask_x(std::integral_constant<int, 0>{}, s0 + 2 * BATCH);
            }
            __builtin_amdgcn_sched_barrier(0);
            multiply(std::integral_constant<int, 1>{}, s0 + BATCH);
        }
    }
    if (wave)
#pragma unroll
        for (int i = 0; i < 16; ++i) part[wave - 1][i][lane] = acc[i];
    __syncthreads();
    if (wave) return;
#pragma unroll
    for (int q = 0; q < NW - 1; ++q)                       // in order of the reduction
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[i] += part[q][i][lane];
    if (FIRST) store_hidden(g, acc, rb, fb);
    else store_rows(g, acc, m0 + (lane & 31), m0 + (lane & 31) < m_end, fb * 32);
}

// ------------------------------------------------------------------ many rows a slot
// Tile = FB blocks of 32 features x at most TBK blocks of 32 tokens, both operands staged through a ring of ST stages in LDS, one step of 64 reduction
// elements a stage.  Four waves, WF along the features and WT along the tokens.  Loads go from memory to LDS without passing through registers,
// ST - 1 steps ahead; each wave issues the same number of them a step, so that one count says what has landed.  The scales of four steps
// come the same way, in front of the first step's operands.
//
// Two workgroups to a compute unit (FB = 8: 80 KB of LDS each), so that one multiplies while the other waits at its barrier, looks its next tile up
// or narrows its results.  A workgroup of 256 x 256 tiles with twice the accumulators moves a third fewer bytes a product, but its waves are alone on
// their SIMDs: 239 us for the 16384 rows of 1024 x 4096 that take 190 here, 210 with its next tile's loads in flight through the stores.  Traces of copies
// without a part (one slot, first + second product, 171 us): without loads 140, without products 143, without stores 133; second product of 4 slots, 92
// us: without loads 68, also without operand reads 55, without loads and products 56, barriers and stores alone 25.
extern __shared__ __align__(16) char mx_lds[];
constexpr int MX_BLK = 2048;              // bytes of a block of one step
constexpr int TILE_COST0 = 20;            // a tile beside its steps, in steps of one token block; 0 to 60 chose tiles of the same speed

__device__ __forceinline__ uint32_t lds_addr(uint32_t off) {
    return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)(mx_lds + off);
}
// Loads from memory to LDS: lane l's 16 (4) bytes land at off + 16 l (4 l), for the lanes of the mask.  Written out because the compiler, which
// cannot tell where the builtin's data lands, would wait for every load in flight before each LDS read.  They have no result registers;
// whoever reads the data counts them (wait_vm) and then passes a barrier.  Nothing else in the kernel uses m0.
__device__ __forceinline__ void dma_16(const void* src, uint32_t off, uint64_t lanes) {
    asm volatile("s_mov_b32 m0, %0\n\ts_mov_b64 exec, %2\n\tglobal_load_lds_dwordx4 %1, off\n\ts_mov_b64 exec, -1" ::"s"(lds_addr(off)), "v"(src), "s"(lanes) : "memory");
}
__device__ __forceinline__ void dma_4(const void* src, uint32_t off) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(lds_addr(off)), "v"(src) : "memory");
}
// Two kilobytes that lie linear in memory (the offset moves both sides).
__device__ __forceinline__ void dma_2k(const char* base, uint32_t lane16, uint32_t off, uint64_t lanes) {
    asm volatile("s_mov_b32 m0, %0\n\ts_mov_b64 exec, %3\n\tglobal_load_lds_dwordx4 %1, %2\n\tglobal_load_lds_dwordx4 %1, %2 offset:1024\n\t"
                 "s_mov_b64 exec, -1" ::"s"(lds_addr(off)), "v"(lane16), "s"(base), "s"(lanes) : "memory");
}
template <int N>
__device__ __forceinline__ void wait_vm() {   // at most the N youngest vector memory operations of this wave are outstanding
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

// Multiples of four in [lo, hi).
constexpr int group_starts(int lo, int hi) { return (hi + 3) / 4 - (lo + 3) / 4; }

constexpr int TBK = 4;                    // most token blocks of a tile
template <int FB, int ST>
struct TileShape {
    static constexpr uint32_t STAGE = (FB + TBK) * MX_BLK;
    static constexpr uint32_t SC = ST * STAGE;             // scales of two groups: weights [FB][256], tokens [TBK][256]
    static constexpr uint32_t SCG = (FB + TBK) * 256;
    static constexpr size_t LDS = SC + 2 * SCG;
};

template <bool FIRST, int FB, int ST>
__global__ __launch_bounds__(256, FB == 8 ? 2 : 3) void tile_mx_kernel(const MxArgs g) {
    using S = TileShape<FB, ST>;
    constexpr int WF = FB == 2 ? 1 : 2, WT = 4 / WF;       // waves along the features and along the tokens
    constexpr int AW = FB / WF, NBW = TBK / WT;            // feature and token blocks that a wave multiplies
    constexpr int WL = FB / 4;                             // feature blocks that a wave loads (0: half a block)
    constexpr int PER = (FB == 2 ? 1 : 2 * WL) + 2, NSC = 2;    // its loads a step, and of the scales a group
    const int tid = threadIdx.x, wave = uni(tid >> 6), lane = tid & 63;
    const int wf = wave % WF, wt = wave / WF;
    const int nfb = g.N >> 5, ftiles = (nfb + FB - 1) / FB, steps = smoe_mx_steps(g.R);
    // This workgroup's item.  Row tiles of all slots in slot order; inside a slot the row tile fastest (first product) or the feature tile.  The
    // dies take an eighth of the list each (workgroups are dealt to them in turn), so that few slots' weights pass through an L2.
    int seg_a, seg_b;                                      // of slot `lane`
    auto segment = [&](int k, int& a, int& b) {
        a = b = 0;
        if (k < g.nslots) {
            a = min(max(g.offsets[k], 0), g.rows);         // clamps guard misuse
            b = max(min(max(g.offsets[k + 1], 0), g.rows), a);
        }
    };
    segment(lane, seg_a, seg_b);
    // Height of the row tiles: those of at most 1, 2, .. blocks are counted, all take the best.
    int H = TBK, G = 0, best = INT_MAX;
#pragma unroll
    for (int h = TBK; h >= 1; --h) {
        int n = 0;
        for (int base = 0; base < g.nslots; base += 64) {
            int a = seg_a, b = seg_b;
            if (base) segment(base + lane, a, b);
            n += __builtin_amdgcn_readlane(smoe_wave_incl_scan((((b - a + 31) >> 5) + h - 1) / h), 63);
        }
        const int cost = ((n * ftiles + g.cus - 1) / g.cus) * (steps * (1 + h) + TILE_COST0);
        if (cost < best) { best = cost; H = h; G = n * ftiles; }
    }
    const int die = blockIdx.x % 8;
    const int lo = (int)((long long)G * die / 8), hi = (int)((long long)G * (die + 1) / 8);
    for (int item = lo + blockIdx.x / 8; item < hi; item += gridDim.x / 8) {
    int slot = 0, slot_a = 0, slot_b = 0, first = 0, pad = 0, tiles = 1;
    {
        int before = 0, pad_before = 0;
        for (int base = 0; base < g.nslots; base += 64) {
            int a = seg_a, b = seg_b;
            if (base) segment(base + lane, a, b);
            const int nblk = (b - a + 31) >> 5, n = (nblk + H - 1) / H;
            const int incl = smoe_wave_incl_scan(n), pincl = smoe_wave_incl_scan(nblk);
            const int all = __builtin_amdgcn_readlane(incl, 63);
            if (item < (before + all) * ftiles) {          // uniform: the slot is among these 64
                const int l = __popcll(__ballot((before + incl) * ftiles <= item));   // slots that end in front of the item
                slot = base + l;
                slot_a = __builtin_amdgcn_readlane(a, l);
                slot_b = __builtin_amdgcn_readlane(b, l);
                tiles = __builtin_amdgcn_readlane(n, l);
                first = before + __builtin_amdgcn_readlane(incl, l) - tiles;
                pad = pad_before + __builtin_amdgcn_readlane(pincl - nblk, l);
                break;
            }
            before += all;
            pad_before += __builtin_amdgcn_readlane(pincl, 63);
        }
    }
    const int local = item - first * ftiles;
    const int ft = FIRST ? local / tiles : local % ftiles, rt = FIRST ? local % tiles : local / ftiles;
    const int nbk = (slot_b - slot_a + 31) >> 5, bq = nbk / tiles, br = nbk - bq * tiles;     // rows and features are cut evenly
    const int b0 = rt * bq + min(rt, br), nb = bq + (rt < br ? 1 : 0);
    const int m0 = slot_a + 32 * b0, pb0 = pad + b0;
    const int fq = nfb / ftiles, fr = nfb - fq * ftiles, fb0 = ft * fq + min(ft, fr), width = fq + (ft < fr ? 1 : 0);
    const int blocks = g.R >> 5;

    // load side
    const char* wslot = (const char*)g.w + (size_t)g.phys[slot] * g.wstride;
    const size_t rowb = smoe_mx_row_bytes(g.R), rows_ = smoe_mx_row_scales(g.R);
    const uint32_t lane16 = lane * 16;
    constexpr int WN = WL ? WL : 1;
    const char* wsrc[WN];
    uint64_t wlanes[WN];
#pragma unroll
    for (int i = 0; i < WN; ++i) {
        const int f = FB == 2 ? wave >> 1 : WL * wave + i;
        wlanes[i] = f < width ? ~0ull : 1;                 // a block that is not there: one lane's load, so that the counts stay
        wsrc[i] = wslot + (size_t)(fb0 + min(f, width - 1)) * rowb;
    }
    const int sblk = FB == 8 ? 2 * wave + ((lane >> 4) & 1) : wave % FB;      // scales: 16 lanes a block
    const char* wscale = wslot + (size_t)nfb * rowb + (size_t)(fb0 + min(sblk, width - 1)) * rows_ + (lane & 15) * 16;
    const int unit = (lane & 3) ^ ((lane >> 3) & 3);       // rows of 64 bytes whose four units are permuted by (row / 2) % 4: of 16 lanes that read
                                                           // operands, two meet in each group of banks (4 cycles a read of the first product)
    const char *tsrc[2], *tscale = nullptr;                // FIRST: this lane's two rows of block `wave`; else a scalar base (tsrc[0])
    const uint64_t tlanes = wave < nb ? ~0ull : 1;
    const int bc = min(wave, nb - 1);
    if (FIRST) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int t = token_of_row(g, min(m0 + bc * 32 + h * 16 + (lane >> 2), slot_b - 1));
            tsrc[h] = (const char*)g.x + (size_t)t * g.R + unit * 16;
        }
        const int t = token_of_row(g, min(m0 + bc * 32 + (lane & 31), slot_b - 1));
        tscale = (const char*)g.xs + (size_t)t * g.pitch + (lane >> 5) * 4;
    } else {
        tsrc[0] = (const char*)g.x + (size_t)(pb0 + bc) * rowb;
        tscale = (const char*)g.xs + (size_t)(pb0 + bc) * rows_ + (lane & 15) * 16;
    }
    uint32_t lst = 0;
    auto issue = [&](int c) {                              // loads of step c into stage lst; past the last: one lane's, nowhere read
        const bool in = c < steps;
        if ((c & 3) == 0) {
            const uint32_t sc = S::SC + ((c >> 2) & 1) * S::SCG;
            const int gr = min(c >> 2, smoe_mx_groups(g.R) - 1);
            dma_16(wscale + (size_t)gr * 256, sc + (FB == 8 ? wave * 512 : wave % FB * 256), FB == 8 ? 0xffffffffull : 0xffffull);
            if (FIRST) dma_4(tscale + gr * 8, sc + FB * 256 + wave * 256);
            else dma_16(tscale + (size_t)gr * 256, sc + FB * 256 + wave * 256, 0xffffull);
        }
        const bool on = c + 1 < steps;                     // the next step's place
        if constexpr (FB == 2) {
            dma_16(wsrc[0] + (wave & 1) * 1024 + lane16, lst + wave * 1024, in ? wlanes[0] : 1);
            wsrc[0] += on ? MX_BLK : 0;
        } else {
#pragma unroll
            for (int i = 0; i < WL; ++i) {
                dma_2k(wsrc[i], lane16, lst + (WL * wave + i) * MX_BLK, in ? wlanes[i] : 1);
                wsrc[i] += on ? MX_BLK : 0;
            }
        }
        const uint32_t at = lst + (FB + wave) * MX_BLK;
        if (FIRST) {
            // a row that ends in the middle of the last step: its last 32 bytes again, which meet zeros
            const int back = c == steps - 1 && (g.R & 32) && unit >= 2 ? 32 : 0;
            dma_16(tsrc[0] - back, at, in ? tlanes : 1);
            dma_16(tsrc[1] - back, at + 1024, in ? tlanes : 1);
            tsrc[0] += on ? 64 : 0;
            tsrc[1] += on ? 64 : 0;
        } else {
            dma_2k(tsrc[0], lane16, at, in ? tlanes : 1);
            tsrc[0] += on ? MX_BLK : 0;
        }
        lst = lst == (ST - 1) * S::STAGE ? 0 : lst + S::STAGE;
    };

    f32x16 acc[AW][NBW];
#pragma unroll
    for (int a = 0; a < AW; ++a)
#pragma unroll
        for (int b = 0; b < NBW; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[a][b][i] = 0.f;
    uint32_t cst = 0;
    uint32_t ws[AW], ts[NBW];
    const uint32_t toff0 = FIRST ? (lane & 31) * 64 + (((lane >> 5) ^ ((lane >> 1) & 3)) * 16) : lane16;
    const uint32_t toff1 = FIRST ? (lane & 31) * 64 + (((2 + (lane >> 5)) ^ ((lane >> 1) & 3)) * 16) : lane16 + 1024;
    auto step = [&](auto uc, int c) {
        constexpr int u = decltype(uc)::value;
        if (u == 0) {
            const uint32_t sc = S::SC + ((c >> 2) & 1) * S::SCG;
#pragma unroll
            for (int a = 0; a < AW; ++a) ws[a] = *(const uint32_t*)(mx_lds + sc + (wf * AW + a) * 256 + lane * 4);
#pragma unroll
            for (int b = 0; b < NBW; ++b) {
                const char* p = mx_lds + sc + FB * 256 + (b * WT + wt) * 256;
                if (FIRST) {
                    const uint32_t x = *(const uint32_t*)(p + (lane & 31) * 4), y = *(const uint32_t*)(p + 128 + (lane & 31) * 4);
                    ts[b] = half_scales(make_uint2(x, y), blocks - (c >> 2) * 8);
                } else {
                    ts[b] = *(const uint32_t*)(p + lane * 4);
                }
            }
        }
        uint4 wv[AW][2], tv[NBW][2];
#pragma unroll
        for (int b = 0; b < NBW; ++b) {
            const char* p = mx_lds + cst + (FB + b * WT + wt) * MX_BLK;
            tv[b][0] = *(const uint4*)(p + toff0);
            tv[b][1] = *(const uint4*)(p + toff1);
        }
#pragma unroll
        for (int a = 0; a < AW; ++a) {
            const char* p = mx_lds + cst + (wf * AW + a) * MX_BLK + lane16;
            wv[a][0] = *(const uint4*)p;
            wv[a][1] = *(const uint4*)(p + 1024);
        }
#pragma unroll
        for (int a = 0; a < AW; ++a)
#pragma unroll
            for (int b = 0; b < NBW; ++b)
                if (b == 0 || b * WT + wt < nb)            // (without the branch, all products in a row: 99 us for 91)
                    smoe_mx_mfma<u>(acc[a][b], wv[a], tv[b], ws[a], ts[b]);
        cst = cst == (ST - 1) * S::STAGE ? 0 : cst + S::STAGE;
    };
    // Step c + 1 has landed: what may be outstanding are the loads of the ST - 2 steps behind it.
    auto landed = [&](auto uc) {
        constexpr int u = decltype(uc)::value;
        constexpr int younger = (ST - 2) * PER + group_starts(u + 2, u + ST) * NSC;
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");     // this wave's reads of the stage that is loaded next are done
        wait_vm<younger>();
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
#pragma unroll 1
    for (int c = 0; c < ST - 1; ++c) issue(c);
    landed(std::integral_constant<int, 3>{});              // step 0: behind it lie steps 1 .. ST - 2, none the first of a group
    for (int c = 0; c < steps; c += 4) {
        auto one = [&](auto uc) {
            constexpr int u = decltype(uc)::value;
            issue(c + u + ST - 1);
            if (c + u < steps) step(uc, c + u);
            landed(uc);
        };
        one(std::integral_constant<int, 0>{});
        one(std::integral_constant<int, 1>{});
        one(std::integral_constant<int, 2>{});
        one(std::integral_constant<int, 3>{});
    }
    wait_vm<0>();                                          // nothing is on its way to LDS when the next tile's loads, or the workgroup's end, come
    __builtin_amdgcn_s_barrier();
#pragma unroll
    for (int b = 0; b < NBW; ++b) {
        const int tb = b * WT + wt;
        if (tb >= nb) continue;
#pragma unroll
        for (int a = 0; a < AW; ++a) {
            if (wf * AW + a >= width) continue;
            if (FIRST) store_hidden(g, acc[a][b], pb0 + tb, fb0 + wf * AW + a);
            else store_rows(g, acc[a][b], m0 + tb * 32 + (lane & 31), m0 + tb * 32 + (lane & 31) < slot_b, (fb0 + wf * AW + a) * 32);
        }
    }
    }
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

template <bool FIRST, int NW, int BATCH, bool NT>
int launch_stream_as(const MxArgs& g, hipStream_t s, const hipEvent_t* e) {
    const size_t tiles = (size_t)(g.rows / 32 + std::min(g.nslots, g.rows));   // an upper bound of the sum of ceil(len / 32)
    smoe_launch_timed(stream_mx_kernel<FIRST, NW, BATCH, NT>, dim3((unsigned)(tiles * (g.N / 32))), dim3(64 * NW), s, e[0], e[1], g);
    return smoe_check_hip(hipGetLastError(), FIRST ? "smoe_expert_ffn_mx: first product launch" : "smoe_expert_ffn_mx: second product launch");
}

template <bool FIRST>
int launch_stream(const MxArgs& g, hipStream_t s, const hipEvent_t* e) {
    // Two waves to a feature block, of two steps a batch, for short reductions; four, of four steps, from 25 steps on, where a wave has more to ask for.
    // (us; 10 slots of 768 x 3072, 13 tokens: first product 7.4 with four steps a batch, 6.8 with two, 7.8 with four waves, and 13.8 with eight of four
    // steps; second product 7.0 with four waves of four steps, 7.2 of two, 8.0 with two waves, 7.7 with eight; 16 slots, 32 tokens: 12.5, 10.3, 12.3 and 21.8;
    // 10.5, 12.9, 10.2 and 13.2)
    if (smoe_mx_steps(g.R) <= 24) return g.past ? launch_stream_as<FIRST, 2, 2, true>(g, s, e) : launch_stream_as<FIRST, 2, 2, false>(g, s, e);
    return g.past ? launch_stream_as<FIRST, 4, 4, true>(g, s, e) : launch_stream_as<FIRST, 4, 4, false>(g, s, e);
}

template <bool FIRST, int FB, int ST>
int launch_tile(const MxArgs& g, hipStream_t s, const hipEvent_t* e) {
    static smoe_lds_raised raised;
    constexpr size_t lds = TileShape<FB, ST>::LDS;
    if (int rc = raised.ensure((const void*)tile_mx_kernel<FIRST, FB, ST>, lds, (int)lds)) return rc;
    smoe_launch_timed_lds(tile_mx_kernel<FIRST, FB, ST>, dim3(2 * g.cus), dim3(256), lds, s, e[0], e[1], g);
    return smoe_check_hip(hipGetLastError(), FIRST ? "smoe_expert_ffn_mx: first product launch" : "smoe_expert_ffn_mx: second product launch");
}

template <bool FIRST>
int launch_product(const MxArgs& g, hipStream_t s, const hipEvent_t* e) {
    switch (smoe_mx_form(g.rows, g.nslots, g.N)) {
        case 8: return launch_tile<FIRST, 8, 3>(g, s, e);
        case 4: return launch_tile<FIRST, 4, 3>(g, s, e);
        case 2: return launch_tile<FIRST, 2, 4>(g, s, e);
    }
    return launch_stream<FIRST>(g, s, e);
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
    g.cus = 256;                                               // of the whole GPU; a multiple of the 8 dies (tile_mx_kernel)
    g.past = smoe_weights_outgrow_cache(L);
    int rc = launch_product<true>(g, s, L->prof_ev);
    if (rc) return rc;
    g.x = h;
    g.xs = hs;
    g.w = (const uint8_t*)L->slot_w2;
    g.R = c.d_ff;
    g.N = c.d_model;
    return launch_product<false>(g, s, L->prof_ev + 2);
}
