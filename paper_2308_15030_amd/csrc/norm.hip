// smoe_add_norm: residual addition and root-mean-square norm in front of the layer,
//     h = x + r,   total = h,   y = h / sqrt(mean(h^2) + eps) * weight,
// y in the layer's type and, or, in 8 bits with a scale for every 32 values (mx.h), the rows smoe_expert_ffn_mx takes.
//
// Memory bounds it: every input is read once and every output written once, because a row stays with its lanes between the sum of
// squares and the scaling: in registers up to 8192 columns (4.7 TB/s there).  Beyond, 16 waves hold it, and h and the residual together are all 128 registers
// that a lane may have, so 42 of them (bf16; fp32: 142) pass through scratch memory: 2.4 (1.9) TB/s at 16384 columns, 3.4 (2.9) at 65536.  A lane holds pieces of 8 consecutive values, W waves share a row, each with up to NP pieces a lane; a block of
// 32 values is four neighbouring lanes, so its largest magnitude takes two exchanges within a quad.  The sum x + r is used as it is in
// fp32, for the norm as for the rounding to `total`.

#include "mx.h"
#include "wave_ops.h"

namespace {

struct NormArgs {
    const void *x, *res;
    const float* weight;
    float eps;
    int T, d, pitch;
    void *total, *y;
    uint8_t *q, *qs;
};

// Eight values of a row; F32 rows end in the middle of a piece where d % 8 == 4.
template <bool F32>
__device__ __forceinline__ void load8(const void* p, size_t at, bool whole, float (&v)[8]) {
    if (F32) {
        const float4* f = (const float4*)((const float*)p + at);
        const float4 a = f[0], b = whole ? f[1] : make_float4(0, 0, 0, 0);
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
        v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    } else {
        const uint4 u = *(const uint4*)((const uint16_t*)p + at);
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(w[i] << 16);
            v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
        }
    }
}

template <bool F32>
__device__ __forceinline__ void store8(void* p, size_t at, bool whole, const float (&v)[8]) {
    if (F32) {
        float4* f = (float4*)((float*)p + at);
        f[0] = make_float4(v[0], v[1], v[2], v[3]);
        if (whole) f[1] = make_float4(v[4], v[5], v[6], v[7]);
    } else {
        *(uint4*)((uint16_t*)p + at) = make_uint4(smoe_pack_bf16(v[0], v[1]), smoe_pack_bf16(v[2], v[3]), smoe_pack_bf16(v[4], v[5]),
                                                  smoe_pack_bf16(v[6], v[7]));
    }
}

template <bool F32, int W, int NP>
__global__ __launch_bounds__(W > 4 ? 64 * W : 256) void add_norm_kernel(const NormArgs a) {
    constexpr int WAVES = W > 4 ? W : 4, ROWS = WAVES / W;     // rows of a workgroup
    __shared__ float s_sum[WAVES];
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    const int row = blockIdx.x * ROWS + wave / W;
    const bool live = row < a.T;
    const size_t r0 = (size_t)min(row, a.T - 1) * a.d;
    float h[NP][8], ss = 0.f;
#pragma unroll
    for (int p = 0; p < NP; ++p) {
        const int col = ((p * W + wave % W) * 64 + lane) * 8;
        if (col < a.d) load8<F32>(a.x, r0 + col, col + 4 < a.d, h[p]);
        else
#pragma unroll
            for (int i = 0; i < 8; ++i) h[p][i] = 0.f;
    }
    if (a.res) {
        float r[NP][8];
#pragma unroll
        for (int p = 0; p < NP; ++p) {
            const int col = ((p * W + wave % W) * 64 + lane) * 8;
            if (col < a.d) load8<F32>(a.res, r0 + col, col + 4 < a.d, r[p]);
            else
#pragma unroll
                for (int i = 0; i < 8; ++i) r[p][i] = 0.f;
        }
#pragma unroll
        for (int p = 0; p < NP; ++p)
#pragma unroll
            for (int i = 0; i < 8; ++i) h[p][i] += r[p][i];
    }
#pragma unroll
    for (int p = 0; p < NP; ++p)
#pragma unroll
        for (int i = 0; i < 8; ++i) ss = fmaf(h[p][i], h[p][i], ss);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) ss += __shfl_xor(ss, o);
    if (W > 1) {
        if (lane == 0) s_sum[wave] = ss;
        __syncthreads();
        ss = 0.f;
#pragma unroll
        for (int w = 0; w < W; ++w) ss += s_sum[wave / W * W + w];
    }
    // once a row in 64 bits: the 8-bit values flip at fewer borders the nearer this is (T = 16384, d = 1024: no change in time)
    const float scale = (float)(1.0 / sqrt((double)ss / a.d + a.eps));
#pragma unroll
    for (int p = 0; p < NP; ++p) {
        const int col = ((p * W + wave % W) * 64 + lane) * 8;
        const bool in = live && col < a.d, whole = col + 4 < a.d;
        if (in && a.total) store8<F32>(a.total, r0 + col, whole, h[p]);
        float y[8], amax = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = 0.f;
        if (in && (a.y || a.q)) {
            float w[8];
            load8<true>(a.weight, col, whole, w);
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = h[p][i] * scale * w[i];
            if (a.y) store8<F32>(a.y, r0 + col, whole, y);
        }
        if (a.q) {
#pragma unroll
            for (int i = 0; i < 8; ++i) amax = fmaxf(amax, fabsf(y[i]));
            amax = fmaxf(amax, __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(amax), 0xB1, 0xf, 0xf, true)));   // lanes 1 0 3 2 of a quad
            amax = fmaxf(amax, __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(amax), 0x4E, 0xf, 0xf, true)));   // lanes 2 3 0 1
            const uint32_t sc = smoe_mx_scale(amax);
            const float inv = smoe_mx_inverse(sc);
            if (in) {
                *(uint2*)(a.q + r0 + col) = make_uint2(smoe_mx_pack(y[0] * inv, y[1] * inv, y[2] * inv, y[3] * inv),
                                                       smoe_mx_pack(y[4] * inv, y[5] * inv, y[6] * inv, y[7] * inv));
            }
            // scale bytes of the row's blocks, and zeros up to the pitch
            if (live && (lane & 3) == 0 && col / 32 < a.pitch) a.qs[(size_t)row * a.pitch + col / 32] = col < a.d ? (uint8_t)sc : 0;
        }
    }
}

template <bool F32>
int launch(const NormArgs& a, hipStream_t s) {
#define SMOE_NORM(W, NP) hipLaunchKernelGGL((add_norm_kernel<F32, W, NP>), dim3((unsigned)((a.T + (W > 4 ? 1 : 4 / W) - 1) / (W > 4 ? 1 : 4 / W))), \
                                            dim3(W > 4 ? 64 * W : 256), 0, s, a)
    if (a.d <= 512) SMOE_NORM(1, 1);
    else if (a.d <= 1024) SMOE_NORM(1, 2);
    else if (a.d <= 2048) SMOE_NORM(1, 4);
    else if (a.d <= 8192) SMOE_NORM(4, 4);
    else SMOE_NORM(16, 8);
#undef SMOE_NORM
    return smoe_check_hip(hipGetLastError(), "smoe_add_norm launch");
}

}  // namespace

int smoe_launch_add_norm(const smoe_layer* L, const void* x, const void* residual, const float* weight, float eps, int T, void* total,
                         void* y, void* q, void* q_scale, hipStream_t s) {
    const smoe_config& c = L->cfg;
    const NormArgs a{x, residual, weight, eps, T, c.d_model, (int)smoe_scale_pitch(c.d_model), total, y,
                     (uint8_t*)q, (uint8_t*)q_scale};
    return c.dtype == SMOE_F32 ? launch<true>(a, s) : launch<false>(a, s);
}
