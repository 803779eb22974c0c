// Gated delta-rule linear attention as a served layer runs it (paper: Background, Eq. 1-2): packed prompts and
// single tokens, bf16 in, states in a pool.  Per value head, K = V = 128, everything below in binary32 or better:
//
//   g_t = -exp(A_log) softplus(a_t + dt_bias),  alpha_t = exp(g_t),  beta_t = sigmoid(b_t)
//   S_t = alpha_t S_{t-1} + beta_t k_t (v_t - kappa_t S_{t-1}^T k_t)^T,      o_t = S_t^T q_t / sqrt(128)
//
// with kappa_t = 1 (Eq. 2) or alpha_t (the other common form: the prediction reads the decayed state), and q, k
// optionally divided by their length first.
#pragma once
#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include "../../include/nvfp4.h"
#include "ptx.cuh"

namespace nvfp4 {

constexpr int kGdnWidth = 128;          // key and value width of a head
constexpr float kGdnL2Eps = 1e-6f;
constexpr float kGdnQScale = 0.08838834764831845f;       // 1 / sqrt(128)

struct GdnParams {
    const uint16_t *q, *k, *v;          // bf16 [T, Hk, 128], [T, Hk, 128], [T, Hv, 128]; heads contiguous in a token
    int64_t ldq, ldk, ldv;              // token strides, in elements
    const void *a, *b;                  // gate pre-activations [T, Hv], bf16 or float
    int64_t lda, ldb;
    const float* A_log;                 // [Hv]
    const float* dt_bias;               // [Hv]
    const int32_t* cu;                  // [nseq + 1] token offsets; null: sequence i is token i (single-token form)
    const int32_t* slots;               // [nseq] state slot of a sequence; null: slot i
    const uint8_t* has_state;           // [nseq] 0: start from zero; null: every sequence continues
    float* state;                       // [nslots, Hv, 128 (k), 128 (v)]
    void* o;                            // bf16 or float [T, Hv, 128], token stride ldo
    int64_t ldo;
    int64_t nslots;
    int32_t T, nseq, Hk, Hv;
    uint32_t flags;
};

// tokens [begin, begin + len) of sequence i; offsets that are out of order or past T give shorter or empty
// sequences, never an access outside the arrays
__device__ __forceinline__ void gdn_sequence(const GdnParams& p, int i, int& begin, int& len) {
    if (p.cu == nullptr) { begin = i; len = 1; return; }
    const int b = min(max(p.cu[i], 0), p.T);
    const int e = min(max(p.cu[i + 1], b), p.T);
    begin = b;
    len = e - b;
}

// state slot of sequence i, or -1: a padding row, nothing of which is read or written
__device__ __forceinline__ int64_t gdn_slot(const GdnParams& p, int i) {
    const int64_t s = p.slots != nullptr ? static_cast<int64_t>(p.slots[i]) : static_cast<int64_t>(i);
    return (s >= 0 && s < p.nslots) ? s : -1;
}

__device__ __forceinline__ float gdn_gate_input(const void* base, int64_t at, uint32_t flags) {
    if ((flags & NVFP4_GDN_GATES_F32) != 0u) return __ldg(static_cast<const float*>(base) + at);
    return __uint_as_float(static_cast<uint32_t>(__ldg(static_cast<const uint16_t*>(base) + at)) << 16);
}

// log of the decay, <= 0.  Below -104 exp() is zero in binary32 anyway; the bound keeps sums of logs finite.
__device__ __forceinline__ float gdn_log_decay(float a, float A_log, float dt_bias) {
    const float x = a + dt_bias;
    const float sp = x > 20.0f ? x : log1pf(expf(x));
    const float g = -expf(A_log) * sp;
    return g < -104.0f ? -104.0f : g;                     // (a NaN stays a NaN)
}

__device__ __forceinline__ float gdn_sigmoid(float x) { return 1.0f / (1.0f + expf(-x)); }

__device__ __forceinline__ void gdn_store(void* o, int64_t at, float v, uint32_t flags) {
    if ((flags & NVFP4_OUT_F32) != 0u) static_cast<float*>(o)[at] = v;
    else static_cast<__nv_bfloat16*>(o)[at] = __float2bfloat16_rn(v);
}

// ------------------------------------------------------------------------------------------ single tokens
// Bound by the state: 64 KB read and written per (sequence, value head), everything else is small.  256 sequences of 48 heads:
// 248 us, 6.5 TB/s, the rate of a plain copy; 37 of 32: 29 us, 5.3 TB/s (20 us replayed on one pool, part of which stays in L2);
// one of 48: 4.2 us from memory, 3.3 us from L2, latency.  (A thread per state column
// with 128 values in registers, the form of the lockstep study, takes 347 us, 39 us and 28 us.)  A CTA of eight warps
// takes COLS columns of one head's state into registers in one go (a lane has float4 pieces of rows, coalesced), forms the
// prediction S^T k (each thread its rows, then across threads), updates its pieces, writes them back and forms S^T q the same
// way.  Three barriers; the loads of several CTAs per SM overlap each other's arithmetic and stores.
constexpr int kGdnDecodeThreads = 256;

template <int COLS>
__global__ void __launch_bounds__(kGdnDecodeThreads, COLS == 128 ? 3 : 4)
gdn_decode_kernel(const __grid_constant__ GdnParams p) {
    constexpr int LANES = COLS / 4;                     // lanes on one row
    constexpr int ROWS = 32 / LANES;                    // rows of a warp per pass
    constexpr int PASSES = kGdnWidth / (8 * ROWS);
    __shared__ __align__(16) float k_s[kGdnWidth], q_s[kGdnWidth];
    __shared__ __align__(16) float part[2][8][COLS];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int h = blockIdx.x / (kGdnWidth / COLS), c0 = (blockIdx.x % (kGdnWidth / COLS)) * COLS, seq = blockIdx.y;
    ptx::pdl_launch_dependents();
    ptx::pdl_wait();
    const int64_t slot = gdn_slot(p, seq);
    if (slot < 0) return;                               // a padding row
    const int hk = h / (p.Hv / p.Hk);
    const int col = (lane % LANES) * 4, row0 = warp * ROWS + lane / LANES;
    float* st = p.state + (slot * p.Hv + h) * (kGdnWidth * kGdnWidth) + static_cast<int64_t>(row0) * kGdnWidth + c0 + col;
    float4 S[PASSES];
#pragma unroll
    for (int i = 0; i < PASSES; ++i) S[i] = __ldcs(reinterpret_cast<const float4*>(st + i * (8 * ROWS) * kGdnWidth));
    const int64_t t = seq;
    const float alpha = expf(gdn_log_decay(gdn_gate_input(p.a, t * p.lda + h, p.flags), p.A_log[h], p.dt_bias[h]));
    const float beta = gdn_sigmoid(gdn_gate_input(p.b, t * p.ldb + h, p.flags));
    const uint2 vraw = __ldg(reinterpret_cast<const uint2*>(p.v + t * p.ldv + h * kGdnWidth + c0 + col));
    if (warp < 2) {
        // warp 0: the key, warp 1: the query; four elements a lane
        const uint16_t* src = warp == 0 ? p.k + t * p.ldk : p.q + t * p.ldq;
        const uint2 x = __ldg(reinterpret_cast<const uint2*>(src + hk * kGdnWidth + lane * 4));
        float4 f = make_float4(__uint_as_float(x.x << 16), __uint_as_float(x.x & 0xFFFF0000u), __uint_as_float(x.y << 16),
                               __uint_as_float(x.y & 0xFFFF0000u));
        float r = 1.0f;
        if ((p.flags & NVFP4_GDN_L2NORM) != 0u) {
            float ss = fmaf(f.x, f.x, fmaf(f.y, f.y, fmaf(f.z, f.z, f.w * f.w)));
#pragma unroll
            for (int off = 16; off >= 1; off >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, off);
            r = 1.0f / sqrtf(ss + kGdnL2Eps);
        }
        if (warp == 1) r *= kGdnQScale;
        float4* dst = reinterpret_cast<float4*>(warp == 0 ? k_s : q_s) + lane;
        *dst = make_float4(f.x * r, f.y * r, f.z * r, f.w * r);
    }
    __syncthreads();
    // sums over the rows: this thread's, the warp's (lanes on other rows), the CTA's
    auto reduce = [&](float4 x, int which) {
#pragma unroll
        for (int off = LANES; off < 32; off <<= 1) {
            x.x += __shfl_xor_sync(0xffffffffu, x.x, off);
            x.y += __shfl_xor_sync(0xffffffffu, x.y, off);
            x.z += __shfl_xor_sync(0xffffffffu, x.z, off);
            x.w += __shfl_xor_sync(0xffffffffu, x.w, off);
        }
        if (lane < LANES) *reinterpret_cast<float4*>(&part[which][warp][col]) = x;
    };
    float4 y = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
        const float kv = k_s[row0 + i * (8 * ROWS)];
        y.x = fmaf(S[i].x, kv, y.x);
        y.y = fmaf(S[i].y, kv, y.y);
        y.z = fmaf(S[i].z, kv, y.z);
        y.w = fmaf(S[i].w, kv, y.w);
    }
    reduce(y, 0);
    __syncthreads();
    float4 pred = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
    for (int w = 0; w < 8; ++w) {
        const float4 x = *reinterpret_cast<const float4*>(&part[0][w][col]);
        pred.x += x.x;
        pred.y += x.y;
        pred.z += x.z;
        pred.w += x.w;
    }
    const float kappa = (p.flags & NVFP4_GDN_DECAY_FIRST) != 0u ? alpha : 1.0f;
    const float4 u = make_float4(beta * (__uint_as_float(vraw.x << 16) - kappa * pred.x),
                                 beta * (__uint_as_float(vraw.x & 0xFFFF0000u) - kappa * pred.y),
                                 beta * (__uint_as_float(vraw.y << 16) - kappa * pred.z),
                                 beta * (__uint_as_float(vraw.y & 0xFFFF0000u) - kappa * pred.w));
    y = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
        const float kv = k_s[row0 + i * (8 * ROWS)], qv = q_s[row0 + i * (8 * ROWS)];
        S[i].x = fmaf(alpha, S[i].x, kv * u.x);
        S[i].y = fmaf(alpha, S[i].y, kv * u.y);
        S[i].z = fmaf(alpha, S[i].z, kv * u.z);
        S[i].w = fmaf(alpha, S[i].w, kv * u.w);
        __stcs(reinterpret_cast<float4*>(st + i * (8 * ROWS) * kGdnWidth), S[i]);
        y.x = fmaf(S[i].x, qv, y.x);
        y.y = fmaf(S[i].y, qv, y.y);
        y.z = fmaf(S[i].z, qv, y.z);
        y.w = fmaf(S[i].w, qv, y.w);
    }
    reduce(y, 1);
    __syncthreads();
    if (tid < COLS) {
        float o = 0.0f;
#pragma unroll
        for (int w = 0; w < 8; ++w) o += part[1][w][tid];
        gdn_store(p.o, t * p.ldo + h * kGdnWidth + c0 + tid, o, p.flags);
    }
}

}  // namespace nvfp4
