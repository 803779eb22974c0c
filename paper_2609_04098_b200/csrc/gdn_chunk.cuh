// The gated delta rule over packed prompts in chunks of 64 tokens (gdn.cuh states the recurrence).
//
// With G_i = g_1 + .. + g_i inside a chunk, E_i = G_{i-1} (kappa = 1) or G_i (kappa = alpha), and S the state in front of
// the chunk, the corrections u_i = beta_i (v_i - kappa_i S_{i-1}^T k_i) solve a unit lower triangular system:
//     (I + diag(beta) L) U = diag(beta) (V - diag(e^E) K S),      L_ij = e^{E_i - G_j} k_i . k_j   (j < i)
//     U = T R,   R = V - diag(e^E) K S,   T = (I + diag(beta) L)^-1 diag(beta)
//     O = diag(e^G) Q S + P U,            P_ij = e^{G_i - G_j} q_i . k_j                            (j <= i)
//     S <- e^{G_C} S + K^T diag(e^{G_C - G}) U
// T and P depend on no state: gdn_chunk_prepare_kernel computes them for all chunks in parallel.  What is serial is
// gdn_chunk_kernel, one CTA per (sequence, value head) walking the chunks with S in registers.
//
// What bounds it (B200, 16 key and 48 value heads).  One 8192-token prompt takes 578 us against 41 us for its bytes (32 KB a
// token) and about 70 us for its arithmetic: 128 chunks one after the other at 3.7 us alone (4.1 us with float output) and 4.3 us
// beside the preparation of the next range, of which the tensor cores work about a quarter -- the rest is the way of S, R and U
// out of accumulators, through a scale, a split and back (conversions and maxima, which share the schedulers, and six barrier
// hops).  16 prompts of 16001 tokens (float output): 640 us, 229 of them the preparation, against 124 us for their bytes.  Beside
// its chunks a CTA costs about 9 us (set-up 1, state 2, first tiles 2, last output 1, state out 1, next CTA 1.5); asking for the state in front
// of the set-up, for the first tiles in front of it, or storing the state in front of the last output all measured slower
// (up to 3 us a CTA: the two then share one burst of loads).  The same serial part on mma.sync with S
// in accumulator layout, 16 columns a warp, no barriers between the products, measured 437 us against 471 us for the single
// prompt (each head on two SMs) and 605 us against 460 us for the batch; a separate warpgroup for the output, sixteen compute
// warps instead of eight, and five preparation CTAs an SM instead of four (96 registers) all measured slower.
//
// Precision.  The products run on fp16 operands with binary32 accumulation.  An operand that is not a bf16 input is split into
// hi + lo fp16 (22 bits) after a power-of-two scale that puts its row's largest value at 2^12; keys and queries are exact in one
// fp16 (8 significant bits, scaled by a power of two per token; what is 2^-24 of a token's largest element or less flushes).
// Products keep hi*hi + hi*lo + lo*hi, those of the read-out too, whatever the output's type: where q.S and P U cancel, an
// operand rounded to 11 bits would show in front of bf16's own rounding (it would save 26 of the 578 us).  Against 64 bits a
// call is 7e-7 off where a binary32 evaluation is 3e-7 off.  The chunk's update is summed in a fresh accumulator and added to S
// with one rounded fma, so the tensor core's own rounding of running sums does not pile up over a long prompt.
#pragma once
#include <cstddef>
#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include "gdn.cuh"
#include "ptx.cuh"

namespace nvfp4 {

constexpr int kGdnChunk = 64;
constexpr int kGdnTileBytes = kGdnChunk * kGdnWidth * 2;          // fp16 [64][128]: keys or queries of a chunk
constexpr int kGdnSquareBytes = kGdnChunk * kGdnChunk * 2;        // fp16 [64][64]: one half of T or P
constexpr int kGdnVecBytes = 1024;                                // float c[64], d[64], w[64], gamma, and from kGdnVecT / kGdnVecP on
                                                                  // 1 / scale of the four blocks of 16 rows of T / P
constexpr int kGdnVecT = 196, kGdnVecP = 200;

// workspace behind the status block; chunk slots: sequence i uses slots begin_i / 64 + i and up (unique and in order
// because ceil(len / 64) <= (begin + len) / 64 - begin / 64 + 1), so no prefix sum over the sequences is needed
struct GdnWorkspace {
    uint8_t* kq;            // [slot][Hk][2][64 x 128 fp16], swizzled tiles
    uint8_t* tp;            // [slot][Hv][T hi | T lo | P hi | P lo | vec]
    uint32_t* status;
    uint64_t wait_limit_ns;
    // the chunks of every sequence that a launch handles: [chunk_begin, chunk_begin + chunk_count); 0: all of them
    int32_t chunk_begin, chunk_count;
    uint32_t sm_count;
};
constexpr int kGdnTpBytes = 4 * kGdnSquareBytes + kGdnVecBytes;

__device__ __forceinline__ int gdn_first_slot(const GdnParams& p, int seq) { return min(max(p.cu[seq], 0), p.T) / kGdnChunk + seq; }

// power of two that brings m to [2^target, 2^(target+1)), and its inverse; finite and exact for every m >= 0
__device__ __forceinline__ void gdn_pow2_scale(float m, int target, float& s, float& inv) {
    const int e = static_cast<int>(__float_as_uint(m) >> 23);             // biased exponent (sign bit is zero)
    const int se = min(254 + target - e, 253);
    s = __uint_as_float(static_cast<uint32_t>(se) << 23);
    inv = __uint_as_float(static_cast<uint32_t>(254 - se) << 23);
}

// two binary32 operations per instruction, each rounded like the scalar one: x * y, x * y + z
__device__ __forceinline__ void gdn_mul2(float& x0, float& x1, float y0, float y1) {
    asm("{\n\t.reg .b64 a, b;\n\tmov.b64 a, {%0, %1};\n\tmov.b64 b, {%2, %3};\n\tmul.rn.f32x2 a, a, b;\n\tmov.b64 {%0, %1}, a;\n\t}\n"
        : "+f"(x0), "+f"(x1) : "f"(y0), "f"(y1));
}
__device__ __forceinline__ void gdn_fma2(float& x0, float& x1, float y0, float y1, float z0, float z1) {
    asm("{\n\t.reg .b64 a, b, c;\n\tmov.b64 a, {%0, %1};\n\tmov.b64 b, {%2, %3};\n\tmov.b64 c, {%4, %5};\n\t"
        "fma.rn.f32x2 a, a, b, c;\n\tmov.b64 {%0, %1}, a;\n\t}\n"
        : "+f"(x0), "+f"(x1) : "f"(y0), "f"(y1), "f"(z0), "f"(z1));
}

// (x0, x1) * s = hi + lo, two fp16 each
__device__ __forceinline__ void gdn_split(float x0, float x1, float s, uint32_t& hi, uint32_t& lo) {
    gdn_mul2(x0, x1, s, s);
    const __half2 h = __floats2half2_rn(x0, x1);
    float2 f = __half22float2(h);
    gdn_fma2(f.x, f.y, -1.0f, -1.0f, x0, x1);
    const __half2 l = __floats2half2_rn(f.x, f.y);
    hi = *reinterpret_cast<const uint32_t*>(&h);
    lo = *reinterpret_cast<const uint32_t*>(&l);
}
__device__ __forceinline__ uint32_t gdn_half2(float a, float b) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}

// max(m, |a|, |b|) in one instruction
__device__ __forceinline__ float gdn_max_abs(float m, float a, float b) {
    float r;
    asm("max.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(m), "f"(a), "f"(b));
    return r;
}

// D += A B, one warp: A 16 x 16 (row g / g + 8 of lane 4 g + t), B 16 x 8, D 16 x 8 binary32
__device__ __forceinline__ void gdn_mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// four 8 x 8 matrices of 16-bit elements, row addresses from lanes 8 i .. 8 i + 7 for matrix i
__device__ __forceinline__ void gdn_ldsm(uint32_t addr, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
}
__device__ __forceinline__ void gdn_ldsm_t(uint32_t addr, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
}
// byte offset of 16-byte piece `c` of row `r`: a tile is two halves of 64 columns, rows of 128 bytes, 128-byte swizzle (what the
// tensor core's descriptors expect, and free of bank conflicts for ldmatrix); a square is one such half
__device__ __forceinline__ uint32_t gdn_tile_at(int r, int c) {
    return static_cast<uint32_t>((c >> 3) * (kGdnTileBytes / 2) + r * 128 + (((c & 7) ^ (r & 7)) << 4));
}
__device__ __forceinline__ uint32_t gdn_square_at(int r, int c) { return static_cast<uint32_t>(r * 128 + ((c ^ (r & 7)) << 4)); }

// ------------------------------------------------------------------------------------------ T and P of every chunk
// One CTA of four warps per (chunk slot, group of value heads that share a key head).  Warp w owns rows 16 w .. 16 w + 15
// of the two 64 x 64 squares, in accumulator layout.
//
// The decay factors e^{G_i - G_j} of the blocks left of a warp's diagonal block factor through the token in front of the
// warp's rows, r = 16 w - 1: e^{G_i - G_r} e^{G_r - G_j}, both at most 1 -- a handful of exponentials per lane instead of
// one per element; only the diagonal blocks need one per element.
//
// (I + A)^-1 of a unit lower triangular matrix by blocks of 16: the four diagonal blocks by forward substitution (a lane
// per column), then D_1 A_10 D_0 and D_3 A_32 D_2, then the 32 x 32 block below them -- all with the tensor cores on hi + lo
// fp16 splits scaled by each block's largest value.
constexpr int kGdnPrepThreads = 128;
constexpr int kGdnBlockBytes = 512;                       // one 16 x 16 fp16 block
struct GdnPrepSmem {
    alignas(128) uint8_t kt[kGdnTileBytes];
    alignas(128) uint8_t qt[kGdnTileBytes];
    alignas(128) uint8_t blk[9][2 * kGdnBlockBytes];      // hi | lo: D_0 .. D_3, T_10, X_20, X_21, X_30, X_31; the last four
                                                          // first hold the binary32 diagonal blocks
    alignas(16) float colf[4][48];
    alignas(16) float rowf[4][32];
    alignas(16) float inv[12];                            // 1 / scale of a block
    alignas(16) float rho[kGdnChunk], sig[kGdnChunk];
    struct Gates {
        alignas(16) float beta[kGdnChunk];
        alignas(16) float Gh[kGdnChunk], Gl[kGdnChunk], Eh[kGdnChunk], El[kGdnChunk];     // in units of log 2
    } gates[2];                                           // of this head and the next one
};

static_assert(offsetof(GdnPrepSmem, gates) % 16 == 0 && sizeof(GdnPrepSmem::Gates) % 16 == 0 && offsetof(GdnPrepSmem, colf) % 8 == 0, "read as float2");
static_assert(2 * kGdnBlockBytes == 16 * 16 * sizeof(float), "a diagonal block fits a split block's place");

__device__ __forceinline__ uint32_t gdn_block_at(int r, int c) { return static_cast<uint32_t>(r * 32 + ((c ^ ((r >> 2) & 1)) << 4)); }

// maximum over the warp of values >= 0 (their bit patterns are in order)
__device__ __forceinline__ float gdn_warp_max(float m) {
    return __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(m)));
}

// a 16 x 16 block in accumulator layout (two column tiles) as a split A operand; returns 1 / scale
__device__ __forceinline__ float gdn_split_block(const float (&x0)[4], const float (&x1)[4], uint32_t (&hi)[4], uint32_t (&lo)[4]) {
    float m = 0.0f;
#pragma unroll
    for (int e = 0; e < 4; ++e) m = gdn_max_abs(m, x0[e], x1[e]);
    float s, inv;
    gdn_pow2_scale(gdn_warp_max(m), 12, s, inv);
    gdn_split(x0[0], x0[1], s, hi[0], lo[0]);
    gdn_split(x0[2], x0[3], s, hi[1], lo[1]);
    gdn_split(x1[0], x1[1], s, hi[2], lo[2]);
    gdn_split(x1[2], x1[3], s, hi[3], lo[3]);
    return inv;
}
__device__ __forceinline__ void gdn_store_block(uint32_t blk, int lane, const uint32_t (&hi)[4], const uint32_t (&lo)[4]) {
    const uint32_t at = gdn_block_at((lane & 7) + ((lane >> 3) & 1) * 8, lane >> 4);
    asm volatile("stmatrix.sync.aligned.m8n8.x4.shared.b16 [%0], {%1, %2, %3, %4};"
                 ::"r"(blk + at), "r"(hi[0]), "r"(hi[1]), "r"(hi[2]), "r"(hi[3]) : "memory");
    asm volatile("stmatrix.sync.aligned.m8n8.x4.shared.b16 [%0], {%1, %2, %3, %4};"
                 ::"r"(blk + kGdnBlockBytes + at), "r"(lo[0]), "r"(lo[1]), "r"(lo[2]), "r"(lo[3]) : "memory");
}
// y += f (A B) with A split in registers, B a stored block
__device__ __forceinline__ void gdn_block_product(float (&y)[2][4], const uint32_t (&ah)[4], const uint32_t (&al)[4], uint32_t blk,
                                                  int lane, float f) {
    uint32_t bh[4], bl[4];
    const uint32_t at = gdn_block_at((lane & 7) + ((lane >> 3) & 1) * 8, lane >> 4);
    gdn_ldsm_t(blk + at, bh);
    gdn_ldsm_t(blk + kGdnBlockBytes + at, bl);
    float d[2][4] = {{0.0f, 0.0f, 0.0f, 0.0f}, {0.0f, 0.0f, 0.0f, 0.0f}};
    gdn_mma(d[0], al, bh[0], bh[1]);
    gdn_mma(d[1], al, bh[2], bh[3]);
    gdn_mma(d[0], ah, bl[0], bl[1]);
    gdn_mma(d[1], ah, bl[2], bl[3]);
    gdn_mma(d[0], ah, bh[0], bh[1]);
    gdn_mma(d[1], ah, bh[2], bh[3]);
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) y[t][e] = fmaf(d[t][e], f, y[t][e]);
}

__global__ void __launch_bounds__(kGdnPrepThreads, 4)
gdn_chunk_prepare_kernel(const __grid_constant__ GdnParams p, const __grid_constant__ GdnWorkspace w, int heads_per_cta) {
    extern __shared__ __align__(128) uint8_t prep_raw[];
    GdnPrepSmem& sm = *reinterpret_cast<GdnPrepSmem*>(prep_raw);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int h0 = blockIdx.y * heads_per_cta;
    ptx::pdl_launch_dependents();                           // (the serial kernel: it waits for this grid's end)
    int seq = 0, slot = blockIdx.x;
    if (w.chunk_count != 0) {                               // one range of chunks of every sequence
        seq = blockIdx.x / w.chunk_count;
        slot = gdn_first_slot(p, seq) + w.chunk_begin + static_cast<int>(blockIdx.x) % w.chunk_count;
    } else {                                                // all: the last sequence whose slots start at or in front of this one
        int hi = p.nseq - 1;
        while (seq < hi) {
            const int mid = (seq + hi + 1) >> 1;
            if (gdn_first_slot(p, mid) <= slot) seq = mid; else hi = mid - 1;
        }
    }
    int begin, len;
    gdn_sequence(p, seq, begin, len);
    const int first = (slot - gdn_first_slot(p, seq)) * kGdnChunk;
    // A later range may run under the serial kernel of the range in front of it (programmatic dependent launch; nothing here
    // depends on that kernel).  The serial kernel behind it waits for this grid only, so one CTA holds this grid's end back
    // until everything in front of it has ended.
    const bool last_out = w.chunk_begin > 0 && blockIdx.x == 0 && blockIdx.y == 0;
    if (first < 0 || first >= len || gdn_slot(p, seq) < 0) {
        if (last_out) ptx::pdl_wait();
        return;
    }
    const int tok0 = begin + first, n = min(kGdnChunk, len - first);
    const int rep = p.Hv / p.Hk, hk = h0 / rep;

    // ---- keys and queries: fp16 with a power-of-two scale per token; half a warp per row
    {
        const int half = tid >> 4, l = tid & 15;
        uint4 kr[8], qr[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int r = half + 8 * i;
            kr[i] = make_uint4(0u, 0u, 0u, 0u);
            qr[i] = kr[i];
            if (r < n) {
                const int64_t t = tok0 + r;
                kr[i] = __ldg(reinterpret_cast<const uint4*>(p.k + t * p.ldk + hk * kGdnWidth + l * 8));
                qr[i] = __ldg(reinterpret_cast<const uint4*>(p.q + t * p.ldq + hk * kGdnWidth + l * 8));
            }
        }
        auto convert = [&](const uint4& x, int r, uint8_t* tile, float* scale) {
            const uint32_t u[4] = {x.x, x.y, x.z, x.w};
            uint32_t m2 = 0u;                              // two running maxima of |x|, bf16
#pragma unroll
            for (int e = 0; e < 4; ++e) m2 = __vmaxu2(m2, u[e] & 0x7FFF7FFFu);
#pragma unroll
            for (int off = 8; off >= 1; off >>= 1) m2 = __vmaxu2(m2, __shfl_xor_sync(0xffffffffu, m2, off));
            float s, inv;
            gdn_pow2_scale(__uint_as_float(max(m2 << 16, m2 & 0xFFFF0000u)), 10, s, inv);
            uint32_t packed[4];
#pragma unroll
            for (int e = 0; e < 4; ++e)
                packed[e] = gdn_half2(__uint_as_float(u[e] << 16) * s, __uint_as_float(u[e] & 0xFFFF0000u) * s);
            *reinterpret_cast<uint4*>(tile + gdn_tile_at(r, l)) = make_uint4(packed[0], packed[1], packed[2], packed[3]);
            if (l == 0) scale[r] = s;
        };
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            convert(kr[i], half + 8 * i, sm.kt, sm.rho);
            convert(qr[i], half + 8 * i, sm.qt, sm.sig);
        }
    }
    const uint32_t kt_s = ptx::smem_u32(sm.kt), qt_s = ptx::smem_u32(sm.qt), blk_s = ptx::smem_u32(sm.blk);
    const int g8 = lane >> 2, t2 = (lane & 3) * 2, row0 = 16 * warp;
    const bool decay_first = (p.flags & NVFP4_GDN_DECAY_FIRST) != 0u;
    ptx::fence_proxy_async_smem();              // the tiles are read by bulk copies below
    __syncthreads();
    {
        // squared lengths of the scaled rows: the diagonals of K K^T and Q Q^T (an element in one lane each), in units of
        // the scale squared:  x / |x| = x s / sqrt(sum (x s)^2 + eps s^2), no overflow for large x
        float sq[2][2][4];
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) sq[x][t][e] = 0.0f;
        const int ar = row0 + (lane & 7) + ((lane >> 3) & 1) * 8, br = row0 + 8 * (lane >> 4) + (lane & 7);
#pragma unroll 2
        for (int c = 0; c < 8; ++c) {
            uint32_t a[4], b[4];
            gdn_ldsm(kt_s + gdn_tile_at(ar, 2 * c + (lane >> 4)), a);
            gdn_ldsm(kt_s + gdn_tile_at(br, 2 * c + ((lane >> 3) & 1)), b);
            gdn_mma(sq[0][0], a, b[0], b[1]);
            gdn_mma(sq[0][1], a, b[2], b[3]);
            gdn_ldsm(qt_s + gdn_tile_at(ar, 2 * c + (lane >> 4)), a);
            gdn_ldsm(qt_s + gdn_tile_at(br, 2 * c + ((lane >> 3) & 1)), b);
            gdn_mma(sq[1][0], a, b[0], b[1]);
            gdn_mma(sq[1][1], a, b[2], b[3]);
        }
        const bool l2 = (p.flags & NVFP4_GDN_L2NORM) != 0u;
        auto factor = [&](float* f, int r, float ss, float extra) {
            const float s = f[r];
            // from s = 2^48 on (a row below 2^-37) the sum, at most 2^29, is below 2^-47 of the epsilon and s * s may overflow
            const float length = s < 0x1p48f ? sqrtf(ss + kGdnL2Eps * s * s) : sqrtf(kGdnL2Eps) * s;
            f[r] = r < n ? extra * (1.0f / (l2 ? length : s)) : 0.0f;                                  // rows that are not there: 0
        };
        if ((g8 >> 1) == (lane & 3)) {                      // this lane holds the diagonal's rows g8 and g8 + 8
            const int odd = g8 & 1;
            factor(sm.rho, row0 + g8, odd ? sq[0][0][1] : sq[0][0][0], 1.0f);
            factor(sm.rho, row0 + g8 + 8, odd ? sq[0][1][3] : sq[0][1][2], 1.0f);
            factor(sm.sig, row0 + g8, odd ? sq[1][0][1] : sq[1][0][0], kGdnQScale);
            factor(sm.sig, row0 + g8 + 8, odd ? sq[1][1][3] : sq[1][1][2], kGdnQScale);
        }
    }

    // gate inputs of tokens 2 lane, 2 lane + 1 (warp 0, which has the least to do otherwise), a head ahead
    float ga[2] = {0.0f, 0.0f}, gb[2] = {0.0f, 0.0f}, gA = 0.0f, gd = 0.0f;
    auto load_gates = [&](int h) {
        gA = p.A_log[h];
        gd = p.dt_bias[h];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const int64_t t = tok0 + min(2 * lane + x, n - 1);
            ga[x] = gdn_gate_input(p.a, t * p.lda + h, p.flags);
            gb[x] = gdn_gate_input(p.b, t * p.ldb + h, p.flags);
        }
    };
    if (warp == 0) load_gates(h0);
    __syncthreads();                                        // lengths of keys and queries are in place, tiles complete
    if (h0 % rep == 0 && tid == 0) {                        // the first value head of a key head leaves the shared tiles behind
        uint8_t* dst = w.kq + (static_cast<int64_t>(slot) * p.Hk + hk) * (2 * kGdnTileBytes);
        ptx::bulk_store(dst, sm.kt, kGdnTileBytes);
        ptx::bulk_store(dst + kGdnTileBytes, sm.qt, kGdnTileBytes);
        ptx::bulk_commit_group();
    }

#pragma unroll 1
    for (int h = h0; h < h0 + heads_per_cta; ++h) {
        GdnPrepSmem::Gates& gt = sm.gates[h & 1];
        if (warp == 0) {
            // ---- gates: running sums of the logs (base 2) in binary64, kept as two binary32
            double g[2];
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const bool there = 2 * lane + x < n;
                g[x] = there ? 1.4426950408889634 * gdn_log_decay(ga[x], gA, gd) : 0.0;
                gt.beta[2 * lane + x] = there ? gdn_sigmoid(gb[x]) : 0.0f;
            }
            if (h + 1 < h0 + heads_per_cta) load_gates(h + 1);
            double sum = g[0] + g[1];
#pragma unroll
            for (int off = 1; off < 32; off <<= 1) {
                const double y = __shfl_up_sync(0xffffffffu, sum, off);
                if (lane >= off) sum += y;
            }
            const double G[2] = {sum - g[1], sum};
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const double E = decay_first ? G[x] : G[x] - g[x];
                const float Gh = static_cast<float>(G[x]), Eh = static_cast<float>(E);
                gt.Gh[2 * lane + x] = Gh;
                gt.Gl[2 * lane + x] = static_cast<float>(G[x] - static_cast<double>(Gh));
                gt.Eh[2 * lane + x] = Eh;
                gt.El[2 * lane + x] = static_cast<float>(E - static_cast<double>(Eh));
            }
        }
        // ---- K K^T and Q K^T, lower triangle, in one walk over K: the column tiles left of the diagonal block, of which a warp
        // has 0, 2, 4 or 6, and the diagonal block's two apart from them -- the same registers and the same code in every warp
        // (with tile numbers 2 w in the code each warp walks a copy of its own, and four copies do not fit the instruction cache)
        float kk[6][4], qk[6][4], kd[2][4], qd[2][4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
#pragma unroll
            for (int t = 0; t < 6; ++t) { kk[t][e] = 0.0f; qk[t][e] = 0.0f; }
            kd[0][e] = kd[1][e] = qd[0][e] = qd[1][e] = 0.0f;
        }
#pragma unroll 2
        for (int c = 0; c < 8; ++c) {
            uint32_t ak[4], aq[4], b[4];
            const uint32_t a_tile_at = gdn_tile_at(row0 + (lane & 7) + ((lane >> 3) & 1) * 8, 2 * c + (lane >> 4));
            gdn_ldsm(kt_s + a_tile_at, ak);
            gdn_ldsm(qt_s + a_tile_at, aq);
            gdn_ldsm(kt_s + gdn_tile_at(row0 + 8 * (lane >> 4) + (lane & 7), 2 * c + ((lane >> 3) & 1)), b);
            gdn_mma(kd[0], ak, b[0], b[1]);
            gdn_mma(kd[1], ak, b[2], b[3]);
            gdn_mma(qd[0], aq, b[0], b[1]);
            gdn_mma(qd[1], aq, b[2], b[3]);
#pragma unroll
            for (int t = 0; t < 6; t += 2) {
                if (t >= 2 * warp) break;
                gdn_ldsm(kt_s + gdn_tile_at(8 * (t + (lane >> 4)) + (lane & 7), 2 * c + ((lane >> 3) & 1)), b);
                gdn_mma(kk[t], ak, b[0], b[1]);
                gdn_mma(kk[t + 1], ak, b[2], b[3]);
                gdn_mma(qk[t], aq, b[0], b[1]);
                gdn_mma(qk[t + 1], aq, b[2], b[3]);
            }
        }
        __syncthreads();                                    // the gates are in place
        uint8_t* dst = w.tp + (static_cast<int64_t>(slot) * p.Hv + h) * kGdnTpBytes;
        float* const vec = reinterpret_cast<float*>(dst + 4 * kGdnSquareBytes);
        if (tid < kGdnChunk) {
            const float Gc = gt.Gh[kGdnChunk - 1];
            vec[tid] = exp2f(gt.Eh[tid]) * sm.rho[tid];
            vec[kGdnChunk + tid] = exp2f(gt.Gh[tid]) * sm.sig[tid];
            vec[2 * kGdnChunk + tid] = exp2f((Gc - gt.Gh[tid]) + (gt.Gl[kGdnChunk - 1] - gt.Gl[tid])) * sm.rho[tid];
            if (tid == 0) vec[3 * kGdnChunk] = exp2f(Gc);
        }
        if (warp > 0) {
            const float rh = gt.Gh[row0 - 1], rl = gt.Gl[row0 - 1];
            const int i = row0 + (lane & 15);
            sm.rowf[warp][lane] = lane < 16 ? exp2f((gt.Eh[i] - rh) + (gt.El[i] - rl)) * sm.rho[i] * gt.beta[i]
                                            : exp2f((gt.Gh[i] - rh) + (gt.Gl[i] - rl)) * sm.sig[i];
            for (int j = lane; j < row0; j += 32) sm.colf[warp][j] = exp2f((rh - gt.Gh[j]) + (rl - gt.Gl[j])) * sm.rho[j];
            __syncwarp();
        }
        // the factors of this lane's elements; the diagonal block's one by one
        auto decays = [&](float (&acc)[6][4], float (&diag)[2][4], bool square) {           // square: A (strictly lower), else P
            const float f0 = sm.rowf[warp][(square ? 0 : 16) + g8], f1 = sm.rowf[warp][(square ? 0 : 16) + g8 + 8];
#pragma unroll
            for (int t = 0; t < 6; ++t) {
                if (t >= 2 * warp) break;
                const float2 cf = *reinterpret_cast<const float2*>(&sm.colf[warp][8 * t + t2]);
                acc[t][0] *= f0 * cf.x;
                acc[t][1] *= f0 * cf.y;
                acc[t][2] *= f1 * cf.x;
                acc[t][3] *= f1 * cf.y;
            }
            float rh[2], rl[2], rf[2];                          // of this lane's two rows: the exponent's part, the factor
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const int i = row0 + g8 + 8 * x;
                rh[x] = square ? gt.Eh[i] : gt.Gh[i];
                rl[x] = square ? gt.El[i] : gt.Gl[i];
                rf[x] = square ? sm.rho[i] * gt.beta[i] : sm.sig[i];
            }
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const float2 jh = *reinterpret_cast<const float2*>(&gt.Gh[row0 + 8 * t + t2]);
                const float2 jl = *reinterpret_cast<const float2*>(&gt.Gl[row0 + 8 * t + t2]);
                const float2 jr = *reinterpret_cast<const float2*>(&sm.rho[row0 + 8 * t + t2]);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int i = g8 + (e >> 1) * 8, j = 8 * t + t2 + (e & 1);
                    const float d = (rh[e >> 1] - ((e & 1) ? jh.y : jh.x)) + (rl[e >> 1] - ((e & 1) ? jl.y : jl.x));
                    diag[t][e] = (square ? j < i : j <= i) ? diag[t][e] * (rf[e >> 1] * ((e & 1) ? jr.y : jr.x)) * exp2f(d) : 0.0f;
                }
            }
        };
        // a strip, split, to the chunk's squares: blocks on and below the diagonal only (nothing reads the others), each block
        // of 16 rows with its own scale
        auto store_strip = [&](const float (&x)[6][4], const float (&diag)[2][4], uint8_t* to, float* inv_at) {
            float m = 0.0f;
#pragma unroll
            for (int e = 0; e < 4; e += 2) m = gdn_max_abs(gdn_max_abs(m, diag[0][e], diag[0][e + 1]), diag[1][e], diag[1][e + 1]);
#pragma unroll
            for (int t = 0; t < 6; ++t) {
                if (t >= 2 * warp) break;
#pragma unroll
                for (int e = 0; e < 4; e += 2) m = gdn_max_abs(m, x[t][e], x[t][e + 1]);
            }
            float sc, inv;
            gdn_pow2_scale(gdn_warp_max(m), 12, sc, inv);
            if (lane == 0) inv_at[warp] = inv;
            auto store_tile = [&](const float (&v)[4], int column_tile) {
#pragma unroll
                for (int e = 0; e < 4; e += 2) {
                    uint8_t* at = to + gdn_square_at(row0 + g8 + (e >> 1) * 8, column_tile) + t2 * 2;
                    uint32_t vh, vl;
                    gdn_split(v[e], v[e + 1], sc, vh, vl);
                    *reinterpret_cast<uint32_t*>(at) = vh;
                    *reinterpret_cast<uint32_t*>(at + kGdnSquareBytes) = vl;
                }
            };
            store_tile(diag[0], 2 * warp);
            store_tile(diag[1], 2 * warp + 1);
#pragma unroll
            for (int t = 0; t < 6; ++t) {
                if (t >= 2 * warp) break;
                store_tile(x[t], t);
            }
        };
        decays(qk, qd, false);
        store_strip(qk, qd, dst + 2 * kGdnSquareBytes, vec + kGdnVecP);
        decays(kk, kd, true);
        // ---- D_w: lanes 0..15 and 16..31 both walk the block's columns; the first half stores hi, the second lo
        float T[6][4], Td[2][4];
        {
            float* dg = reinterpret_cast<float*>(sm.blk[5 + warp]);
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) dg[(g8 + (e >> 1) * 8) * 16 + 8 * t + t2 + (e & 1)] = kd[t][e];
            __syncwarp();
            const int col = lane & 15;
            float x[16], m = 0.0f;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                float acc0 = i == col ? 1.0f : 0.0f, acc1 = 0.0f;
#pragma unroll
                for (int m4 = 0; m4 < (i + 3) / 4; ++m4) {
                    const float4 a = *reinterpret_cast<const float4*>(dg + i * 16 + 4 * m4);
                    const float av[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        if (4 * m4 + e >= i) continue;
                        if (e & 1) acc1 = fmaf(-av[e], x[4 * m4 + e], acc1); else acc0 = fmaf(-av[e], x[4 * m4 + e], acc0);
                    }
                }
                x[i] = acc0 + acc1;
                m = fmaxf(m, fabsf(x[i]));
            }
            float s, inv;
            gdn_pow2_scale(gdn_warp_max(m), 12, s, inv);
            if (lane == 0) sm.inv[warp] = inv;
            __syncwarp();                                   // the block has been read
            uint8_t* dst = sm.blk[warp] + (lane >> 4) * kGdnBlockBytes + (col & 7) * 2;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const float v = x[i] * s;
                const __half vh = __float2half_rn(v);
                *reinterpret_cast<__half*>(dst + gdn_block_at(i, col >> 3)) = lane < 16 ? vh : __float2half_rn(v - __half2float(vh));
                if (lane < 16) dg[i * 16 + col] = x[i];
            }
            __syncwarp();
#pragma unroll
            for (int e = 0; e < 4; ++e) {
#pragma unroll
                for (int t = 0; t < 6; ++t) T[t][e] = 0.0f;
#pragma unroll
                for (int t = 0; t < 2; ++t) Td[t][e] = dg[(g8 + (e >> 1) * 8) * 16 + 8 * t + t2 + (e & 1)];
            }
        }
        __syncthreads();
        const uint32_t a_at = gdn_block_at((lane & 7) + ((lane >> 3) & 1) * 8, lane >> 4);
        // T_{w j} tiles of this warp's row block <- -(D_w X), X a stored block; m is the index of D_w
        auto from_left = [&](float (&y)[2][4], int m, int xblk) {
            uint32_t dh[4], dl[4];
            gdn_ldsm(blk_s + m * (2 * kGdnBlockBytes) + a_at, dh);
            gdn_ldsm(blk_s + m * (2 * kGdnBlockBytes) + kGdnBlockBytes + a_at, dl);
            gdn_block_product(y, dh, dl, blk_s + xblk * (2 * kGdnBlockBytes), lane, -sm.inv[m] * sm.inv[xblk]);
        };
        auto store_split = [&](const float (&x)[2][4], int blk) {
            uint32_t xh[4], xl[4];
            const float inv = gdn_split_block(x[0], x[1], xh, xl);
            gdn_store_block(blk_s + blk * (2 * kGdnBlockBytes), lane, xh, xl);
            if (lane == 0) sm.inv[blk] = inv;
            __syncwarp();
        };
        // level 1: T_10 and T_32
        if (warp & 1) {
            uint32_t ah[4], al[4];
            float a0[4], a1[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) { a0[e] = warp == 1 ? kk[0][e] : kk[4][e]; a1[e] = warp == 1 ? kk[1][e] : kk[5][e]; }
            const float ia = gdn_split_block(a0, a1, ah, al);
            float x[2][4] = {{0.0f, 0.0f, 0.0f, 0.0f}, {0.0f, 0.0f, 0.0f, 0.0f}};
            gdn_block_product(x, ah, al, blk_s + (warp - 1) * (2 * kGdnBlockBytes), lane, ia * sm.inv[warp - 1]);
            const int xb = warp == 1 ? 5 : 7;               // (X_20 and X_30 come later)
            store_split(x, xb);
            float y[2][4] = {{0.0f, 0.0f, 0.0f, 0.0f}, {0.0f, 0.0f, 0.0f, 0.0f}};
            from_left(y, warp, xb);
            if (warp == 1) store_split(y, 4);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (warp == 1) { T[0][e] = y[0][e]; T[1][e] = y[1][e]; }
                else           { T[4][e] = y[0][e]; T[5][e] = y[1][e]; }
            }
        }
        __syncthreads();
        // level 2: X_w0 = A_w0 D_0 + A_w1 T_10, X_w1 = A_w1 D_1 for w = 2, 3
        if (warp >= 2) {
            uint32_t ah[4], al[4], ch[4], cl[4];
            const float ia = gdn_split_block(kk[0], kk[1], ah, al), ic = gdn_split_block(kk[2], kk[3], ch, cl);
            float x[2][4] = {{0.0f, 0.0f, 0.0f, 0.0f}, {0.0f, 0.0f, 0.0f, 0.0f}};
            gdn_block_product(x, ah, al, blk_s, lane, ia * sm.inv[0]);
            gdn_block_product(x, ch, cl, blk_s + 4 * (2 * kGdnBlockBytes), lane, ic * sm.inv[4]);
            store_split(x, warp == 2 ? 5 : 7);
            float z[2][4] = {{0.0f, 0.0f, 0.0f, 0.0f}, {0.0f, 0.0f, 0.0f, 0.0f}};
            gdn_block_product(z, ch, cl, blk_s + 1 * (2 * kGdnBlockBytes), lane, ic * sm.inv[1]);
            store_split(z, warp == 2 ? 6 : 8);
        }
        __syncthreads();
        if (warp >= 2) {
            float y[2][4] = {{0.0f, 0.0f, 0.0f, 0.0f}, {0.0f, 0.0f, 0.0f, 0.0f}};
            float z[2][4] = {{0.0f, 0.0f, 0.0f, 0.0f}, {0.0f, 0.0f, 0.0f, 0.0f}};
            from_left(y, warp, warp == 2 ? 5 : 7);
            from_left(z, warp, warp == 2 ? 6 : 8);
            if (warp == 3) {                                // - T_32 X_2j
                uint32_t th[4], tl[4];
                const float it = gdn_split_block(T[4], T[5], th, tl);
                gdn_block_product(y, th, tl, blk_s + 5 * (2 * kGdnBlockBytes), lane, -it * sm.inv[5]);
                gdn_block_product(z, th, tl, blk_s + 6 * (2 * kGdnBlockBytes), lane, -it * sm.inv[6]);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) { T[0][e] = y[0][e]; T[1][e] = y[1][e]; T[2][e] = z[0][e]; T[3][e] = z[1][e]; }
        }
        // T = (I + A)^-1 diag(beta)
        auto times_beta = [&](float (&v)[4], int column_tile) {
            const float2 b = *reinterpret_cast<const float2*>(&gt.beta[8 * column_tile + t2]);
            gdn_mul2(v[0], v[1], b.x, b.y);
            gdn_mul2(v[2], v[3], b.x, b.y);
        };
        times_beta(Td[0], 2 * warp);
        times_beta(Td[1], 2 * warp + 1);
#pragma unroll
        for (int t = 0; t < 6; ++t) {
            if (t >= 2 * warp) break;
            times_beta(T[t], t);
        }
        store_strip(T, Td, dst, vec + kGdnVecT);
    }
    if (tid == 0) ptx::bulk_wait_group_read<0>();
    if (last_out) ptx::pdl_wait();
}

// ------------------------------------------------------------------------------------------ the serial part
// One CTA per (sequence, value head), 384 threads.  Everything of a chunk is a product with the 128 value columns of the head as
// M: the tensor core's A operand is S^T, R^T or U^T, written to tensor memory by the threads that own its rows and read from
// there; B operands are the chunk's tiles in shared memory (K both ways: rows of K as columns of B, and, for the update, B = K
// with its tokens as the contraction).
//   warps 0-7   compute; thread = one value column (TMEM lane), warps 0-3 and 4-7 half of the other index each.  S stays in
//               registers (64 binary32 a thread), its split copy goes to TMEM once a chunk; R and U are formed from an
//               accumulator and written back split; O leaves in two steps beside the next chunk's products.  The scale of a
//               split row is the largest value of both halves, exchanged between the two warps that share 32 rows.
//   warp 8      issues the MMAs of a chunk in four groups behind the barriers below (warp-convergent, one predicated lane)
//   warp 9      brings the next chunk's tiles (bulk copies) and V (a bulk copy per token)
// TMEM columns (all 512): S hi, S lo, X -> R hi | lo -> U hi | lo for the read-out, Q S, U -> U w hi | lo, U P, update.
// Every wait is bounded; a warp that gives up raises the abort flag and goes on through the barriers of its chunk, so that
// nobody waits for it, and the pairs leave the loop together.
template <bool F32>
struct GdnChunkCfg {
    static constexpr int STAGES = 2;
    static constexpr int TP_BYTES = kGdnTpBytes;
    static constexpr int V_BYTES = kGdnChunk * kGdnWidth * 2;
    static constexpr int KQ_OFF = 0;                                   // 1024-byte aligned, as T and P behind it
    static constexpr int TP_OFF = 2 * kGdnTileBytes;
    static constexpr int VEC_OFF = TP_OFF + TP_BYTES - kGdnVecBytes;
    static constexpr int V_OFF = TP_OFF + TP_BYTES;
    static constexpr int STAGE_BYTES = V_OFF + V_BYTES;
    static constexpr int MAX_BYTES = 4 * 2 * kGdnWidth * 4;            // [exchange][half][row]
    static constexpr int SIDE_BYTES = 8 * 2 * 36 * 4;                  // of a compute warp, by chunk parity: d of its tokens, 1 / scale(P)
    static constexpr int OUT_BYTES = F32 ? 0 : 8 * 16 * 64;            // bf16 [16 tokens][32 columns] of a compute warp
    static constexpr int SMEM_BYTES = 1024 + STAGES * STAGE_BYTES + MAX_BYTES + SIDE_BYTES + OUT_BYTES + 16 * 8 + 16;
    static_assert(STAGE_BYTES % 1024 == 0 && TP_OFF % 1024 == 0, "swizzled tiles start on 1024 bytes");
    static_assert(SMEM_BYTES <= 232448 && SMEM_BYTES > 116 * 1024, "one CTA per SM: it takes all of TMEM");
};
constexpr int kGdnChunkThreads = 384;
constexpr uint32_t kTmSh = 0, kTmSl = 64, kTmX = 128, kTmQ = 192, kTmU = 256, kTmY = 320, kTmD = 384;

// A operand [128 x 16] fp16 at TMEM address `a`, B from shared memory; issued by the lane whose `pred` is set
__device__ __forceinline__ void gdn_mma_ts(uint32_t d, uint32_t a, uint32_t b_lo, uint32_t b_hi, uint32_t idesc, uint32_t accumulate, uint32_t pred) {
    asm volatile(
        "{\n\t"
        ".reg .pred p, q;\n\t"
        ".reg .b64 b;\n\t"
        "mov.b64 b, {%2, %3};\n\t"
        "setp.ne.b32 p, %5, 0;\n\t"
        "setp.ne.b32 q, %6, 0;\n\t"
        "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %4, p;\n\t"
        "}\n"
        ::"r"(d), "r"(a), "r"(b_lo), "r"(b_hi), "r"(idesc), "r"(accumulate), "r"(pred)
        : "memory");
}
// barrier of THREADS threads; true where all of them pass true
template <int THREADS>
__device__ __forceinline__ bool gdn_and_barrier(int id, bool ok) {
    uint32_t r;
    asm volatile(
        "{\n\t"
        ".reg .pred p, q;\n\t"
        "setp.ne.b32 p, %2, 0;\n\t"
        "barrier.cta.red.and.pred q, %1, %3, p;\n\t"
        "selp.u32 %0, 1, 0, q;\n\t"
        "}\n"
        : "=r"(r) : "r"(id), "r"(static_cast<uint32_t>(ok)), "n"(THREADS) : "memory");
    return r != 0u;
}

template <bool F32>
__global__ void __launch_bounds__(kGdnChunkThreads, 1)
gdn_chunk_kernel(const __grid_constant__ GdnParams p, const __grid_constant__ GdnWorkspace w) {
    using C = GdnChunkCfg<F32>;
    extern __shared__ uint8_t chunk_raw[];
    uint8_t* const smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(chunk_raw) + 1023) & ~uintptr_t(1023));
    float* const mx = reinterpret_cast<float*>(smem + C::STAGES * C::STAGE_BYTES);
    float* const side = mx + C::MAX_BYTES / 4;
    uint8_t* const out_s = reinterpret_cast<uint8_t*>(side) + C::SIDE_BYTES;
    uint64_t* const bars = reinterpret_cast<uint64_t*>(out_s + C::OUT_BYTES);
    uint64_t* const full = bars;                         // a stage's tiles have landed
    uint64_t* const empty = bars + C::STAGES;            // the MMAs and the compute warps are done with a stage
    uint64_t* const s_ready = bars + 2 * C::STAGES;      // S is in TMEM (8 warps)
    uint64_t* const r_ready = s_ready + 1;
    uint64_t* const u_ready = s_ready + 2;
    uint64_t* const x_full = s_ready + 3;                // accumulators complete
    uint64_t* const u_full = s_ready + 4;
    uint64_t* const y_full = s_ready + 5;
    uint64_t* const d_full = s_ready + 6;
    uint64_t* const o_done = s_ready + 7;                // a chunk's read-out products are in registers (8 warps)
    uint64_t* const drain = s_ready + 8;
    uint32_t* const tmem_slot = reinterpret_cast<uint32_t*>(s_ready + 9);
    volatile uint32_t* const abort_flag = tmem_slot + 1;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int h = blockIdx.x;
    int seq = blockIdx.y, begin, len;
    if (gridDim.x * gridDim.y > w.sm_count && gridDim.y <= 32) {
        // More CTAs than SMs: CTAs start in the order of their index, so the longest sequence goes first and short ones fill the
        // end.  Lane i counts the sequences in front of sequence i.  16 sequences of 100 to 1540 tokens in ascending order, 48 heads:
        // 543 us in that order, 506 us so; six of 200 and one of 2000 behind them: 235 and 194 us.  More than 32 sequences, one
        // more than a lane each, start in the caller's order, and a long one behind them waits: 40 of 64 tokens and one of 8192
        // take 802 us with the long one last and 668 us with it first.
        const int mine = static_cast<int>(lane);
        begin = 0;
        len = -1;
        if (mine < p.nseq) gdn_sequence(p, mine, begin, len);
        int rank = 0;
        for (int j = 0; j < p.nseq; ++j) {
            const int other = __shfl_sync(0xffffffffu, len, j);
            rank += (other > len || (other == len && j < mine)) ? 1 : 0;
        }
        seq = __ffs(static_cast<int>(__ballot_sync(0xffffffffu, mine < p.nseq && rank == seq))) - 1;
    }
    const int64_t sslot = gdn_slot(p, seq);
    gdn_sequence(p, seq, begin, len);
    const bool fresh = w.chunk_begin == 0 && p.has_state != nullptr && p.has_state[seq] == 0;
    // chunks of this launch; the pointers below start at its first one
    const int all = (len + kGdnChunk - 1) / kGdnChunk;
    const int chunks = w.chunk_count != 0 ? min(all - w.chunk_begin, w.chunk_count) : all;
    if (sslot < 0 || (len == 0 && !fresh) || (w.chunk_begin > 0 && chunks <= 0)) {
        ptx::pdl_wait();                                         // (nothing behind this grid starts before its preparation ended)
        return;
    }
    const int slot0 = gdn_first_slot(p, seq) + w.chunk_begin;
    begin += w.chunk_begin * kGdnChunk;
    len -= w.chunk_begin * kGdnChunk;

    if (tid == 0) {
        for (int s = 0; s < C::STAGES; ++s) {
            ptx::mbar_init(&full[s], 1);
            ptx::mbar_init(&empty[s], 9);                        // eight compute warps and the MMAs' commit
        }
        for (int i = 0; i < 3; ++i) ptx::mbar_init(&s_ready[i], 8);
        for (int i = 3; i < 7; ++i) ptx::mbar_init(&s_ready[i], 1);
        ptx::mbar_init(o_done, 8);
        ptx::mbar_init(drain, 1);
        *abort_flag = 0u;
        ptx::fence_barrier_init();
    }
    if (warp == 8) {
        ptx::tmem_alloc(tmem_slot, 512);
        ptx::tmem_relinquish();
    }
    ptx::tc_fence_before();
    __syncthreads();
    ptx::tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    // 384 threads start with 168 registers each.  The warpgroup of the loads and the MMAs (two of its warps have nothing to do)
    // keeps 104, the two of the compute warps take 200: 128 * (104 + 2 * 200) = 384 * 168, what the CTA was launched with.
    if (warp >= 8) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 104;");
    if (warp == 9) {
        // ------------------------------------------------------------ loads
        // This kernel starts under the tail of the preparation (programmatic dependent launch); what that wrote is read by this
        // warp's copies alone.  The preparation of the next range of chunks may start now.
        ptx::pdl_wait();
        ptx::pdl_launch_dependents();
        const int hk = h / (p.Hv / p.Hk);
        const uint8_t* kq_src = w.kq + (static_cast<int64_t>(slot0) * p.Hk + hk) * (2 * kGdnTileBytes);
        const uint8_t* tp_src = w.tp + (static_cast<int64_t>(slot0) * p.Hv + h) * C::TP_BYTES;
        int c = 0;
        for (; c < chunks; ++c) {
            const int s = c & 1;
            bool ok = true;
            if (lane == 0 && c >= C::STAGES) ok = ptx::mbar_wait_bounded(&empty[s], static_cast<uint32_t>(c / C::STAGES - 1) & 1u, abort_flag, w.wait_limit_ns);
            if (__shfl_sync(0xffffffffu, static_cast<int>(ok), 0) == 0) break;
            uint8_t* st = smem + s * C::STAGE_BYTES;
            const int n = min(kGdnChunk, len - c * kGdnChunk);
            if (lane == 0) {
                ptx::mbar_arrive_expect_tx(&full[s], 2 * kGdnTileBytes + C::TP_BYTES + n * 256);
                ptx::bulk_load(st + C::KQ_OFF, kq_src + static_cast<int64_t>(c) * p.Hk * (2 * kGdnTileBytes), 2 * kGdnTileBytes, &full[s]);
                ptx::bulk_load(st + C::TP_OFF, tp_src + static_cast<int64_t>(c) * p.Hv * C::TP_BYTES, C::TP_BYTES, &full[s]);
            }
            __syncwarp();
            const uint16_t* v = p.v + static_cast<int64_t>(begin + c * kGdnChunk) * p.ldv + h * kGdnWidth;
            for (int i = lane; i < n; i += 32) ptx::bulk_load(st + C::V_OFF + i * 256, v + i * p.ldv, 256, &full[s]);
        }
        if (c < chunks) {
            // gave up: a bounded chance for what is in flight to land before the CTA goes
            for (int i = max(0, c - C::STAGES); i < c; ++i)
                for (int spin = 0; spin < 4096 && !ptx::mbar_try_wait(&full[i & 1], static_cast<uint32_t>(i / C::STAGES) & 1u); ++spin) {}
        }
    } else if (warp == 8) {
        // ------------------------------------------------------------ MMAs
        const uint32_t lp = ptx::elect_one() ? 1u : 0u;
        constexpr uint32_t kIdesc = (1u << 4) | (8u << 24);                               // binary32 += fp16 x fp16, M = 128
        constexpr uint32_t kN64 = kIdesc | (8u << 17), kN128T = kIdesc | (16u << 17) | (1u << 16);   // (B by columns)
        // descriptor words: 128-byte swizzle, 1024 bytes between groups of eight rows; by columns also the distance of the
        // 64-column halves of K
        constexpr uint32_t kHi = (1024u >> 4) | (1u << 14) | (2u << 29);
        constexpr uint32_t kLo = 1u << 16, kLoT = (kGdnTileBytes / 2 >> 4) << 16;
        bool ok = true;
        for (int c = 0; ok && c < chunks; ++c) {
            const uint32_t s = static_cast<uint32_t>(c & 1), ph = static_cast<uint32_t>(c) & 1u;
            const uint32_t st = ((ptx::smem_u32(smem) + s * C::STAGE_BYTES) & 0x3FFFFu) >> 4;
            const uint32_t k_d = st, q_d = st + (kGdnTileBytes >> 4), t_d = st + (C::TP_OFF >> 4), p_d = t_d + (2 * kGdnSquareBytes >> 4);
            ok = ptx::mbar_wait_bounded(&full[s], static_cast<uint32_t>(c / C::STAGES) & 1u, abort_flag, w.wait_limit_ns);
            if (ok) ok = ptx::mbar_wait_bounded(s_ready, ph, abort_flag, w.wait_limit_ns);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            ptx::tc_fence_after();
            // X^T = S^T K^T, then S^T Q^T: step k of 16 is 32 bytes into its 64-column half
            auto product = [&](uint32_t d, uint32_t a, uint32_t b, uint32_t first) {
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    gdn_mma_ts(d, a + 8 * k, (b + (k >> 2) * (kGdnTileBytes / 2 >> 4) + (k & 3) * 2) | kLo, kHi, kN64, first != 0u ? k > 0 : 1u, lp);
            };
            product(tmem + kTmX, tmem + kTmSh, k_d, 1u);
            product(tmem + kTmX, tmem + kTmSl, k_d, 0u);
            ptx::tc_commit_if(x_full, lp);
            // U^T = R^T T^T: T is lower triangular, tokens 16 j .. 16 j + 15 of R reach columns 16 j and up only
            ok = ptx::mbar_wait_bounded(r_ready, ph, abort_flag, w.wait_limit_ns);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            ptx::tc_fence_after();
            auto lower = [&](uint32_t d, uint32_t a, uint32_t b, uint32_t first) {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    gdn_mma_ts(d + 16 * j, a + 32 * (j >> 1) + 8 * (j & 1), (b + j * (2048 >> 4) + j * 2) | kLo, kHi,
                               kIdesc | (static_cast<uint32_t>(8 - 2 * j) << 17), first != 0u ? j > 0 : 1u, lp);
            };
            lower(tmem + kTmU, tmem + kTmX, t_d, 1u);
            lower(tmem + kTmU, tmem + kTmX + 16, t_d, 0u);
            lower(tmem + kTmU, tmem + kTmX, t_d + (kGdnSquareBytes >> 4), 0u);
            ptx::tc_commit_if(u_full, lp);
            // the update U^T diag(w) K, which the chain waits for; the read-out S^T Q^T and U^T P^T behind it
            ok = ptx::mbar_wait_bounded(u_ready, ph, abort_flag, w.wait_limit_ns);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            ptx::tc_fence_after();
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    gdn_mma_ts(tmem + kTmD, tmem + kTmU + 32 * (j >> 1) + 8 * (j & 1) + 16 * x, (k_d + j * (2048 >> 4)) | kLoT, kHi, kN128T, (x | j) != 0, lp);
            ptx::tc_commit_if(d_full, lp);
            if (c > 0) ok = ptx::mbar_wait_bounded(o_done, ph ^ 1u, abort_flag, w.wait_limit_ns);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            ptx::tc_fence_after();
            product(tmem + kTmQ, tmem + kTmSh, q_d, 1u);
            product(tmem + kTmQ, tmem + kTmSl, q_d, 0u);
            lower(tmem + kTmY, tmem + kTmX, p_d, 1u);
            lower(tmem + kTmY, tmem + kTmX + 16, p_d, 0u);
            lower(tmem + kTmY, tmem + kTmX, p_d + (kGdnSquareBytes >> 4), 0u);
            ptx::tc_commit_if(y_full, lp);
            ptx::tc_commit_if(&empty[s], lp);
        }
        if (!ok) {
            // let issued MMAs finish before TMEM is freed
            ptx::tc_commit_if(drain, lp);
            for (int spin = 0; spin < (1 << 16) && !ptx::mbar_try_wait(drain, 0u); ++spin) {}
        }
    }
    } else {
        // ------------------------------------------------------------ compute
        asm volatile("setmaxnreg.inc.sync.aligned.u32 200;");
        const int half = warp >> 2, row = (warp & 3) * 32 + lane;     // value column of the head
        const uint32_t tq = tmem + (static_cast<uint32_t>((warp & 3) * 32) << 16);
        float* const state = p.state + (sslot * p.Hv + h) * (kGdnWidth * kGdnWidth) + static_cast<int64_t>(64 * half) * kGdnWidth + row;
        float S[64];
#pragma unroll
        for (int i = 0; i < 64; ++i) S[i] = fresh ? 0.0f : state[i * kGdnWidth];
        // the larger of both halves' values of a row
        auto exchange = [&](int which, float m, bool ok_in, bool& ok_out) {
            float* slot = mx + which * (2 * kGdnWidth);
            slot[half * kGdnWidth + row] = m;
            ok_out = gdn_and_barrier<64>(1 + (warp & 3), ok_in);          // (the two warps that share 32 rows)
            return fmaxf(m, slot[(half ^ 1) * kGdnWidth + row]);
        };
        // O of chunk c, 16 of this warp's 32 tokens (part 0 or 1), from S^T Q^T and U^T P^T: it leaves beside the products of the
        // next chunk.  is, iu: the scales of S and U in those products.
        const uint32_t stage_s = ptx::smem_u32(out_s) + static_cast<uint32_t>(warp) * 1024u;
        auto output = [&](int c, int part, float is, float iu) {
            const float* sd = side + (warp * 2 + (c & 1)) * 36;
            const int t0 = 32 * half + 16 * part, n = min(kGdnChunk, len - c * kGdnChunk) - t0;
            uint32_t x[16], y[16];
            ptx::tmem_ld_32x16(tq + kTmQ + t0, x);
            ptx::tmem_ld_32x16(tq + kTmY + t0, y);
            ptx::tmem_ld_wait();
            if (part == 1) {
                ptx::tc_fence_before();
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(o_done);
            }
            const float fy = iu * sd[32 + part];
            const int64_t at = static_cast<int64_t>(begin + c * kGdnChunk + t0) * p.ldo + h * kGdnWidth + (warp & 3) * 32;
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
                float4 dd = *reinterpret_cast<const float4*>(sd + 16 * part + i);
                gdn_mul2(dd.x, dd.y, is, is);
                gdn_mul2(dd.z, dd.w, is, is);
                float o[4] = {__uint_as_float(x[i]), __uint_as_float(x[i + 1]), __uint_as_float(x[i + 2]), __uint_as_float(x[i + 3])};
                float q[4] = {__uint_as_float(y[i]), __uint_as_float(y[i + 1]), __uint_as_float(y[i + 2]), __uint_as_float(y[i + 3])};
                gdn_mul2(q[0], q[1], fy, fy);
                gdn_mul2(q[2], q[3], fy, fy);
                gdn_fma2(o[0], o[1], dd.x, dd.y, q[0], q[1]);
                gdn_fma2(o[2], o[3], dd.z, dd.w, q[2], q[3]);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (F32) {                                    // 32 lanes: one line per token
                        if (i + e < n) static_cast<float*>(p.o)[at + (i + e) * p.ldo + lane] = o[e];
                    } else {
                        const __nv_bfloat16 b = __float2bfloat16_rn(o[e]);
                        asm volatile("st.shared.b16 [%0], %1;" ::"r"(stage_s + static_cast<uint32_t>((i + e) * 64 + lane * 2)),
                                     "h"(*reinterpret_cast<const uint16_t*>(&b)) : "memory");
                    }
                }
            }
            if (!F32) {                                           // across shared memory: 16 bytes a lane, 64 contiguous a token
                __syncwarp();
                __nv_bfloat16* o = static_cast<__nv_bfloat16*>(p.o) + at + (lane & 3) * 8;
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int token = 8 * i + (lane >> 2);
                    const uint4 q = ptx::ld_shared_v4(stage_s + static_cast<uint32_t>(token * 64 + (lane & 3) * 16));
                    if (token < n) *reinterpret_cast<uint4*>(o + token * p.ldo) = q;
                }
                __syncwarp();
            }
        };
        float is_prev = 0.0f, iu_prev = 0.0f;
        bool ok = true;
        for (int c = 0; c < chunks; ++c) {
            const int s = c & 1;
            const uint32_t ph = static_cast<uint32_t>(c) & 1u;
            const uint8_t* st = smem + s * C::STAGE_BYTES;
            const float* vec = reinterpret_cast<const float*>(st + C::VEC_OFF);
            const int n = min(kGdnChunk, len - c * kGdnChunk);
            // ---- S, split, to TMEM
            float m = 0.0f;
#pragma unroll
            for (int i = 0; i < 64; i += 2) m = gdn_max_abs(m, S[i], S[i + 1]);
            bool both;
            m = exchange(0, m, ok, both);
            if (!both) {                                         // (the two warps of these rows leave together)
                ok = false;
                break;
            }
            float sc, is;
            gdn_pow2_scale(m, 12, sc, is);
            {
                uint32_t hi[32], lo[32];
#pragma unroll
                for (int i = 0; i < 32; ++i) gdn_split(S[2 * i], S[2 * i + 1], sc, hi[i], lo[i]);
                if (c > 0) {                                     // the read-out of the chunk in front has read the old S
                    ok = ptx::mbar_wait_bounded(y_full, ph ^ 1u, abort_flag, w.wait_limit_ns) && ok;
                    ok = __all_sync(0xffffffffu, ok);
                    ptx::tc_fence_after();
                }
                ptx::tmem_st_32x32(tq + kTmSh + 32 * half, hi);
                ptx::tmem_st_32x32(tq + kTmSl + 32 * half, lo);
            }
            ptx::tmem_st_wait();
            ptx::tc_fence_before();
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(s_ready);
            if (c > 0 && ok) output(c - 1, 0, is_prev, iu_prev); // (while the first products run)
            // ---- R = V - diag(c) X for tokens 32 half .. + 31
            ok = ptx::mbar_wait_bounded(&full[s], static_cast<uint32_t>(c / C::STAGES) & 1u, abort_flag, w.wait_limit_ns) && ok;
            {
                // what the output of this chunk needs of the stage, kept until then
                float* sd = side + (warp * 2 + s) * 36;
                sd[lane] = vec[kGdnChunk + 32 * half + lane];
                if (lane < 2) sd[32 + lane] = vec[kGdnVecP + 2 * half + lane];
            }
            const uint16_t* v = reinterpret_cast<const uint16_t*>(st + C::V_OFF) + 32 * half * kGdnWidth + row;
            uint32_t vv[32];
#pragma unroll
            for (int i = 0; i < 32; ++i) vv[i] = static_cast<uint32_t>(v[i * kGdnWidth]) << 16;
            if (n < kGdnChunk) {
#pragma unroll
                for (int i = 0; i < 32; ++i) vv[i] = 32 * half + i < n ? vv[i] : 0u;     // (what is there instead may be anything)
            }
            ok = ptx::mbar_wait_bounded(x_full, ph, abort_flag, w.wait_limit_ns) && ok;
            ok = __all_sync(0xffffffffu, ok);
            ptx::tc_fence_after();
            float r[32];
            float i0, s0;
            {
                uint32_t x[32];
                ptx::tmem_ld_32x32(tq + kTmX + 32 * half, x);
                ptx::tmem_ld_wait();
                m = 0.0f;
#pragma unroll
                for (int i = 0; i < 32; i += 4) {
                    float4 cc = *reinterpret_cast<const float4*>(vec + 32 * half + i);
                    gdn_mul2(cc.x, cc.y, -is, -is);
                    gdn_mul2(cc.z, cc.w, -is, -is);
#pragma unroll
                    for (int e = 0; e < 4; ++e) r[i + e] = __uint_as_float(x[i + e]);
                    gdn_fma2(r[i], r[i + 1], cc.x, cc.y, __uint_as_float(vv[i]), __uint_as_float(vv[i + 1]));
                    gdn_fma2(r[i + 2], r[i + 3], cc.z, cc.w, __uint_as_float(vv[i + 2]), __uint_as_float(vv[i + 3]));
#pragma unroll
                    for (int e = 0; e < 4; e += 2) m = gdn_max_abs(m, r[i + e], r[i + e + 1]);
                }
            }
            m = exchange(1, m, ok, both);
            gdn_pow2_scale(m, 12, s0, i0);
            {
                uint32_t hi[16], lo[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) gdn_split(r[2 * i], r[2 * i + 1], s0, hi[i], lo[i]);
                ptx::tmem_st_32x16(tq + kTmX + 32 * half, hi);
                ptx::tmem_st_32x16(tq + kTmX + 32 * half + 16, lo);
            }
            ptx::tmem_st_wait();
            ptx::tc_fence_before();
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(r_ready);
            // ---- U, and U diag(w), split
            ok = ptx::mbar_wait_bounded(u_full, ph, abort_flag, w.wait_limit_ns) && ok;
            ok = __all_sync(0xffffffffu, ok);
            ptx::tc_fence_after();
            float iu, su, iw, sw;
            {
                uint32_t x[32];
                ptx::tmem_ld_32x32(tq + kTmU + 32 * half, x);
                ptx::tmem_ld_wait();
                const float i16[2] = {i0 * vec[kGdnVecT + 2 * half], i0 * vec[kGdnVecT + 2 * half + 1]};
                float wm = 0.0f;
                float u[32];
                m = 0.0f;
#pragma unroll
                for (int i = 0; i < 32; i += 2) {
                    u[i] = __uint_as_float(x[i]);
                    u[i + 1] = __uint_as_float(x[i + 1]);
                    gdn_mul2(u[i], u[i + 1], i16[i >> 4], i16[i >> 4]);
                    m = gdn_max_abs(m, u[i], u[i + 1]);
                    r[i] = u[i];
                    r[i + 1] = u[i + 1];
                }
#pragma unroll
                for (int i = 0; i < 32; i += 4) {
                    const float4 ww = *reinterpret_cast<const float4*>(vec + 2 * kGdnChunk + 32 * half + i);
                    gdn_mul2(r[i], r[i + 1], ww.x, ww.y);
                    gdn_mul2(r[i + 2], r[i + 3], ww.z, ww.w);
#pragma unroll
                    for (int e = 0; e < 4; e += 2) wm = gdn_max_abs(wm, r[i + e], r[i + e + 1]);
                }
                // both maxima in one exchange
                float* slot = mx + 2 * (2 * kGdnWidth);
                float* slot2 = mx + 3 * (2 * kGdnWidth);
                slot[half * kGdnWidth + row] = m;
                slot2[half * kGdnWidth + row] = wm;
                gdn_and_barrier<64>(1 + (warp & 3), true);
                m = fmaxf(m, slot[(half ^ 1) * kGdnWidth + row]);
                wm = fmaxf(wm, slot2[(half ^ 1) * kGdnWidth + row]);
                gdn_pow2_scale(m, 12, su, iu);
                gdn_pow2_scale(wm, 12, sw, iw);
                uint32_t hi[16], lo[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) gdn_split(u[2 * i], u[2 * i + 1], su, hi[i], lo[i]);
                ptx::tmem_st_32x16(tq + kTmX + 32 * half + 16, lo);
                ptx::tmem_st_32x16(tq + kTmX + 32 * half, hi);
#pragma unroll
                for (int i = 0; i < 16; ++i) gdn_split(r[2 * i], r[2 * i + 1], sw, hi[i], lo[i]);
                ptx::tmem_st_32x16(tq + kTmU + 32 * half, hi);
                ptx::tmem_st_32x16(tq + kTmU + 32 * half + 16, lo);
            }
            ptx::tmem_st_wait();
            ptx::tc_fence_before();
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(u_ready);
            const float gamma = vec[3 * kGdnChunk];
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(&empty[s]);          // (the last read of this stage by this warp)
            if (c > 0 && ok) output(c - 1, 1, is_prev, iu_prev); // (while the update's products run)
            is_prev = is;
            iu_prev = iu;
            // ---- S <- gamma S + update
            ok = ptx::mbar_wait_bounded(d_full, ph, abort_flag, w.wait_limit_ns) && ok;
            ok = __all_sync(0xffffffffu, ok);
            ptx::tc_fence_after();
            {
                uint32_t x[64];
                ptx::tmem_ld_32x64(tq + kTmD + 64 * half, x);
                ptx::tmem_ld_wait();
#pragma unroll
                for (int i = 0; i < 64; i += 2) {
                    float d0 = __uint_as_float(x[i]), d1 = __uint_as_float(x[i + 1]);
                    gdn_mul2(d0, d1, iw, iw);
                    gdn_fma2(S[i], S[i + 1], gamma, gamma, d0, d1);
                }
            }
        }
        if (ok && chunks > 0) {
            ok = ptx::mbar_wait_bounded(y_full, static_cast<uint32_t>(chunks - 1) & 1u, abort_flag, w.wait_limit_ns);
            ok = __all_sync(0xffffffffu, ok);
            ptx::tc_fence_after();
        }
        // Every compute warp passes here once, whichever way it left the loop.  If one gave up, none writes: a head's state in the
        // pool is the one from before or the one from behind these chunks, never some of both.
        ok = gdn_and_barrier<256>(5, ok);
        if (ok) {
            if (chunks > 0) {
                output(chunks - 1, 0, is_prev, iu_prev);
                output(chunks - 1, 1, is_prev, iu_prev);
            }
#pragma unroll
            for (int i = 0; i < 64; ++i) state[i * kGdnWidth] = S[i];
        }
    }
    ptx::tc_fence_before();
    __syncthreads();
    if (*abort_flag != 0u) __nanosleep(50000);
    if (warp == 8) {
        ptx::tc_fence_after();
        ptx::tmem_dealloc(tmem, 512);
    }
    if (tid == 0 && *abort_flag != 0u) atomicExch(w.status, static_cast<uint32_t>(NVFP4_ERR_TIMEOUT));
}

}  // namespace nvfp4
