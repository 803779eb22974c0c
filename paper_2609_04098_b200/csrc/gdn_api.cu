// Host side of the served gated delta-rule calls declared in include/nvfp4.h: argument checks and launches.
#include <cstring>
#include <mutex>
#include <unordered_map>

#include <cuda_runtime.h>

#include "../../include/nvfp4.h"
#include "gdn.cuh"
#include "gdn_chunk.cuh"
#include "host.h"

using namespace nvfp4;

namespace {
constexpr uint32_t kGdnFlags = NVFP4_OUT_F32 | NVFP4_GDN_L2NORM | NVFP4_GDN_GATES_F32 | NVFP4_GDN_DECAY_FIRST;

// the checks that the prefill and the single-token call share; fills everything but cu, has_state
nvfp4_status gdn_check(GdnParams& p, const void* d_q, int64_t ldq, const void* d_k, int64_t ldk, const void* d_v, int64_t ldv,
                       const void* d_a, int64_t lda, const void* d_b, int64_t ldb, const float* d_A_log,
                       const float* d_dt_bias, int64_t T, int Hk, int Hv, int64_t nseq, float* d_state, int64_t nslots,
                       const int32_t* d_slots, void* d_o, int64_t ldo, uint32_t flags) {
    if (T != 0 && (d_q == nullptr || d_k == nullptr || d_v == nullptr || d_a == nullptr || d_b == nullptr || d_o == nullptr))
        return NVFP4_ERR_NULL;                                   // (without tokens there may be no arrays)
    if (d_A_log == nullptr || d_dt_bias == nullptr || d_state == nullptr) return NVFP4_ERR_NULL;
    if (T < 0 || T >= (1ll << 31) - 256 || nseq < 0 || nseq > 65535 || nslots < 0 || Hk < 1 || Hv < 1 || Hv > 65535 ||
        (Hv % Hk) != 0 || (flags & ~kGdnFlags) != 0u)
        return NVFP4_ERR_SHAPE;
    const int64_t wk = static_cast<int64_t>(Hk) * kGdnWidth, wv = static_cast<int64_t>(Hv) * kGdnWidth;
    if (ldq < wk || ldk < wk || ldv < wv || lda < Hv || ldb < Hv || ldo < wv) return NVFP4_ERR_SHAPE;
    const bool out_f32 = (flags & NVFP4_OUT_F32) != 0u;
    const uintptr_t gate_mask = (flags & NVFP4_GDN_GATES_F32) != 0u ? 3u : 1u;
    if (!aligned16(d_q) || !aligned16(d_k) || !aligned16(d_v) || !aligned16(d_state) || !aligned16(d_o) || (ldq % 8) != 0 ||
        (ldk % 8) != 0 || (ldv % 8) != 0 || (ldo % (out_f32 ? 4 : 8)) != 0 ||
        ((reinterpret_cast<uintptr_t>(d_a) | reinterpret_cast<uintptr_t>(d_b)) & gate_mask) != 0 ||
        ((reinterpret_cast<uintptr_t>(d_A_log) | reinterpret_cast<uintptr_t>(d_dt_bias) |
          reinterpret_cast<uintptr_t>(d_slots)) & 3u) != 0)
        return NVFP4_ERR_ALIGN;
    // o over an input: other CTAs (a prefill's later chunks too) read what one would write.  Columns side by side are fine.
    const int64_t os = out_f32 ? 4 : 2, gs = (flags & NVFP4_GDN_GATES_F32) != 0u ? 4 : 2;
    auto under_o = [&](const void* x, int64_t stride, int64_t width) { return blocks_overlap(x, stride, width, d_o, ldo * os, wv * os, T); };
    if (under_o(d_q, ldq * 2, wk * 2) || under_o(d_k, ldk * 2, wk * 2) || under_o(d_v, ldv * 2, wv * 2) ||
        under_o(d_a, lda * gs, Hv * gs) || under_o(d_b, ldb * gs, Hv * gs) ||
        (nslots > 0 && T > 0 && blocks_overlap(d_o, 0, ((T - 1) * ldo + wv) * os, d_state, 0, nslots * wv * (kGdnWidth * 4), 1)))
        return NVFP4_ERR_SHAPE;
    std::memset(&p, 0, sizeof(p));
    p.q = static_cast<const uint16_t*>(d_q);
    p.k = static_cast<const uint16_t*>(d_k);
    p.v = static_cast<const uint16_t*>(d_v);
    p.ldq = ldq;
    p.ldk = ldk;
    p.ldv = ldv;
    p.a = d_a;
    p.b = d_b;
    p.lda = lda;
    p.ldb = ldb;
    p.A_log = d_A_log;
    p.dt_bias = d_dt_bias;
    p.slots = d_slots;
    p.state = d_state;
    p.nslots = nslots;
    p.o = d_o;
    p.ldo = ldo;
    p.T = static_cast<int32_t>(T);
    p.nseq = static_cast<int32_t>(nseq);
    p.Hk = Hk;
    p.Hv = Hv;
    p.flags = flags;
    return NVFP4_OK;
}

int64_t gdn_chunk_slots(int64_t T, int64_t nseq) { return T / kGdnChunk + nseq; }
size_t gdn_kq_bytes(int64_t T, int64_t nseq, int Hk) {
    return static_cast<size_t>(gdn_chunk_slots(T, nseq)) * static_cast<size_t>(Hk) * (2 * kGdnTileBytes);
}

template <bool F32>
nvfp4_status launch_gdn_chunks(const GdnParams& p, const GdnWorkspace& w, bool early, cudaStream_t stream) {
    using C = GdnChunkCfg<F32>;
    static std::mutex mu;
    static std::unordered_map<int, bool> configured;
    int dev = 0;
    cudaGetDevice(&dev);
    {
        std::lock_guard<std::mutex> lock(mu);
        if (!configured[dev]) {
            if (cudaFuncSetAttribute(gdn_chunk_kernel<F32>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM_BYTES) != cudaSuccess)
                return NVFP4_ERR_CUDA;
            configured[dev] = true;
        }
    }
    cudaLaunchConfig_t cfg;
    std::memset(&cfg, 0, sizeof(cfg));
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;      // (the kernel waits for its predecessor itself)
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.gridDim = dim3(static_cast<unsigned>(p.Hv), static_cast<unsigned>(p.nseq));
    cfg.blockDim = dim3(kGdnChunkThreads);
    cfg.dynamicSmemBytes = C::SMEM_BYTES;
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = early ? 1 : 0;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, gdn_chunk_kernel<F32>, p, w);
    g_launches.fetch_add(1, std::memory_order_relaxed);
    return e == cudaSuccess ? NVFP4_OK : NVFP4_ERR_CUDA;
}
}  // namespace

extern "C" {

size_t nvfp4_gdn_prefill_workspace_bytes(int64_t T, int64_t nseq, int Hk, int Hv, uint32_t /* flags: no part of it so far */) {
    if (T < 0 || nseq < 0 || Hk < 1 || Hv < 1) return 0;
    return kStatusBytes + gdn_kq_bytes(T, nseq, Hk) +
           static_cast<size_t>(gdn_chunk_slots(T, nseq)) * static_cast<size_t>(Hv) * kGdnTpBytes;
}

nvfp4_status nvfp4_gdn_prefill(const void* d_q, int64_t ldq, const void* d_k, int64_t ldk, const void* d_v, int64_t ldv,
                               const void* d_a, int64_t lda, const void* d_b, int64_t ldb, const float* d_A_log,
                               const float* d_dt_bias, int64_t T, int Hk, int Hv, const int32_t* d_cu_seqlens, int64_t nseq,
                               float* d_state, int64_t nslots, const int32_t* d_slots, const uint8_t* d_has_state,
                               void* d_o, int64_t ldo, uint32_t flags, void* d_workspace, size_t workspace_bytes,
                               void* stream) {
    GdnParams p;
    nvfp4_status st = gdn_check(p, d_q, ldq, d_k, ldk, d_v, ldv, d_a, lda, d_b, ldb, d_A_log, d_dt_bias, T, Hk, Hv, nseq,
                                d_state, nslots, d_slots, d_o, ldo, flags);
    if (st != NVFP4_OK) return st;
    if (d_cu_seqlens == nullptr) return NVFP4_ERR_NULL;
    if ((reinterpret_cast<uintptr_t>(d_cu_seqlens) & 3u) != 0) return NVFP4_ERR_ALIGN;
    if (d_workspace == nullptr || workspace_bytes < nvfp4_gdn_prefill_workspace_bytes(T, nseq, Hk, Hv, flags))
        return NVFP4_ERR_WORKSPACE;
    if ((reinterpret_cast<uintptr_t>(d_workspace) & 255u) != 0) return NVFP4_ERR_ALIGN;
    p.cu = d_cu_seqlens;
    p.has_state = d_has_state;
    if (nseq == 0) return NVFP4_OK;
    DeviceInfo info;
    st = check_arch(info);
    if (st != NVFP4_OK) return st;
    const bool out_f32 = (flags & NVFP4_OUT_F32) != 0u;
    cudaStream_t s = as_stream(stream);
    GdnWorkspace w;
    std::memset(&w, 0, sizeof(w));
    w.status = static_cast<uint32_t*>(d_workspace);
    w.kq = static_cast<uint8_t*>(d_workspace) + kStatusBytes;
    w.tp = w.kq + gdn_kq_bytes(T, nseq, Hk);
    const uint64_t lim = g_wait_limit_ns.load(std::memory_order_relaxed);
    w.sm_count = static_cast<uint32_t>(info.sm_count);
    w.wait_limit_ns = lim != 0 ? lim : kWaitLimitNs;
    {
        static std::mutex mu;
        static std::unordered_map<int, bool> configured;
        int dev = 0;
        cudaGetDevice(&dev);
        std::lock_guard<std::mutex> lock(mu);
        if (!configured[dev]) {
            if (cudaFuncSetAttribute(gdn_chunk_prepare_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                     static_cast<int>(sizeof(GdnPrepSmem))) != cudaSuccess)
                return NVFP4_ERR_CUDA;
            configured[dev] = true;
        }
    }
    const int64_t slots = gdn_chunk_slots(T, nseq);
    auto prepare = [&](int64_t ctas_x, bool early) {
        // the value heads of one key head in one CTA (keys and queries converted once) when that still gives every SM
        // several CTAs; one CTA per value head otherwise, for latency.  16 key and 48 value heads, whole calls, one head a CTA
        // against three: 17 tokens 17.7 and 27.0 us, 512 49.6 and 55.7, 1024 91 and 90, 2048 172 and 165, 7 prompts of 1500
        // each 490 and 451
        const int heads = ctas_x * Hk >= 4ll * info.sm_count ? Hv / Hk : 1;
        cudaLaunchConfig_t cfg;
        std::memset(&cfg, 0, sizeof(cfg));
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[0].val.programmaticStreamSerializationAllowed = 1;
        cfg.gridDim = dim3(static_cast<unsigned>(ctas_x), static_cast<unsigned>(Hv / heads));
        cfg.blockDim = dim3(kGdnPrepThreads);
        cfg.dynamicSmemBytes = sizeof(GdnPrepSmem);
        cfg.stream = s;
        cfg.attrs = attr;
        cfg.numAttrs = early ? 1 : 0;
        const cudaError_t e = cudaLaunchKernelEx(&cfg, gdn_chunk_prepare_kernel, p, w, heads);
        g_launches.fetch_add(1, std::memory_order_relaxed);
        return e == cudaSuccess ? NVFP4_OK : NVFP4_ERR_CUDA;
    };
    auto serial = [&](bool early) { return out_f32 ? launch_gdn_chunks<true>(p, w, early, s) : launch_gdn_chunks<false>(p, w, early, s); };
    // Few long sequences leave SMs idle during the serial part: the chunks go in ranges, and the next range is prepared under
    // the serial kernel of the current one.  8192 tokens, 48 heads: 624 us in one piece; 593 / 584 / 577 / 581 us in ranges of
    // 16 / 24 / 32 / 48 chunks.  With every SM busy ranges only cost (16 prompts of 1000 tokens each, float output: 690 us in one
    // piece, 830 us in ranges): the preparation then takes from the serial kernel what it hides.  Between half and all of the SMs
    // it goes either way -- 96 CTAs: two prompts of 8192 730 us in one piece and 669 us in ranges, three of 4096 at 32 heads
    // 384 and 372; 128 and 144 CTAs: four of 4096 at 32 heads 421 and 450, three at 48 heads 436 and 460 -- and the rule takes
    // one piece.
    // Lengths are on the device: the longest sequence may have all T tokens, and a range that no sequence reaches still costs
    // its two launches, so an average length decides.
    constexpr int64_t kRange = 32;
    const int64_t longest = (T + kGdnChunk - 1) / kGdnChunk;
    if (2 * nseq * Hv > info.sm_count || longest <= (kRange + kRange / 2) * nseq) {
        if (T > 0) st = prepare(slots, false);
        return st == NVFP4_OK ? serial(T > 0) : st;
    }
    w.chunk_count = static_cast<int32_t>(kRange);
    for (int64_t c = 0; c < longest && st == NVFP4_OK; c += kRange) {
        w.chunk_begin = static_cast<int32_t>(c);
        st = prepare(nseq * kRange, c > 0);
        if (st == NVFP4_OK) st = serial(false);        // (started early it measured slower: 590 us against 559)
    }
    return st;
}

nvfp4_status nvfp4_gdn_decode(const void* d_q, int64_t ldq, const void* d_k, int64_t ldk, const void* d_v, int64_t ldv,
                              const void* d_a, int64_t lda, const void* d_b, int64_t ldb, const float* d_A_log,
                              const float* d_dt_bias, int64_t batch, int Hk, int Hv, float* d_state, int64_t nslots,
                              const int32_t* d_slots, void* d_o, int64_t ldo, uint32_t flags, void* stream) {
    GdnParams p;
    nvfp4_status st = gdn_check(p, d_q, ldq, d_k, ldk, d_v, ldv, d_a, lda, d_b, ldb, d_A_log, d_dt_bias, batch, Hk, Hv,
                                batch, d_state, nslots, d_slots, d_o, ldo, flags);
    if (st != NVFP4_OK) return st;
    if (batch == 0) return NVFP4_OK;
    DeviceInfo info;
    st = check_arch(info);
    if (st != NVFP4_OK) return st;
    // a whole head per CTA; a quarter of one while that still leaves SMs idle (few sequences: latency, not bandwidth).  48 heads,
    // quarters against whole heads: 1 sequence 3.3 and 4.2 us, 3 4.5 and 5.8, 6 8.0 and 7.5, 7 9.8 and 7.9, 12 14.5 and 10.9
    const bool quarters = batch * Hv <= 2ll * info.sm_count;
    cudaLaunchConfig_t cfg;
    std::memset(&cfg, 0, sizeof(cfg));
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;      // (the kernel waits for its predecessor itself)
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.gridDim = dim3(static_cast<unsigned>(Hv * (quarters ? 4 : 1)), static_cast<unsigned>(batch), 1);
    cfg.blockDim = dim3(kGdnDecodeThreads, 1, 1);
    cfg.stream = as_stream(stream);
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    const cudaError_t e = quarters ? cudaLaunchKernelEx(&cfg, gdn_decode_kernel<32>, p) : cudaLaunchKernelEx(&cfg, gdn_decode_kernel<128>, p);
    g_launches.fetch_add(1, std::memory_order_relaxed);
    return e == cudaSuccess ? NVFP4_OK : NVFP4_ERR_CUDA;
}

}  // extern "C"
