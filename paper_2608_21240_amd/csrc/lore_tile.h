// The LoRE down tiles of the GEMM kernels (bf16 / MXFP4 experts: expert_gemm.hip, 8-bit ones:
// expert_ffn_i8.hip; internal linkage: each source compiles its own copy).  C is the kernel's tile shape;
// Args has d, r, u and y_slots; Job the tile's w (B_e), row0, tok0, ntok and start.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace spice {
namespace {

constexpr int kLoreDown = 4;  // BM-row blocks of a LORE down tile (short: r is small)

typedef float lore_f32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t lore_u32x4_t __attribute__((ext_vector_type(4)));

// D = U B_e^T of BM rows of B_e x BT bucket entries (a LORE tile takes kLoreDown such blocks:
// one alone is shorter than the block's start; draft rollout, T = 64: 17.8 -> 12.7 us), contraction
// r.  fp32 MFMAs
// (16x16x4), so that U keeps its 32 bits; operands straight from L2, whose reuse is within the
// block.  A 32-k step gives each lane 8 consecutive k of its row (quad), and MFMA i takes
// element i of every lane; the next step's loads are out before this one's MFMAs.  Rows past d
// and entries past the bucket read the last one.
template <class C, class Args, class Job>
__device__ __forceinline__ void lore_down(const Args& a, const Job& j) {
    const int lane = threadIdx.x & 63, m = lane & 15, quad = lane >> 4;
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wf = w % C::WF, wt = w / C::WF;
    const int nlive = min(C::RT, max(0, (j.ntok - j.tok0 - 16 * wt + C::kTStride - 1) / C::kTStride));
    if (nlive == 0) return;
    const uint16_t* B = static_cast<const uint16_t*>(j.w);
    lore_f32x4_t acc[C::RF][C::RT];
#pragma unroll
    for (int s = 0; s < C::RF; ++s)
#pragma unroll
        for (int t = 0; t < C::RT; ++t) acc[s][t] = lore_f32x4_t{0.f, 0.f, 0.f, 0.f};
    const uint16_t* brow[C::RF];
    const float* urow[C::RT];
#pragma unroll
    for (int s = 0; s < C::RF; ++s)
        brow[s] = B + (size_t)min(j.row0 + wf * (C::BM / C::WF) + s * 16 + m, a.d - 1) * a.r;
#pragma unroll
    for (int t = 0; t < C::RT; ++t)
        urow[t] = a.u + (size_t)(j.start + min(j.tok0 + t * C::kTStride + wt * 16 + m, j.ntok - 1)) * a.r;
    struct Step {
        lore_u32x4_t b[C::RF];
        lore_f32x4_t u[C::RT][2];
    };
    auto fetch = [&](int k0, Step& st) {
        const int k = k0 + quad * 8;
        const bool in = k < a.r;  // r is a multiple of 8
#pragma unroll
        for (int s = 0; s < C::RF; ++s)
            st.b[s] = in ? *reinterpret_cast<const lore_u32x4_t*>(brow[s] + k) : lore_u32x4_t{0u, 0u, 0u, 0u};
#pragma unroll
        for (int t = 0; t < C::RT; ++t)
#pragma unroll
            for (int h = 0; h < 2; ++h)
                st.u[t][h] = in && t < nlive ? *reinterpret_cast<const lore_f32x4_t*>(urow[t] + k + 4 * h)
                                             : lore_f32x4_t{0.f, 0.f, 0.f, 0.f};
    };
    auto mul = [&](const Step& st) {
#pragma unroll
        for (int s = 0; s < C::RF; ++s) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t v = st.b[s][i >> 1];
                const float av = __uint_as_float(i & 1 ? v & 0xFFFF0000u : v << 16);
#pragma unroll
                for (int t = 0; t < C::RT; ++t)
                    if (t < nlive)
                        acc[s][t] = __builtin_amdgcn_mfma_f32_16x16x4f32(av, st.u[t][i >> 2][i & 3], acc[s][t], 0, 0, 0);
            }
        }
    };
    Step cur, nxt;
    fetch(0, cur);
    for (int k0 = 0; k0 < a.r; k0 += 32) {
        if (k0 + 32 < a.r) fetch(k0 + 32, nxt);
        mul(cur);
        cur = nxt;
    }
#pragma unroll
    for (int t = 0; t < C::RT; ++t) {
        const int pos = j.tok0 + t * C::kTStride + wt * 16 + m;
        if (pos >= j.ntok) continue;
        float* dst = a.y_slots + (size_t)(j.start + pos) * a.d;
#pragma unroll
        for (int s = 0; s < C::RF; ++s) {
            const int f = j.row0 + wf * (C::BM / C::WF) + s * 16 + quad * 4;
            if (f < a.d) *reinterpret_cast<lore_f32x4_t*>(dst + f) = acc[s][t];
        }
    }
}

}  // namespace
}  // namespace spice
