// Grouped SwiGLU FFN of the HIT experts' buckets and of the shared block with 8-bit weights and
// activations (moe_expert_ffn_grouped_i8), three launches:
//
//   up    : H[pos][f] = silu(sx s1[f] sum_k W1[f][k] x[k]) * (sx s3[f] sum_k W3[f][k] x[k])  (fp32)
//   quant : per row of H, sh = max |h| / 127 and qh = round(h / sh)  (int8; few rows: in down)
//   down  : Y[pos][j] = sh s2[j] sum_k W2[j][k] qh[k]                                         (fp32)
//
// The sums are int32 MFMAs (v_mfma_i32_16x16x64_i8) and exact, whatever their order; H stays fp32 until
// its row's maximum is known, so its only rounding to 8 bits is the one the format has (bf16 in between
// would move about 1 % of the codes).
//
// A block computes BM weight rows x BT tokens over the contraction, 128 k per stage, weights as the A
// operand, tokens as B.  For `up` the rows are BM / 2 W1 rows and the same W3 rows, so a wave holds the
// gate and up sums of its features and applies the scales and SwiGLU in registers.  A wave's token
// sub-tiles are interleaved with the other waves' (rows kTStride t + 16 wt), so the ragged last tile of an
// expert spreads over the SIMDs; sub-tiles without a live token are not read and issue no MFMA, and their
// rows are not fetched.
// The LoRE corrections of the LORE buckets (Eq. 9) run beside them: U = A_e x of a bucket is a tile of the
// up launch on the same stages with bf16 MFMAs, U B_e^T one of the down launch; they come first, since an
// up tile's bf16 rows are twice as long (block of 16 tokens 97 -> 84 us).
// Staging: buffer loads straight to LDS into a ring of S stages of 128-byte rows whose 16-byte chunks are
// XOR-swizzled by row (chunk c of row r at c ^ ((r >> 1) & 7)).  A chunk past the end of a row, and a row
// past the end of a matrix or a bucket, reads zero (an offset past the buffer).
// Pipeline: the fragments of a stage's two k-steps are read half a stage ahead of their MFMAs; one barrier
// per stage, in the middle of the MFMAs, frees the buffer just read for the stage S ahead.  In the tall tiles
// the weights' ring is a stage deeper than the tokens', which L2 holds (T = 4096 below 2117 -> 2022 us).
//
// What bounds it, with the us of a whole call (the launches one by one on a stream): short buckets the
// weights' way from memory, by which a call of 32 tokens (DeepSeek-V2-Lite sizes, 48 of 64 experts resident,
// about 410 MB of weights) takes 83 us, its up launch at 5.4 TB/s of the 6.25 that a plain read reaches; one token
// (43 MB) the launches' starts and ends, 17 us; long buckets the matrix units (Qwen2 sizes, T = 4096, 3.6
// TOP: 2000 us with up at 1.95 and down at 1.80 POP/s, where a plain int8 product of 8192^3 reaches 2.13; the
// matrix units are busy for 46 and 43 % of the SIMDs' cycles).  In between (T = 1000, 152 us) neither: 2.75 rounds of
// blocks, matrix units busy for 16 and 14 %, 115 us even where every expert has the same weights, which L2 then holds.
// Kernels that kept a few tokens' rows in registers and streamed the weights past them, and weights and tokens
// loaded by different waves, were not faster for any T.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "lore_tile.h"
#include "route_last.h"
#include "spice_internal.h"

namespace spice {
namespace {

template <int BM_, int BT_, int WF_, int WT_, int S_, int SW_>
struct Shape {
    static constexpr int BM = BM_, BT = BT_, WF = WF_, WT = WT_;
    static constexpr int S = S_, SW = SW_;         // stages of tokens and of weights in LDS
    static constexpr int kThreads = 64 * WF * WT;
    static constexpr int kLoaders = 256;           // threads that issue the stages' loads
    static constexpr int RF = BM / WF / 16;        // 16-row sub-tiles per wave
    static constexpr int RT = BT / WT / 16;        // 16-token sub-tiles per wave
    static constexpr int kTStride = 16 * WT;       // tile rows between a wave's token sub-tiles
    static constexpr int kUpFeat = BM / 2;         // features of an up tile (W1 rows = W3 rows)
    static constexpr int kTopGroup = kUpFeat / WF; // features of a wave: those of a partial maximum of H
    static constexpr int kWTile = BM * 128;        // bytes of a stage's weight rows
    static constexpr int kXTile = BT * 128;        // and of its token rows
    static constexpr int kLds = SW * kWTile + S * kXTile;
    static constexpr int kRowStep = kLoaders / 8;  // rows one load instruction of the loaders covers
    static constexpr int kWLoads = BM / kRowStep, kXLoads = BT / kRowStep;
    static constexpr int kXcdBlocks = 32 * std::max(1, 163840 / kLds);  // resident blocks per XCD
    static constexpr int kAccs = RF * RT * 4;      // sums per thread
    static_assert(kRowStep % 16 == 0 && kUpFeat % kRowStep == 0, "staged rows keep their swizzle");
    static_assert(BM % kRowStep == 0 && (BT % kRowStep == 0 || BT < kRowStep), "whole load instructions");
    static_assert(SW == S || SW == S + 1, "weights are at most a stage ahead of the tokens");
    static_assert(S * (kWLoads + kXLoads) < 64, "vmcnt holds the loads in flight");
};
using Tile64x32 = Shape<64, 32, 2, 2, 4, 4>;
using OwnTile = Shape<64, 16, 4, 1, 4, 4>;  // down, a tile's own codes of H
using Tile128x64 = Shape<128, 64, 2, 2, 3, 3>;
using Tile128x128 = Shape<128, 128, 2, 4, 2, 3>;
using Tile256x256 = Shape<256, 256, 2, 4, 2, 3>;
template <class C>
constexpr bool matches(const I8Shape& s) {
    return C::BM == s.rows && C::BT == s.tokens && C::kLds == s.lds;
}
static_assert(matches<Tile64x32>(kI8Shapes[0]) && matches<Tile128x64>(kI8Shapes[1]) && matches<Tile128x128>(kI8Shapes[2]) &&
                  matches<Tile256x256>(kI8Shapes[3]),
              "the shapes as the rules know them");

constexpr int kBK = 128;                         // contraction per stage
constexpr uint32_t kOutOfRange = 0xFFFFFFF0u;    // an offset past every buffer
constexpr int kRawBufferWord3 = 0x00020000;      // gfx9 raw buffer: 32-bit data format

typedef int i32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));

__device__ __forceinline__ float silu(float u) { return u / (1.0f + __expf(-u)); }

__device__ __forceinline__ float max_or_nan(float a, float b) {
    return a != a || b != b ? __builtin_nanf("") : fmaxf(a, b);
}

// Factors from a row's values to its codes, by its maximum: lift, a power of two and exact, keeps 127 / top finite
// where top is tiny (below 3.7e-37 it would overflow); inv 0 for a row of zeros, or one that is not finite (top NaN).
struct CodeScale {
    float lift, inv;
};
__device__ __forceinline__ CodeScale code_scale(float top) {
    const float lift = top < 0x1p-96f ? 0x1p+96f : 1.f;
    return {lift, top > 0.f ? 127.f / (top * lift) : 0.f};
}

// Codes of 4 values.
__device__ __forceinline__ uint32_t pack_codes(const f32x4_t& v, CodeScale c) {
    uint32_t bits = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) bits |= (uint32_t)((int)rintf(c.inv == 0.f ? 0.f : v[k] * c.lift * c.inv) & 255) << (8 * k);
    return bits;
}

// Bytes of a row of K codes in whole stages; what an OwnTile block keeps in front of its rows.
__host__ __device__ constexpr int nk_pad(int K) { return (K + kBK - 1) / kBK * kBK; }
constexpr int kOwnTops = 64;

// Logical tile of block b: rounds of 8 x per_xcd blocks give each XCD (block b runs on XCD b % 8) per_xcd
// consecutive tiles, which share operands in that XCD's L2.  A bijection on [0, G).
__device__ __forceinline__ int xcd_tile(int b, int G, int per_xcd) {
    const int round = 8 * per_xcd;
    if (b >= (G / round) * round) return b;
    const int x = b & 7, slot = b >> 3;
    return (slot / per_xcd) * round + x * per_xcd + slot % per_xcd;
}

struct Job {
    FfnI8Args a;
    int32_t super[2];  // shared-block super-tile (weight tiles, token tiles)
    int32_t parts;     // splits of the shared block's down contraction
    int32_t lore;      // first blocks of the launch, which take the LORE tiles (a bound)
    int32_t xcd;       // whether neighbouring tiles run on one XCD
    int32_t group;     // features per partial maximum of H
    int32_t own_rows;  // rows of codes that an OwnTile block has room for
};

struct Tile {
    bool shared, lore;
    const void* w;        // the matrix's blob (A_e or B_e of a LORE tile)
    uint32_t w_bytes;     // of its codes
    int kdim, nfeat;      // bytes of a row (the contraction, but for a LORE tile), output features
    int up_off;           // up: rows from a tile row of the first half to its partner of the second
    int row0;             // first feature
    int tok0, ntok;       // first token of the tile in its group, tokens of the group
    int start;            // the group's first bucket position (0 for the shared block)
    int k0, k1;           // stages of the contraction this tile takes
    int split;            // which of the shared block's output tiles, where its contraction is split; or -1
    int part;             // and which part of it
};

// The bucket of class c holding tile L of nt tiles per token tile, by a wave's scan of the offsets; slot:
// its pool slot (class HIT).  A bucket outside the slots raises a flag and has no tiles, so it takes none of
// the grid's from the others.
__device__ bool find_bucket(const FfnI8Args& a, int c, int nt, int BT, int& L, int lane, int& e_, int& st_, int& n_,
                            int& slot_) {
    const int32_t* off = a.offsets + c * (a.N + 1);
    const uint32_t slots = (uint32_t)(a.T * a.K);
    for (int e0 = 0; e0 < a.N; e0 += 64) {
        const int e = e0 + lane;
        int st = 0, n = 0, slot = -1;
        if (e < a.N) {
            st = off[e];
            n = (int)((uint32_t)off[e + 1] - (uint32_t)st);
            if (c == SPICE_CLASS_HIT) slot = a.resident_slot[e];
            if ((uint32_t)st > slots || (uint32_t)n > slots - (uint32_t)st) {  // not inside the T K slots: no tiles
                atomicOr(&a.ctrl[kWordFlags], (uint32_t)SPICE_FLAG_BAD_INDEX);
                n = 0;
            }
        }
        const int tiles = n > 0 ? ((n + BT - 1) / BT) * nt : 0;
        int incl = tiles;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int up = __shfl_up(incl, o);
            if (lane >= o) incl += up;
        }
        const int excl = incl - tiles;
        const unsigned long long hit = __ballot(tiles > 0 && L >= excl && L < incl);
        if (hit) {
            const int src = __builtin_amdgcn_readfirstlane(__ffsll((long long)hit) - 1);
            e_ = e0 + src;
            st_ = __builtin_amdgcn_readlane(st, src);
            n_ = __builtin_amdgcn_readlane(n, src);
            slot_ = __builtin_amdgcn_readlane(slot, src);
            L -= __builtin_amdgcn_readlane(excl, src);
            return true;
        }
        L -= __builtin_amdgcn_readlane(incl, 63);
    }
    return false;
}

// Tile L of a matrix's nt weight tiles x mt token tiles: the token tiles of a weight tile are 8 blocks
// apart, so they run on one XCD, one after the other, and read the weights once into its L2.
__device__ __forceinline__ void spread(int L, int nt, int mt, int& w, int& t) {
    const int g = L / (8 * mt), wide = min(8, nt - 8 * g), in = L - g * 8 * mt;
    t = in / wide;
    w = 8 * g + in - t * wide;
}

// Logical tile L of a launch (every wave resolves it for itself): the LORE tiles in the first job.lore
// blocks, then the shared block's, in groups of about an XCD's blocks that share operand tiles in its L2,
// then the HIT buckets in id order, the token tiles of one weight tile next to each other.
template <bool kUp, class C>
__device__ bool resolve(const Job& job, int L, Tile& j) {
    const FfnI8Args& a = job.a;
    constexpr int feat = kUp ? C::kUpFeat : C::BM;
    j.k0 = 0;
    j.split = -1;
    j.part = 0;
    j.shared = j.lore = false;
    int e = 0, st = 0, n = 0, slot = -1;
    const int lane = threadIdx.x & 63;
    if (L < job.lore) {
        constexpr int rows = kUp ? C::BM : C::BM * kLoreDown;
        const int nt = ((kUp ? a.r : a.d) + rows - 1) / rows;
        if (!find_bucket(a, SPICE_CLASS_LORE, nt, C::BT, L, lane, e, st, n, slot)) return false;
        j.lore = true;
        j.w = (kUp ? a.lore_A : a.lore_B) + (size_t)e * a.r * a.d;
        j.w_bytes = (uint32_t)a.r * (uint32_t)a.d * 2u;
        j.kdim = kUp ? 2 * a.d : 2 * a.r;
        j.nfeat = kUp ? a.r : a.d;
        j.up_off = C::kUpFeat;  // BM consecutive rows of A
    } else {
        L -= job.lore;
        const int nt_sh = ((kUp ? a.Is : a.d) + feat - 1) / feat, nt_e = ((kUp ? a.I : a.d) + feat - 1) / feat;
        const int mt_sh = (a.T + C::BT - 1) / C::BT;
        const int parts = kUp ? 1 : job.parts, per_part = nt_sh * mt_sh;
        const int tiles_sh = a.Is > 0 ? per_part * parts : 0;
        if (L < tiles_sh) {
            j.part = L / per_part;
            L -= j.part * per_part;
            if (parts > 1) j.split = L;
            j.shared = true;
            j.w = kUp ? a.w13s : a.w2s;
            j.w_bytes = (uint32_t)(kUp ? 2 : 1) * (uint32_t)a.Is * (uint32_t)a.d;
            j.kdim = kUp ? a.d : a.Is;
            j.nfeat = kUp ? a.Is : a.d;
            j.up_off = j.nfeat;
            if (job.xcd) {
                const int sn = job.super[0], sm = job.super[1];
                const int g = L / (sn * sm), in = L - g * (sn * sm), mg = mt_sh / sm;
                j.row0 = ((g / mg) * sn + in / sm) * feat;
                j.tok0 = ((g % mg) * sm + in % sm) * C::BT;
            } else {
                spread(L, nt_sh, mt_sh, j.row0, j.tok0);
                j.row0 *= feat;
                j.tok0 *= C::BT;
            }
            j.ntok = a.T;
            j.start = 0;
            const int nk = (j.kdim + kBK - 1) / kBK;
            j.k0 = j.part * nk / parts;
            j.k1 = (j.part + 1) * nk / parts;
            return true;
        }
        L -= tiles_sh;
        if (a.C <= 0 || !find_bucket(a, SPICE_CLASS_HIT, nt_e, C::BT, L, lane, e, st, n, slot)) return false;
        if (slot < 0 || slot >= a.C) {
            if (threadIdx.x == 0) atomicOr(&a.ctrl[kWordFlags], (uint32_t)SPICE_FLAG_BAD_SLOT);
            return false;
        }
        const size_t elems = (size_t)(kUp ? 2 : 1) * a.I * a.d, rows = kUp ? 2 * (size_t)a.I : (size_t)a.d;
        j.w = (kUp ? a.w13_pool : a.w2_pool) + (size_t)slot * (elems + 4 * rows);
        j.w_bytes = (uint32_t)elems;
        j.kdim = kUp ? a.d : a.I;
        j.nfeat = kUp ? a.I : a.d;
        j.up_off = j.nfeat;
    }
    const int mt = (n + C::BT - 1) / C::BT, rows = !j.lore ? feat : kUp ? C::BM : C::BM * kLoreDown;
    if (job.xcd) {
        j.row0 = L / mt * rows;
        j.tok0 = L % mt * C::BT;
    } else {
        spread(L, (j.nfeat + rows - 1) / rows, mt, j.row0, j.tok0);
        j.row0 *= rows;
        j.tok0 *= C::BT;
    }
    j.ntok = n;
    j.start = st;
    j.k1 = (j.kdim + kBK - 1) / kBK;
    return true;
}

// Byte offset of 16-byte chunk c of staged row r inside an operand tile.
__device__ __forceinline__ uint32_t lds_off(int r, int c) {
    return (uint32_t)(r * 128 + ((c ^ ((r >> 1) & 7)) << 4));
}

typedef __amdgpu_buffer_rsrc_t rsrc_t;
__device__ __forceinline__ rsrc_t raw_buffer(const void* p, uint32_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, (int)bytes, kRawBufferWord3);
}

// 16 bytes from offset off of a buffer to LDS byte lds + 16 * lane, lds uniform over the wave (counted by
// vmcnt; an offset past the buffer writes zeros).  Device pass only: the host pass of a kernel naming
// this target builtin would lose its launch stub.
__device__ __forceinline__ void load_lds16(rsrc_t b, uint32_t off, unsigned char* lds) {
#if defined(__HIP_DEVICE_COMPILE__)
    __builtin_amdgcn_raw_ptr_buffer_load_lds(b, (__attribute__((address_space(3))) void*)lds, 16, (int)off, 0, 0, 0);
#endif
}

// s_waitcnt with vmcnt(n) lgkmcnt(0), then the block's barrier: no wait for loads to LDS beyond those
// the caller names (a __syncthreads would drain them all).
template <int n>
__device__ __forceinline__ void wait_and_barrier() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt((n & 15) | ((n >> 4) << 14) | 0x70);
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// Fragments of one 64-k step: RF weight sub-tiles and the NL live token sub-tiles.
template <class C, int NL>
struct Frags {
    i32x4_t a[C::RF], b[NL];
};

// The main loop of one tile with NL live token sub-tiles in this wave (NL = 0: the wave only loads and
// keeps the barriers).  kBf16: rows of bf16, 64 k per stage.  kOwn: the tokens' codes of all stages are in
// LDS, the lane's of stage kt at own(kt).
template <class C, bool kUp, bool kBf16, bool kOwn, int NL, class Load, class Own>
__device__ __forceinline__ void product(unsigned char* s_lds, int nk, uint32_t fbase, uint32_t tbase, Load load, Own own,
                                        i32x4_t (&acc)[C::RF][C::RT]) {
    constexpr int N1 = NL > 0 ? NL : 1;
    // loads in flight past the next stage's: whole stages, and the last weights issued, which are a stage ahead
    constexpr int kLoads = (C::S - 2) * (C::kWLoads + C::kXLoads) + (C::SW - C::S) * C::kWLoads;
    auto read = [&](int kt, int wbuf, int xbuf, uint32_t kx, Frags<C, N1>& f) {
        if constexpr (NL > 0) {
            const unsigned char* wbase = s_lds + wbuf * C::kWTile;
            const unsigned char* xbase = s_lds + C::SW * C::kWTile + xbuf * C::kXTile;
#pragma unroll
            for (int t = 0; t < NL; ++t)
                f.b[t] = *reinterpret_cast<const i32x4_t*>(kOwn ? s_lds + own(kt) + kx
                                                                : xbase + ((tbase + t * C::kTStride * 128) ^ kx));
#pragma unroll
            for (int s = 0; s < C::RF; ++s) {
                const int row = kUp ? (s % (C::RF / 2)) * 16 + (s / (C::RF / 2)) * C::kUpFeat : s * 16;
                f.a[s] = *reinterpret_cast<const i32x4_t*>(wbase + ((fbase + row * 128) ^ kx));
            }
        }
    };
    auto mma = [&](const Frags<C, N1>& f) {
        if constexpr (NL > 0) {
            __builtin_amdgcn_s_setprio(1);  // favour the wave that is issuing MFMAs
#pragma unroll
            for (int t = 0; t < NL; ++t)
#pragma unroll
                for (int s = 0; s < C::RF; ++s) {
                    if constexpr (kBf16)  // a LORE tile's sums are fp32, in the same registers
                        acc[s][t] = __builtin_bit_cast(
                            i32x4_t, __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                                         __builtin_bit_cast(bf16x8_t, f.a[s]), __builtin_bit_cast(bf16x8_t, f.b[t]),
                                         __builtin_bit_cast(f32x4_t, acc[s][t]), 0, 0, 0));
                    else
                        acc[s][t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(f.a[s], f.b[t], acc[s][t], 0, 0, 0);
                }
            __builtin_amdgcn_s_setprio(0);
        }
    };
    wait_and_barrier<kLoads + C::kWLoads + C::kXLoads>();  // stage 0 of the S in flight has landed
    Frags<C, N1> f0, f1;
    read(0, 0, 0, 0u, f0);
    int wbuf = 0, xbuf = 0;
    for (int kt = 0; kt < nk; ++kt) {
        read(kt, wbuf, xbuf, 64u, f1);
        __builtin_amdgcn_sched_barrier(0);
        mma(f0);
        __builtin_amdgcn_sched_barrier(0);
        // stage kt + 1 has landed and every wave has read all of stage kt
        wait_and_barrier<kLoads>();
        load(wbuf, xbuf, kt);
        wbuf = wbuf + 1 == C::SW ? 0 : wbuf + 1;
        xbuf = xbuf + 1 == C::S ? 0 : xbuf + 1;
        read(kt + 1, wbuf, xbuf, 0u, f0);  // past the last stage: zeros, unused
        __builtin_amdgcn_sched_barrier(0);
        mma(f1);
        __builtin_amdgcn_sched_barrier(0);
    }
    __builtin_amdgcn_s_waitcnt(0x70);  // no load to LDS outlives the block
}

// Token of slot s (token 0 and a flag for a slot out of range).
__device__ __forceinline__ int slot_token(const FfnI8Args& a, int s) {
    if (s < 0 || s >= a.T * a.K) {
        atomicOr(&a.ctrl[kWordFlags], (uint32_t)SPICE_FLAG_BAD_INDEX);
        return 0;
    }
    return s / a.K;
}

// Leaves a part's sums at the device-coherent level and counts it; true for the last of the tile's parts,
// whose acc then holds the sum of all.
template <class C>
__device__ __forceinline__ bool split_sums(const FfnI8Args& a, int parts, int tile, int mine, int32_t* part,
                                           i32x4_t (&acc)[C::RF][C::RT], int* s_last) {
    int32_t* own = part + (size_t)mine * C::kAccs * C::kThreads;
#pragma unroll
    for (int s = 0; s < C::RF; ++s)
#pragma unroll
        for (int t = 0; t < C::RT; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                __hip_atomic_store(own + ((s * C::RT + t) * 4 + i) * C::kThreads, acc[s][t][i], __ATOMIC_RELAXED,
                                   __HIP_MEMORY_SCOPE_AGENT);
    if (!route_last_block(&a.ctrl[kWordI8Parts + tile], parts, s_last)) return false;
    for (int p = 0; p < parts; ++p) {
        if (p == mine) continue;
        const int32_t* other = part + (size_t)p * C::kAccs * C::kThreads;
#pragma unroll
        for (int s = 0; s < C::RF; ++s)
#pragma unroll
            for (int t = 0; t < C::RT; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    acc[s][t][i] += __hip_atomic_load(other + ((s * C::RT + t) * 4 + i) * C::kThreads, __ATOMIC_RELAXED,
                                                      __HIP_MEMORY_SCOPE_AGENT);
    }
    return true;
}

template <bool kUp, class C, bool kOwn>
__global__ __launch_bounds__(C::kThreads) __attribute__((amdgpu_waves_per_eu(2))) void i8_gemm_kernel(Job job) {
    extern __shared__ __align__(16) unsigned char s_lds[];
    const FfnI8Args& a = job.a;
    Tile j;
    if (!resolve<kUp, C>(job, job.xcd ? xcd_tile(blockIdx.x, gridDim.x, C::kXcdBlocks) : (int)blockIdx.x, j)) return;
    if constexpr (!kUp) {
        if (j.lore) {
            for (int b = 0; b < kLoreDown && j.row0 < a.d; ++b, j.row0 += C::BM) lore_down<C>(a, j);
            return;
        }
    }
    const int tid = threadIdx.x, lane = tid & 63;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wf = w % C::WF, wt = w / C::WF;  // wave's feature part and token lane group
    const int m = lane & 15, quad = lane >> 4;
    const int frow0 = wf * ((kUp ? C::kUpFeat : C::BM) / C::WF);
    // token sub-tiles of this wave with a live row
    const int nlive = min(C::RT, max(0, (j.ntok - j.tok0 - 16 * wt + C::kTStride - 1) / C::kTStride));
    i32x4_t acc[C::RF][C::RT];
#pragma unroll
    for (int s = 0; s < C::RF; ++s)
#pragma unroll
        for (int t = 0; t < C::RT; ++t) acc[s][t] = i32x4_t{0, 0, 0, 0};

    // Staging: a loader wave's load writes 64 x 16 bytes to consecutive LDS, 8 staged rows of 8 chunks.
    // Lane l fills LDS chunk l % 8 of row r0 = tid / 8 (+ kRowStep i), which holds the row's chunk
    // (l % 8) ^ swizzle(row), so that is the chunk it fetches.
    const int r0 = tid / 8;
    const bool loader = C::kLoaders == C::kThreads || tid < C::kLoaders;
    const int c16 = (int)((lds_off(r0, tid & 7) & 127u) >> 4);
    const uint32_t ldx = kUp ? (uint32_t)j.kdim : (uint32_t)i8_row(j.kdim);
    // up: all tokens' rows (1 GiB at most); down: the tile's, which are consecutive
    const size_t row_first = (size_t)j.start + j.tok0;
    const rsrc_t wbuf = raw_buffer(j.w, j.w_bytes);
    const rsrc_t xbuf = kUp ? raw_buffer(j.lore ? static_cast<const void*>(a.x) : a.xq, (uint32_t)a.T * ldx)
                            : raw_buffer((j.shared ? a.hqs : a.hq) + row_first * ldx, (uint32_t)min(C::BT, j.ntok - j.tok0) * ldx);
    const uint32_t wstep = (uint32_t)j.kdim;
    const uint32_t woff0 = (uint32_t)(j.row0 + r0) * wstep + c16 * 16;
    const int klim = j.kdim - c16 * 16;  // the lane's chunk of stage kt is in the row while 128 kt < klim
    const int nk = j.k1 - j.k0;
    // Weight rows whose stride is a multiple of 2 KiB start on a few memory channels only: each weight
    // tile starts its k order at another stage.
    const int rot = wstep % 2048 == 0 ? (int)((uint32_t)(j.row0 / C::kUpFeat) * 5u % (uint32_t)nk) : 0;
    // stage kt of the tile's nk; past the last one, a stage past the row
    auto stage_k = [&](int kt) { return kt >= nk ? 0x800000 : j.k0 + (kt + rot >= nk ? kt + rot - nk : kt + rot); };
    auto load_w = [&](int buf, int kt) {
        if (!loader) return;
        unsigned char* run = s_lds + buf * C::kWTile + w * 1024;
        kt = stage_k(kt);
        const bool in = kt * kBK < klim;
#pragma unroll
        for (int i = 0; i < C::kWLoads; ++i) {
            const int r = C::kRowStep * i;
            const uint32_t delta = (uint32_t)(kUp && r >= C::kUpFeat ? j.up_off + r - C::kUpFeat : r) * wstep;
            load_lds16(wbuf, in ? woff0 + delta + (uint32_t)kt * kBK : kOutOfRange, run + i * C::kRowStep * 128);
        }
    };
    constexpr int kXN = C::kXLoads > 0 ? C::kXLoads : 1;
    uint32_t xoff[kXN];
    auto load_x = [&](int buf, int kt) {
        if (!loader) return;
        unsigned char* run = s_lds + C::SW * C::kWTile + buf * C::kXTile + w * 1024;
        kt = stage_k(kt);
        const bool in = kt * kBK < klim;
#pragma unroll
        for (int i = 0; i < C::kXLoads; ++i)
            load_lds16(xbuf, in && xoff[i] != kOutOfRange ? xoff[i] + (uint32_t)kt * kBK : kOutOfRange,
                       run + i * C::kRowStep * 128);
    };
    // what takes the place of stage kt, the tokens first: a wait for them by count leaves the weights in flight
    auto load = [&](int wbuf, int xbuf, int kt) {
        load_x(xbuf, kt + C::S);
        load_w(wbuf, kt + C::SW);
    };
    // the slot ids of the tile's rows, the weights of stage 0, then (once the ids are there) its token
    // rows and the other stages of the ring
    int sid[kXN];
#pragma unroll
    for (int i = 0; i < C::kXLoads; ++i) {
        const int pos = j.tok0 + r0 + C::kRowStep * i;
        sid[i] = -1;
        if (loader && pos < j.ntok) sid[i] = !kUp ? pos - j.tok0 : j.shared ? pos : a.perm[j.start + pos];
    }
    // What the epilogue needs is on its way before the ring's first loads (a wait by count then waits for
    // it too): the scales of the wave's weight rows and of its tokens, else one or two trips to memory at
    // the end of a short tile.
    constexpr bool kEarly = C::RF <= 4;  // registers: the scales of a 256-row tile are loaded late
    const float* scales = reinterpret_cast<const float*>(static_cast<const char*>(j.w) + j.w_bytes);
    auto row_scale = [&](int s) {
        const int f = j.row0 + frow0 + (kUp ? s % (C::RF / 2) : s) * 16 + quad * 4;
        return *reinterpret_cast<const f32x4_t*>(scales + (f < j.nfeat ? f : 0) + (kUp && s >= C::RF / 2 ? j.nfeat : 0));
    };
    auto row_id = [&](int t) {
        const int p = min(j.tok0 + t * C::kTStride + wt * 16 + m, j.ntok - 1);
        return !kUp || j.shared ? p : a.perm[j.start + p];
    };
    auto row_factor = [&](int id) {
        if constexpr (kUp) {
            return a.xs[j.shared ? id : slot_token(a, id)];
        } else {
            const size_t pos = (size_t)j.start + id;
            return (kOwn ? 1.f : (j.shared ? a.hscale_s : a.hscale)[pos]) * (j.shared && a.sgate ? a.sgate[pos] : 1.f);
        }
    };
    f32x4_t sc[C::RF];
    int rid[C::RT];
    float factor[C::RT];
    if constexpr (kEarly) {
#pragma unroll
        for (int s = 0; s < C::RF; ++s)
            if (!j.lore) sc[s] = row_scale(s);
#pragma unroll
        for (int t = 0; t < C::RT; ++t) rid[t] = row_id(t);
    }
    // kOwn: the waves make the codes of the rows as the quantisation launch does, a wave each, or a half or a
    // quarter of one or two rows; the first values come before the ring's first loads
    const int own_rows = kOwn ? min(min(j.ntok - j.tok0, C::BT), job.own_rows) : 0, nv = j.kdim / 4;
    const int own_ld = nk_pad(j.kdim) + 16, segs = own_rows == 1 ? 4 : own_rows == 2 ? 2 : 1;
    const int v_all = j.k0 * (kBK / 4), v_end = min(j.k1 * (kBK / 4), nv), seg_len = (v_end - v_all + segs - 1) / segs;
    float* s_top = reinterpret_cast<float*>(s_lds + C::SW * C::kWTile);
    constexpr int kOwnVec = 6;
    f32x4_t hv[kOwnVec];
    float hp = 0.f;
    auto own_load = [&](int it) {
        const int row = it / segs, v0 = v_all + it % segs * seg_len;
        const float* part = (j.shared ? a.top_s : a.top) + (row_first + row) * (j.kdim / 16);
        const int np = (j.kdim + job.group - 1) / job.group;
        hp = 0.f;
        for (int i = lane; i < np; i += 64) hp = max_or_nan(hp, part[i]);
        const f32x4_t* hr = reinterpret_cast<const f32x4_t*>((j.shared ? a.hs : a.h) + (row_first + row) * j.kdim);
#pragma unroll
        for (int c = 0; c < kOwnVec; ++c) hv[c] = hr[min(v0 + lane + 64 * c, nv - 1)];
    };
    auto own_store = [&](int it) {
        const int row = it / segs, v0 = v_all + it % segs * seg_len, v1 = min(v0 + seg_len, v_end);
        float top = hp;
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) top = max_or_nan(top, __shfl_xor(top, o));
        if (lane == 0) s_top[row] = top / 127.f;
        const CodeScale scale = code_scale(top);
        const f32x4_t* hr = reinterpret_cast<const f32x4_t*>((j.shared ? a.hs : a.h) + (row_first + row) * j.kdim);
        uint32_t* codes = reinterpret_cast<uint32_t*>(s_lds + C::SW * C::kWTile + kOwnTops + row * own_ld);
#pragma unroll
        for (int c = 0; c < kOwnVec; ++c) {
            const int i = v0 + lane + 64 * c;
            if (i < v1) codes[i] = pack_codes(hv[c], scale);
        }
        for (int i = v0 + lane + 64 * kOwnVec; i < v1; i += 64) codes[i] = pack_codes(hr[i], scale);
    };
    if constexpr (kOwn) {
        if (w < own_rows * segs) own_load(w);
    }
    __builtin_amdgcn_sched_barrier(0);
    load_w(0, 0);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < C::kXLoads; ++i) {
        const int pos = j.tok0 + r0 + C::kRowStep * i;
        xoff[i] = kOutOfRange;
        if (loader && pos < j.ntok) xoff[i] = (uint32_t)(!kUp || j.shared ? sid[i] : slot_token(a, sid[i])) * ldx + c16 * 16;
    }
    load_x(0, 0);
    if constexpr (kEarly) {
#pragma unroll
        for (int t = 0; t < C::RT; ++t) factor[t] = row_factor(rid[t]);
    }
#pragma unroll
    for (int s = 1; s < C::SW; ++s) {
        load_w(s, s);
        if (s < C::S) load_x(s, s);
    }

    if constexpr (kOwn) {
        for (int it = w; it < own_rows * segs; it += C::kThreads / 64) {
            if (it != w) own_load(it);
            own_store(it);
        }
    }
    const uint32_t own_row = C::SW * C::kWTile + kOwnTops + (m < own_rows ? m : 0) * own_ld + quad * 16;
    auto own = [&](int kt) { return own_row + (uint32_t)(kt < nk ? stage_k(kt) : j.k0) * kBK; };

    // LDS addresses of the fragments of k-step 0 (k-step 1 reads chunk c ^ 4: bit 6 flipped).  The swizzle
    // of row r depends on (r >> 1) & 7, which steps of 16 rows leave unchanged.
    const uint32_t fbase = lds_off(frow0 + m, quad);
    const uint32_t tbase = lds_off(wt * 16 + m, quad);
    static_assert(C::RT == 1 || C::RT == 2 || C::RT == 4, "token sub-tiles per wave");
    auto multiply = [&](auto bf16) {
        constexpr bool kBf16 = decltype(bf16)::value;
        if (nlive == C::RT) product<C, kUp, kBf16, kOwn, C::RT>(s_lds, nk, fbase, tbase, load, own, acc);
        else if (nlive == 0) product<C, kUp, kBf16, kOwn, 0>(s_lds, nk, fbase, tbase, load, own, acc);
        else if constexpr (C::RT > 2) {
            if (nlive == 1) product<C, kUp, kBf16, kOwn, 1>(s_lds, nk, fbase, tbase, load, own, acc);
            else if (nlive == 2) product<C, kUp, kBf16, kOwn, 2>(s_lds, nk, fbase, tbase, load, own, acc);
            else product<C, kUp, kBf16, kOwn, 3>(s_lds, nk, fbase, tbase, load, own, acc);
        } else if constexpr (C::RT > 1) {
            product<C, kUp, kBf16, kOwn, 1>(s_lds, nk, fbase, tbase, load, own, acc);
        }
    };
    if constexpr (kUp) {
        if (j.lore) {
            multiply(std::true_type{});
#pragma unroll
            for (int t = 0; t < C::RT; ++t) {
                const int p = j.tok0 + t * C::kTStride + wt * 16 + m;
                if (p >= j.ntok) continue;
                float* dst = a.u + (size_t)(j.start + p) * a.r;
#pragma unroll
                for (int s = 0; s < C::RF; ++s) {
                    const int q = j.row0 + frow0 + (s % (C::RF / 2)) * 16 + (s / (C::RF / 2)) * C::kUpFeat + quad * 4;
                    if (q < a.r) *reinterpret_cast<i32x4_t*>(dst + q) = acc[s][t];
                }
            }
            return;
        }
    }
    multiply(std::false_type{});

    if constexpr (!kUp) {
        if (j.split >= 0) {
            // the last of the tile's parts to arrive adds the others' sums to its own (exact: in any order)
            int32_t* part = a.part + (size_t)j.split * job.parts * C::kAccs * C::kThreads + tid;
            if (!split_sums<C>(a, job.parts, j.split, j.part, part, acc, reinterpret_cast<int*>(s_lds))) return;
        }
    }

    // Epilogue: lane holds features 4 quad .. + 3 of sub-tile s for token m of sub-tile t.
#pragma unroll
    for (int t = 0; t < C::RT; ++t) {
        const int p = j.tok0 + t * C::kTStride + wt * 16 + m;
        if (p >= j.ntok) continue;
        const size_t pos = (size_t)j.start + p;
        if constexpr (kUp) {
            const float sx = kEarly ? factor[t] : row_factor(row_id(t));
            float* dst = (j.shared ? a.hs : a.h) + pos * j.nfeat;
            float top = 0.f, bad = 0.f;  // bad: NaN once a value is not finite
#pragma unroll
            for (int s = 0; s < C::RF / 2; ++s) {
                const int f = j.row0 + frow0 + s * 16 + quad * 4;
                if (f >= j.nfeat) continue;
                const f32x4_t sg = kEarly ? sc[s] : row_scale(s), su = kEarly ? sc[s + C::RF / 2] : row_scale(s + C::RF / 2);
                f32x4_t h;
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    h[i] = silu((float)acc[s][t][i] * (sx * sg[i])) * ((float)acc[s + C::RF / 2][t][i] * (sx * su[i]));
                *reinterpret_cast<f32x4_t*>(dst + f) = h;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    top = fmaxf(top, fabsf(h[i]));
                    bad = fmaf(h[i], 0.f, bad);
                }
            }
            // the row's partial maximum over the wave's features
            top += bad;
            top = max_or_nan(top, __shfl_xor(top, 16));
            top = max_or_nan(top, __shfl_xor(top, 32));
            const int f0 = j.row0 + frow0;
            if (quad == 0 && f0 < j.nfeat) (j.shared ? a.top_s : a.top)[pos * (j.nfeat / 16) + f0 / C::kTopGroup] = top;
        } else {
            float sh = kEarly ? factor[t] : row_factor(row_id(t));
            if constexpr (kOwn) sh *= s_top[m < own_rows ? m : 0];
            float* dst = (j.shared ? a.y_shared : a.y_slots) + pos * a.d;
#pragma unroll
            for (int s = 0; s < C::RF; ++s) {
                const int f = j.row0 + frow0 + s * 16 + quad * 4;
                if (f >= a.d) continue;
                const f32x4_t s2 = kEarly ? sc[s] : row_scale(s);
                f32x4_t y;
#pragma unroll
                for (int i = 0; i < 4; ++i) y[i] = (float)acc[s][t][i] * (sh * s2[i]);
                *reinterpret_cast<f32x4_t*>(dst + f) = y;
            }
        }
    }
}

// Rows of H to 8 bits: a block per kQuantRow values of a row, the T shared rows first, then the HIT slots'
// positions.  The row's maximum comes from the partial maxima that the up tiles left, one per `group`
// features, so a row's blocks need not wait for each other; the values are on their way meanwhile.  Bound by
// memory: Qwen2 sizes, T = 4096, 671 MB read and 168 MB written in 148 us, 5.7 TB/s; a few rows take 4 us, little
// more than a launch's own time.
constexpr int kQuantThreads = 256;
constexpr int kQuantVec = 4;  // 16-byte chunks per thread
constexpr int kQuantRow = kQuantVec * 4 * kQuantThreads;
__global__ __launch_bounds__(kQuantThreads) void i8_quant_kernel(FfnI8Args a, int nsh, int segs_sh, int segs, int group) {
    __shared__ float s_top[kQuantThreads / 64];
    const bool shared = (int)blockIdx.x < nsh * segs_sh;
    const int b = shared ? blockIdx.x : blockIdx.x - nsh * segs_sh, per = shared ? segs_sh : segs;
    const int row = b / per, seg = b - row * per;
    if (!shared && (uint32_t)row >= (uint32_t)a.offsets[a.N]) return;  // the HIT buckets' end
    const int tid = threadIdx.x, n = shared ? a.Is : a.I, nv = n / 4, nt = (n + group - 1) / group;
    const f32x4_t* h = reinterpret_cast<const f32x4_t*>((shared ? a.hs : a.h) + (size_t)row * n);
    const float* part = (shared ? a.top_s : a.top) + (size_t)row * (n / 16);
    uint32_t* q = reinterpret_cast<uint32_t*>((shared ? a.hqs : a.hq) + (size_t)row * i8_row(n));
    const int i0 = seg * (kQuantRow / 4) + tid;
    f32x4_t v[kQuantVec];
#pragma unroll
    for (int c = 0; c < kQuantVec; ++c)
        if (c == 0 || seg * (kQuantRow / 4) + c * kQuantThreads < nv) v[c] = h[min(i0 + c * kQuantThreads, nv - 1)];
    float top = 0.f;
    for (int i = tid; i < nt; i += kQuantThreads) top = max_or_nan(top, part[i]);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) top = max_or_nan(top, __shfl_xor(top, o));
    if ((tid & 63) == 0) s_top[tid >> 6] = top;
    __syncthreads();
    top = s_top[0];
#pragma unroll
    for (int i = 1; i < kQuantThreads / 64; ++i) top = max_or_nan(top, s_top[i]);
    if (tid == 0 && seg == 0) (shared ? a.hscale_s : a.hscale)[row] = top / 127.f;
    // a row that is not finite has a maximum of NaN: codes 0, and the scale NaN
    const CodeScale scale = code_scale(top);
#pragma unroll
    for (int c = 0; c < kQuantVec; ++c) {
        const int i = i0 + c * kQuantThreads;
        if (i >= nv) break;
        q[i] = pack_codes(v[c], scale);
    }
}

// Super-tile of the shared block: sn weight tiles x sm token tiles with sn | nt and sm | mt, at most one
// XCD's resident blocks, as square as possible.
void super_shape(int mt, int nt, int most, int32_t* out) {
    int best_n = 1, best_m = 1, best_score = -1;
    for (int sm = 1; sm <= mt && sm <= most; ++sm) {
        if (mt % sm) continue;
        for (int sn = 1; sn <= nt && sn * sm <= most; ++sn) {
            if (nt % sn) continue;
            const int score = sn * sm * 64 - (sn + sm);
            if (score > best_score) { best_score = score; best_n = sn; best_m = sm; }
        }
    }
    out[0] = best_n;
    out[1] = best_m;
}

long long tiles_of(long long n, int per) { return (n + per - 1) / per; }

template <bool kUp, class C, bool kOwn = false>
hipError_t launch_pass(const FfnI8Args& a, const I8Plan& plan, int group, int own_bytes, hipStream_t s) {
    constexpr int feat = kUp ? C::kUpFeat : C::BM;
    // HIT buckets at most.  Experts may share a pool slot, so there can be more than C (a grid for C of them / this, us
    // per call with 40 and 48 of 64 experts resident: a layer's T = 16 82.4 / 81.2, T = 32 88.1 / 87.1).
    const long long slots = (long long)a.T * a.K, buckets = a.C > 0 ? std::min<long long>(a.N, slots) : 0;
    const long long nt_sh = tiles_of(kUp ? a.Is : a.d, feat), nt_e = tiles_of(kUp ? a.I : a.d, feat);
    Job job{a, {1, 1}, kUp || !a.part ? 1 : plan.parts, 0, plan.xcd, group, (int)std::min<long long>(slots, C::BT)};
    const long long lore_b = a.r > 0 ? std::min<long long>(a.N, slots) : 0;
    const long long lore = lore_b ? (slots / C::BT + lore_b) * tiles_of(kUp ? a.r : a.d, kUp ? C::BM : C::BM * kLoreDown) : 0;
    // upper bound: sum_e ceil(n_e / BT) <= buckets + (slots - buckets) / BT; blocks past the live tiles exit
    const long long tiles = (a.Is > 0 ? tiles_of(a.T, C::BT) * nt_sh * job.parts : 0) +
                            (buckets > 0 ? (buckets + (slots - buckets) / C::BT) * nt_e : 0) + lore;
    if (tiles == 0) return hipSuccess;
    if (tiles > 0x7FFFFFFFll) return hipErrorInvalidValue;
    job.lore = (int32_t)lore;
    if (a.Is > 0 && plan.xcd) super_shape((int)tiles_of(a.T, C::BT), (int)nt_sh, C::kXcdBlocks, job.super);
    hipLaunchKernelGGL((i8_gemm_kernel<kUp, C, kOwn>), dim3((unsigned)tiles), dim3(C::kThreads),
                       kOwn ? C::SW * C::kWTile + kOwnTops + own_bytes : C::kLds, s, job);
    return hipGetLastError();
}

hipError_t launch_quant(const FfnI8Args& a, int group, hipStream_t s) {
    const long long nsh = a.Is > 0 ? a.T : 0, slots = a.C > 0 ? (long long)a.T * a.K : 0;
    const long long segs_sh = (a.Is + kQuantRow - 1) / kQuantRow, segs = (a.I + kQuantRow - 1) / kQuantRow;
    const long long blocks = nsh * segs_sh + slots * segs;
    if (blocks > 0x7FFFFFFFll) return hipErrorInvalidValue;
    if (blocks == 0) return hipSuccess;
    hipLaunchKernelGGL(i8_quant_kernel, dim3((unsigned)blocks), dim3(kQuantThreads), 0, s, a, (int)nsh, (int)segs_sh, (int)segs,
                       group);
    return hipGetLastError();
}

// A few short rows need no launch of their own: each down tile makes their codes for itself, while its
// weights are on their way.  us per call with the launch / without: d = 512, 16 experts of 256, shared 512,
// T = 1 14.3 / 10.1, T = 8 14.3 / 11.2; DeepSeek-V2-Lite sizes T = 1 22.5 / 20.2, T = 2 26.0 / 23.2; Qwen2 sizes
// T = 1 86.4 / 83.9.  Bytes of the rows that a block holds at most, or 0 where three blocks of a CU have no
// room for them (with two, T = 4 37.4 / 36.5, T = 12 65.6 / 68.1) or the tokens do not fit the tile.
int own_bytes(const FfnI8Args& a) {
    const long long rows = std::min<long long>((long long)a.T * a.K, OwnTile::BT);
    const long long bytes = std::max(a.Is > 0 ? (long long)a.T * (nk_pad(a.Is) + 16) : 0, rows * (nk_pad(a.I) + 16));
    return a.T <= OwnTile::BT && bytes <= 163840 / 3 - OwnTile::SW * OwnTile::kWTile - kOwnTops ? (int)bytes : 0;
}

template <class C>
hipError_t launch_all(const FfnI8Args& a, const I8Plan& plan, hipStream_t s) {
    hipError_t e = launch_pass<true, C>(a, plan, C::kTopGroup, 0, s);
    if constexpr (std::is_same_v<C, Tile64x32>) {
        const int own = own_bytes(a);
        if (e == hipSuccess && own > 0) return launch_pass<false, OwnTile, true>(a, plan, C::kTopGroup, own, s);
    }
    if (e == hipSuccess) e = launch_quant(a, C::kTopGroup, s);
    return e == hipSuccess ? launch_pass<false, C>(a, plan, C::kTopGroup, 0, s) : e;
}

}  // namespace

hipError_t launch_expert_ffn_i8(const FfnI8Args& a, hipStream_t s) {
    const I8Plan plan = i8_plan(a.T, a.d, a.N, a.K, a.C, a.I, a.Is);
    switch (plan.shape) {
        case 0: return launch_all<Tile64x32>(a, plan, s);
        case 1: return launch_all<Tile128x64>(a, plan, s);
        case 2: return launch_all<Tile128x128>(a, plan, s);
        default: return launch_all<Tile256x256>(a, plan, s);
    }
}

}  // namespace spice
