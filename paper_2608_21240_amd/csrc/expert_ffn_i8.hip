// Grouped SwiGLU FFN of the HIT experts' buckets and of the shared block with 8-bit weights and
// activations (moe_expert_ffn_grouped_i8), three launches:
//
//   up    : H[pos][f] = silu(sx s1[f] sum_k W1[f][k] x[k]) * (sx s3[f] sum_k W3[f][k] x[k])  (fp32)
//   quant : per row of H, sh = max |h| / 127 and qh = round(h / sh)                          (int8)
//   down  : Y[pos][j] = sh s2[j] sum_k W2[j][k] qh[k]                                         (fp32)
//
// The sums are int32 MFMAs (v_mfma_i32_16x16x64_i8) and exact, whatever their order; H stays fp32
// until its row's maximum is known, so its only rounding to 8 bits is the one the format has.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "spice_internal.h"

namespace spice {
namespace {

typedef int i32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256, kWaves = 4;
constexpr int kTok = 16;  // tokens of a tile

__device__ __forceinline__ float silu(float u) { return u / (1.0f + __expf(-u)); }

// A tile of a launch: which matrix, which rows of it and which tokens.
struct Tile {
    bool shared;
    const char* w;       // the matrix's blob: codes, then the scales of its rows
    int row0;            // first feature
    int tok0, ntok;      // first token of the tile in its group, tokens of the group
    int start;           // the group's first bucket position (0 for the shared block)
};

// The HIT bucket that holds tile L, of nt weight tiles per token tile, found by a wave's scan of the
// offsets (uniform results); false past the last one.
__device__ bool find_bucket(const FfnI8Args& a, int nt, int& L, int& e_, int& st_, int& n_) {
    const int lane = threadIdx.x & 63;
    const int32_t* off = a.offsets + SPICE_CLASS_HIT * (a.N + 1);
    for (int e0 = 0; e0 < a.N; e0 += 64) {
        const int e = e0 + lane;
        int st = 0, n = 0;
        if (e < a.N) {
            st = off[e];
            n = off[e + 1] - st;
        }
        if (n > a.T * a.K) n = 0;
        const int tiles = n > 0 ? ((n + kTok - 1) / kTok) * nt : 0;
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
            L -= __builtin_amdgcn_readlane(excl, src);
            return true;
        }
        L -= __builtin_amdgcn_readlane(incl, 63);
    }
    return false;
}

template <bool kUp, int kFeat>
__device__ bool find_tile(const FfnI8Args& a, int L, Tile& t) {
    const int mt_sh = (a.T + kTok - 1) / kTok;
    const int nt_sh = ((kUp ? a.Is : a.d) + kFeat - 1) / kFeat, nt_e = ((kUp ? a.I : a.d) + kFeat - 1) / kFeat;
    const int tiles_sh = a.Is > 0 ? nt_sh * mt_sh : 0;
    if (L < tiles_sh) {
        t.shared = true;
        t.w = kUp ? a.w13s : a.w2s;
        t.row0 = L / mt_sh * kFeat;
        t.tok0 = L % mt_sh * kTok;
        t.ntok = a.T;
        t.start = 0;
        return true;
    }
    L -= tiles_sh;
    int e, st, n;
    if (a.C <= 0 || !find_bucket(a, nt_e, L, e, st, n)) return false;
    const int slot = a.resident_slot[e];
    if (st < 0 || st + n > a.T * a.K || slot < 0 || slot >= a.C) {
        if (threadIdx.x == 0)
            atomicOr(&a.ctrl[kWordFlags], (uint32_t)(slot < 0 || slot >= a.C ? SPICE_FLAG_BAD_SLOT : SPICE_FLAG_BAD_INDEX));
        return false;
    }
    const int mt = (n + kTok - 1) / kTok;
    const size_t elems = (size_t)(kUp ? 2 : 1) * a.I * a.d, rows = kUp ? 2 * (size_t)a.I : (size_t)a.d;
    t.shared = false;
    t.w = (kUp ? a.w13_pool : a.w2_pool) + (size_t)slot * (elems + 4 * rows);
    t.row0 = L / mt * kFeat;
    t.tok0 = L % mt * kTok;
    t.ntok = n;
    t.start = st;
    return true;
}

constexpr int kDepth = 4;  // 64-byte steps in flight per wave and row stream

// Sums of NR row streams (16 rows each, 16 bytes per lane and step) with 16 tokens, over the wave's
// share of the contraction; lane (m, quad) holds bytes 16 quad .. 16 quad + 15 of a step of row m and
// token m.  Bytes past the row are read as the row's first ones, with the token's taken as 0.
template <int NR>
__device__ __forceinline__ void wave_sums(const char* const (&wr)[NR], const char* xr, bool live, int K, i32x4_t (&acc)[NR]) {
    const int lane = threadIdx.x & 63, quad = lane >> 4;
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int nst = (K + 63) / 64, s0 = w * nst / kWaves, s1 = (w + 1) * nst / kWaves;
    for (int s = s0; s < s1; s += kDepth) {
        i32x4_t wv[kDepth][NR], xv[kDepth];
#pragma unroll
        for (int u = 0; u < kDepth; ++u) {
            const int k = (s + u) * 64 + quad * 16;
            const bool in = s + u < s1 && k < K;
            const int at = in ? k : 0;
#pragma unroll
            for (int r = 0; r < NR; ++r) wv[u][r] = *reinterpret_cast<const i32x4_t*>(wr[r] + at);
            xv[u] = i32x4_t{0, 0, 0, 0};
            if (in && live) xv[u] = *reinterpret_cast<const i32x4_t*>(xr + k);
        }
#pragma unroll
        for (int u = 0; u < kDepth; ++u)
#pragma unroll
            for (int r = 0; r < NR; ++r) acc[r] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wv[u][r], xv[u], acc[r], 0, 0, 0);
    }
}

// Up: 16 features (16 gate and 16 up rows) x 16 tokens per block, the contraction split over the waves.
__global__ __launch_bounds__(kThreads) void i8_up_kernel(FfnI8Args a) {
    __shared__ int s_red[2][kWaves][16][17];  // [gate / up][wave][token][feature]
    Tile t;
    if (!find_tile<true, 16>(a, blockIdx.x, t)) return;
    const int tid = threadIdx.x, lane = tid & 63, m = lane & 15, quad = lane >> 4, w = tid >> 6;
    const int nf = t.shared ? a.Is : a.I, d = a.d;
    auto token = [&](int p) -> int {  // the token of the tile's p-th column, or -1
        if (t.tok0 + p >= t.ntok) return -1;
        if (t.shared) return t.tok0 + p;
        const int s = a.perm[t.start + t.tok0 + p];
        if (s >= 0 && s < a.T * a.K) return s / a.K;
        atomicOr(&a.ctrl[kWordFlags], (uint32_t)SPICE_FLAG_BAD_INDEX);
        return 0;
    };
    const int tok = token(m);
    const char* rows[2] = {t.w + (size_t)(t.row0 + m) * d, t.w + (size_t)(nf + t.row0 + m) * d};
    i32x4_t acc[2] = {};
    wave_sums<2>(rows, reinterpret_cast<const char*>(a.xq) + (size_t)(tok < 0 ? 0 : tok) * d, tok >= 0, d, acc);
#pragma unroll
    for (int r = 0; r < 2; ++r)
#pragma unroll
        for (int i = 0; i < 4; ++i) s_red[r][w][m][quad * 4 + i] = acc[r][i];
    __syncthreads();
    const int p = tid >> 4, f = tid & 15;
    const int tp = token(p);
    if (tp < 0) return;
    int g = 0, u = 0;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) {
        g += s_red[0][i][p][f];
        u += s_red[1][i][p][f];
    }
    const float* scale = reinterpret_cast<const float*>(t.w + (size_t)2 * nf * d);
    const float sx = a.xs[tp];
    const float gv = (float)g * (sx * scale[t.row0 + f]), uv = (float)u * (sx * scale[nf + t.row0 + f]);
    float* h = t.shared ? a.hs : a.h;
    h[(size_t)(t.start + t.tok0 + p) * nf + t.row0 + f] = silu(gv) * uv;
}

// Rows of H to 8 bits: a block per row; the T shared rows first, then the HIT slots' positions.
__global__ __launch_bounds__(kThreads) void i8_quant_kernel(FfnI8Args a) {
    __shared__ float s_top[kWaves];
    const int nsh = a.Is > 0 ? a.T : 0;
    const bool shared = (int)blockIdx.x < nsh;
    const int row = shared ? blockIdx.x : blockIdx.x - nsh;
    if (!shared && row >= a.offsets[a.N]) return;  // the HIT buckets' end
    const int tid = threadIdx.x, n = shared ? a.Is : a.I;
    const float* h = (shared ? a.hs : a.h) + (size_t)row * n;
    int8_t* q = (shared ? a.hqs : a.hq) + (size_t)row * i8_row(n);
    float top = 0.f, bad = 0.f;
    for (int i = tid * 4; i < n; i += kThreads * 4) {
        const f32x4_t v = *reinterpret_cast<const f32x4_t*>(h + i);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            top = fmaxf(top, fabsf(v[k]));
            bad = fmaf(v[k], 0.f, bad);
        }
    }
    top += bad;  // NaN for a row that is not finite
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        const float other = __shfl_xor(top, o);
        top = other != other || top != top ? __builtin_nanf("") : fmaxf(top, other);
    }
    if ((tid & 63) == 0) s_top[tid >> 6] = top;
    __syncthreads();
    top = 0.f;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) top = s_top[i] != s_top[i] || top != top ? __builtin_nanf("") : fmaxf(top, s_top[i]);
    const bool nan = top != top;
    const float inv = nan || top == 0.f ? 0.f : 127.f / top;
    if (tid == 0) (shared ? a.hscale_s : a.hscale)[row] = top / 127.f;
    for (int i = tid * 4; i < n; i += kThreads * 4) {
        const f32x4_t v = *reinterpret_cast<const f32x4_t*>(h + i);
        uint32_t b = 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) b |= (uint32_t)((int)(nan ? 0.f : rintf(v[k] * inv)) & 255) << (8 * k);
        *reinterpret_cast<uint32_t*>(q + i) = b;
    }
}

// Down: 32 output features x 16 tokens per block, the contraction split over the waves.
constexpr int kDownR = 2;
__global__ __launch_bounds__(kThreads) void i8_down_kernel(FfnI8Args a) {
    __shared__ int s_red[kDownR][kWaves][16][17];
    Tile t;
    if (!find_tile<false, 16 * kDownR>(a, blockIdx.x, t)) return;
    const int tid = threadIdx.x, lane = tid & 63, m = lane & 15, quad = lane >> 4, w = tid >> 6;
    const int K = t.shared ? a.Is : a.I, d = a.d;
    const char* rows[kDownR];
#pragma unroll
    for (int r = 0; r < kDownR; ++r) rows[r] = t.w + (size_t)min(t.row0 + 16 * r + m, d - 1) * K;
    const bool live = t.tok0 + m < t.ntok;
    const char* x = reinterpret_cast<const char*>(t.shared ? a.hqs : a.hq) +
                    (size_t)(live ? t.start + t.tok0 + m : 0) * i8_row(K);
    i32x4_t acc[kDownR] = {};
    wave_sums<kDownR>(rows, x, live, K, acc);
#pragma unroll
    for (int r = 0; r < kDownR; ++r)
#pragma unroll
        for (int i = 0; i < 4; ++i) s_red[r][w][m][quad * 4 + i] = acc[r][i];
    __syncthreads();
    const int p = tid >> 4, f = tid & 15;
    if (t.tok0 + p >= t.ntok) return;
    const int pos = t.start + t.tok0 + p;
    const float* scale = reinterpret_cast<const float*>(t.w + (size_t)d * K);
    float sh = (t.shared ? a.hscale_s : a.hscale)[pos];
    if (t.shared && a.sgate) sh *= a.sgate[pos];
    float* y = (t.shared ? a.y_shared : a.y_slots) + (size_t)pos * d;
#pragma unroll
    for (int r = 0; r < kDownR; ++r) {
        const int j = t.row0 + 16 * r + f;
        if (j >= d) continue;
        int sum = 0;
#pragma unroll
        for (int i = 0; i < kWaves; ++i) sum += s_red[r][i][p][f];
        y[j] = (float)sum * (sh * scale[j]);
    }
}

// Upper bound of a launch's tiles: sum_e ceil(n_e / 16) <= slots / 16 + buckets.
long long tile_bound(const FfnI8Args& a, int nf_sh, int nf_e, int feat) {
    const long long slots = (long long)a.T * a.K, buckets = std::min<long long>(std::min(a.N, a.C), slots);
    const long long nt_sh = (nf_sh + feat - 1) / feat, nt_e = (nf_e + feat - 1) / feat;
    return (a.Is > 0 ? (a.T + kTok - 1) / kTok * nt_sh : 0) + (slots / kTok + buckets) * (buckets > 0 ? nt_e : 0);
}

}  // namespace

hipError_t launch_expert_ffn_i8(const FfnI8Args& a, hipStream_t s) {
    const long long up = tile_bound(a, a.Is, a.I, 16), down = tile_bound(a, a.d, a.d, 16 * kDownR);
    const long long rows = (a.Is > 0 ? a.T : 0) + (a.C > 0 ? (long long)a.T * a.K : 0);
    if (rows == 0) return hipSuccess;
    if (std::max({up, down, rows}) > 0x7FFFFFFFll) return hipErrorInvalidValue;
    const bool gemm = expert_gemm_i8_applies(a);
    hipError_t e = hipSuccess;
    if (gemm) e = launch_expert_gemm_i8(a, true, s);
    else hipLaunchKernelGGL(i8_up_kernel, dim3((unsigned)up), dim3(kThreads), 0, s, a);
    hipLaunchKernelGGL(i8_quant_kernel, dim3((unsigned)rows), dim3(kThreads), 0, s, a);
    if (e == hipSuccess && gemm) e = launch_expert_gemm_i8(a, false, s);
    else if (!gemm) hipLaunchKernelGGL(i8_down_kernel, dim3((unsigned)down), dim3(kThreads), 0, s, a);
    return e == hipSuccess ? hipGetLastError() : e;
}

}  // namespace spice
