// RMS norm with the residual's addition and an 8-bit output with a scale per token
// (moe_rmsnorm_quant): the input of a layer's routing and 8-bit experts.
//
//   s = x + resid;  h = s;  y = s w / sqrt(mean(s^2) + eps);  q = round(127 a / max |a|), a = s w
//
// The row's factor 1 / sqrt(..) cancels in q, so one pass over the row in registers finds both the
// sum of squares and max |a|, and a second one, over the same registers, writes every output.
// Everything is fp64 until the one rounding of each output, so a code is the nearest integer of the exact
// quotient.  Each byte is read and written once: memory's rate is the bound of many rows (bf16, 8192 x 3584
// with a residual and all outputs, 264 MB: 54 us, 4.9 TB/s, a copy's rate on the same card; call after call in a
// graph 57 us, with the time between two launches), the launch and one trip to memory that of a few (1 x 2048:
// 2.6 us, in a graph 3.0).  A chunk per thread, so that none idles through a second round, and cheaper conversions
// took the first from 73 us in a graph.
#include <hip/hip_runtime.h>

#include <cmath>

#include "spice_internal.h"

namespace spice {
namespace {

template <int DT>
struct Row;

template <>
struct Row<SPICE_BF16> {
    static constexpr int V = 8;  // elements per 16 bytes
    typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
    typedef float f32x2_t __attribute__((ext_vector_type(2)));
    __device__ static void widen(const uint4& q, double (&v)[8]) {
        const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = (double)__uint_as_float(w[i] << 16);
            v[2 * i + 1] = (double)__uint_as_float(w[i] & 0xFFFF0000u);
        }
    }
    __device__ static uint4 pack(const double (&v)[8]) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {  // round to nearest even in one instruction
            const f32x2_t f = {(float)v[2 * i], (float)v[2 * i + 1]};
            w[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f, bf16x2_t));
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
};

template <>
struct Row<SPICE_F32> {
    static constexpr int V = 4;
    __device__ static void widen(const uint4& q, double (&v)[4]) {
        v[0] = (double)__uint_as_float(q.x);
        v[1] = (double)__uint_as_float(q.y);
        v[2] = (double)__uint_as_float(q.z);
        v[3] = (double)__uint_as_float(q.w);
    }
    __device__ static uint4 pack(const double (&v)[4]) {
        return make_uint4(__float_as_uint((float)v[0]), __float_as_uint((float)v[1]), __float_as_uint((float)v[2]),
                          __float_as_uint((float)v[3]));
    }
};

// One 16-byte chunk of a row per thread: rows of more than 64 chunks take a block each (kWaveRows false),
// shorter ones `lanes` lanes of a wave, a power of two.
template <int DT, bool kWaveRows>
__global__ __launch_bounds__(kWaveRows ? 256 : 1024) void rmsnorm_quant_kernel(NormArgs a, int lanes) {
    using R = Row<DT>;
    constexpr int V = R::V;
    const int nc = a.d / V, tid = threadIdx.x;
    const size_t row = kWaveRows ? (size_t)blockIdx.x * (256 / lanes) + tid / lanes : blockIdx.x;
    const int i = kWaveRows ? tid & (lanes - 1) : tid;
    if (kWaveRows && row >= (size_t)a.T) return;  // whole groups of lanes
    const bool in = i < nc;
    const size_t at = row * nc + (in ? i : 0);
    const uint4 zero = {0u, 0u, 0u, 0u};
    uint4 xv = static_cast<const uint4*>(a.x)[at], rv = zero, wv = zero;
    if (a.resid) rv = static_cast<const uint4*>(a.resid)[at];
    if (a.weight) wv = static_cast<const uint4*>(a.weight)[in ? i : 0];
    double s[V], p[V];  // s and s * w
    R::widen(in ? xv : zero, s);
    if (a.resid) {
        double r[V];
        R::widen(in ? rv : zero, r);
#pragma unroll
        for (int k = 0; k < V; ++k) s[k] += r[k];
    }
    if (a.weight) {
        double w[V];
        R::widen(wv, w);
#pragma unroll
        for (int k = 0; k < V; ++k) p[k] = s[k] * w[k];
    } else {
#pragma unroll
        for (int k = 0; k < V; ++k) p[k] = s[k];
    }
    double ss = 0.0, top = 0.0, bad = 0.0;  // bad: NaN once a product is not finite
#pragma unroll
    for (int k = 0; k < V; ++k) {
        ss = fma(s[k], s[k], ss);
        top = fmax(top, fabs(p[k]));
        bad = fma(p[k], 0.0, bad);
    }
    for (int o = (kWaveRows ? lanes : 64) / 2; o > 0; o >>= 1) {
        ss += __shfl_xor(ss, o);
        top = fmax(top, __shfl_xor(top, o));
    }
    bool nan = __ballot(bad != bad) != 0;
    if constexpr (kWaveRows) {
        const unsigned long long mine = lanes == 64 ? ~0ull : ((1ull << lanes) - 1) << ((tid & 63) & ~(lanes - 1));
        nan = (__ballot(bad != bad) & mine) != 0;
    } else {
        __shared__ double s_part[16][2];
        __shared__ int s_nan[16];
        const int nw = (int)(blockDim.x >> 6), w = tid >> 6;
        if ((tid & 63) == 0) {
            s_part[w][0] = ss;
            s_part[w][1] = top;
            s_nan[w] = nan;
        }
        __syncthreads();
        ss = top = 0.0;
        int any = 0;
        for (int k = 0; k < nw; ++k) {
            ss += s_part[k][0];
            top = fmax(top, s_part[k][1]);
            any |= s_nan[k];
        }
        nan = any != 0;
    }
    const double rstd = ss == 0.0 ? 0.0 : rsqrt(fma(ss, a.inv_d, a.eps));
    if (a.q && i == 0) a.q_scale[row] = nan ? __builtin_nanf("") : (float)(top * rstd / 127.0);
    if (!in) return;
    if (a.h) static_cast<uint4*>(a.h)[at] = R::pack(s);
    if (a.y) {
        double y[V];
#pragma unroll
        for (int k = 0; k < V; ++k) y[k] = p[k] * rstd;
        static_cast<uint4*>(a.y)[at] = R::pack(y);
    }
    if (!a.q) return;
    // p * (127 / max) is off by 2e-12 at most: where that can decide between two codes (bf16 rows hold exact
    // halves), the one rounding of 127 p / max does.  v_rcp_f64 is documented to 2^29 units in the last place,
    // 2^-23 relative; a step of Newton's squares that, 1.4e-14, on quotients of up to 127
    double inv = __builtin_amdgcn_rcp(top);
    inv = top > 0.0 ? 127.0 * fma(fma(-top, inv, 1.0), inv, inv) : 0.0;
    int q[V];
    bool near = false;
#pragma unroll
    for (int k = 0; k < V; ++k) {
        const double v = p[k] * inv, n = rint(v);
        near |= fabs(v - n) > 0.5 - 1e-9;
        q[k] = (int)n;
    }
    if (near) {
#pragma unroll
        for (int k = 0; k < V; ++k) q[k] = (int)rint(127.0 * p[k] / top);
    }
    uint32_t b[V / 4];
#pragma unroll
    for (int k = 0; k < V / 4; ++k)
        b[k] = nan ? 0u
                   : (uint32_t)(q[4 * k] & 255) | (uint32_t)(q[4 * k + 1] & 255) << 8 | (uint32_t)(q[4 * k + 2] & 255) << 16 |
                         (uint32_t)q[4 * k + 3] << 24;
    uint32_t* out = reinterpret_cast<uint32_t*>(a.q + row * a.d) + (size_t)i * (V / 4);
    if constexpr (V == 8) *reinterpret_cast<uint2*>(out) = make_uint2(b[0], b[1]);
    else *out = b[0];
}

template <int DT>
hipError_t launch_norm(const NormArgs& a, hipStream_t s) {
    const int nc = a.d / Row<DT>::V;
    if (nc > 64) {
        hipLaunchKernelGGL((rmsnorm_quant_kernel<DT, false>), dim3((unsigned)a.T), dim3((nc + 63) / 64 * 64), 0, s, a, 64);
    } else {
        int lanes = 1;
        while (lanes < nc) lanes *= 2;
        const int rows = 256 / lanes;
        hipLaunchKernelGGL((rmsnorm_quant_kernel<DT, true>), dim3((unsigned)((a.T + rows - 1) / rows)), dim3(256), 0, s, a,
                           lanes);
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_rmsnorm_quant(const NormArgs& a, hipStream_t s) {
    return a.dtype == SPICE_BF16 ? launch_norm<SPICE_BF16>(a, s) : launch_norm<SPICE_F32>(a, s);
}

}  // namespace spice
