// RMS norm with the residual's addition and an 8-bit output with a scale per token
// (moe_rmsnorm_quant): the input of a layer's routing and 8-bit experts.
//
//   s = x + resid;  h = s;  y = s w / sqrt(mean(s^2) + eps);  q = round(127 a / max |a|), a = s w
//
// The row's factor 1 / sqrt(..) cancels in q, so one pass over the row in registers finds both the
// sum of squares and max |a|, and a second one, over the same registers, writes every output.
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
    __device__ static void widen(const uint4& q, double (&v)[8]) {
        const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = (double)__uint_as_float(w[i] << 16);
            v[2 * i + 1] = (double)__uint_as_float(w[i] & 0xFFFF0000u);
        }
    }
    __device__ static uint32_t rne(double x) {
        const uint32_t u = __float_as_uint((float)x);
        if ((u & 0x7FFFFFFFu) > 0x7F800000u) return 0x7FC0u;
        return (u + 0x7FFFu + ((u >> 16) & 1u)) >> 16;
    }
    __device__ static uint4 pack(const double (&v)[8]) {
        uint4 q;
        q.x = rne(v[0]) | (rne(v[1]) << 16);
        q.y = rne(v[2]) | (rne(v[3]) << 16);
        q.z = rne(v[4]) | (rne(v[5]) << 16);
        q.w = rne(v[6]) | (rne(v[7]) << 16);
        return q;
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

constexpr int kNormThreads = 256;
constexpr int kNormChunks = 4;  // 16-byte chunks of a row per thread: rows of at most 16 KiB

// One block per row.
template <int DT>
__global__ __launch_bounds__(kNormThreads) void rmsnorm_quant_kernel(NormArgs a) {
    using R = Row<DT>;
    constexpr int V = R::V, NW = kNormThreads / 64;
    __shared__ double s_part[NW][3];
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const size_t row = blockIdx.x;
    const int nc = a.d / V;
    const uint4* x = static_cast<const uint4*>(a.x) + row * nc;
    const uint4* r = a.resid ? static_cast<const uint4*>(a.resid) + row * nc : nullptr;
    const uint4* wt = static_cast<const uint4*>(a.weight);
    uint4 xv[kNormChunks], rv[kNormChunks], wv[kNormChunks];
#pragma unroll
    for (int c = 0; c < kNormChunks; ++c) {
        const int i = c * kNormThreads + tid;
        const uint4 zero = {0u, 0u, 0u, 0u};
        xv[c] = rv[c] = wv[c] = zero;
        if (i < nc) {
            xv[c] = x[i];
            if (r) rv[c] = r[i];
            if (wt) wv[c] = wt[i];
        }
    }
    auto load = [&](int c, double (&s)[V], double (&p)[V]) {  // s and s * w
        double rr[V], ww[V];
        R::widen(xv[c], s);
        R::widen(rv[c], rr);
        R::widen(wv[c], ww);
#pragma unroll
        for (int k = 0; k < V; ++k) {
            if (r) s[k] += rr[k];
            p[k] = wt ? s[k] * ww[k] : s[k];
        }
    };
    double ss = 0.0, top = 0.0, bad = 0.0;  // bad: NaN once a product is not finite
#pragma unroll
    for (int c = 0; c < kNormChunks; ++c) {
        if (c * kNormThreads >= nc) break;  // uniform
        double s[V], p[V];
        load(c, s, p);
#pragma unroll
        for (int k = 0; k < V; ++k) {
            ss = fma(s[k], s[k], ss);
            top = fmax(top, fabs(p[k]));
            bad = fma(p[k], 0.0, bad);
        }
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        ss += __shfl_xor(ss, o);
        top = fmax(top, __shfl_xor(top, o));
        bad += __shfl_xor(bad, o);
    }
    if (lane == 0) {
        s_part[w][0] = ss;
        s_part[w][1] = top;
        s_part[w][2] = bad;
    }
    __syncthreads();
    ss = s_part[0][0];
    top = s_part[0][1];
    bad = s_part[0][2];
#pragma unroll
    for (int i = 1; i < NW; ++i) {
        ss += s_part[i][0];
        top = fmax(top, s_part[i][1]);
        bad += s_part[i][2];
    }
    const double rstd = ss == 0.0 ? 0.0 : 1.0 / sqrt(ss / a.d + a.eps);
    const bool nan = bad != bad;
    const double inv = nan || top == 0.0 ? 0.0 : 127.0 / top;
    if (a.q && tid == 0) a.q_scale[row] = nan ? __builtin_nanf("") : (float)(top * rstd / 127.0);
#pragma unroll
    for (int c = 0; c < kNormChunks; ++c) {
        const int i = c * kNormThreads + tid;
        if (i >= nc) break;
        double s[V], p[V], y[V];
        load(c, s, p);
        if (a.h) static_cast<uint4*>(a.h)[row * nc + i] = R::pack(s);
#pragma unroll
        for (int k = 0; k < V; ++k) y[k] = p[k] * rstd;
        if (a.y) static_cast<uint4*>(a.y)[row * nc + i] = R::pack(y);
        if (a.q) {
            // p * (127 / max) is off by a few units in the last place: where that can decide between two
            // codes (bf16 rows hold exact halves), the one rounding of 127 p / max does
            int q[V];
            bool near = false;
#pragma unroll
            for (int k = 0; k < V; ++k) {
                const double v = nan ? 0.0 : p[k] * inv, n = rint(v);
                near |= fabs(fabs(v - n) - 0.5) < 1e-9;
                q[k] = (int)n;
            }
            if (near) {
#pragma unroll
                for (int k = 0; k < V; ++k) q[k] = (int)rint(127.0 * p[k] / top);
            }
            uint32_t b[V / 4];
#pragma unroll
            for (int k = 0; k < V / 4; ++k)
                b[k] = (uint32_t)(q[4 * k] & 255) | (uint32_t)(q[4 * k + 1] & 255) << 8 |
                       (uint32_t)(q[4 * k + 2] & 255) << 16 | (uint32_t)(q[4 * k + 3] & 255) << 24;
            uint32_t* out = reinterpret_cast<uint32_t*>(a.q + row * a.d) + (size_t)i * (V / 4);
            if constexpr (V == 8) *reinterpret_cast<uint2*>(out) = make_uint2(b[0], b[1]);
            else *out = b[0];
        }
    }
}

}  // namespace

hipError_t launch_rmsnorm_quant(const NormArgs& a, hipStream_t s) {
    if (a.dtype == SPICE_BF16)
        hipLaunchKernelGGL(rmsnorm_quant_kernel<SPICE_BF16>, dim3((unsigned)a.T), dim3(kNormThreads), 0, s, a);
    else
        hipLaunchKernelGGL(rmsnorm_quant_kernel<SPICE_F32>, dim3((unsigned)a.T), dim3(kNormThreads), 0, s, a);
    return hipGetLastError();
}

}  // namespace spice
