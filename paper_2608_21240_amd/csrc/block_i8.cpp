// C-ABI entry points of the 8-bit block: the norm in front of it and its grouped expert FFN
// (argument checks and launches; no exception leaves them).
#include <cmath>
#include <cstdint>
#include <exception>
#include <string>

#include "spice_internal.h"

namespace spice {
spice_status_t set_error(spice_status_t st, const char* msg);
spice_status_t validate(const spice_moe_cfg_t* cfg, int32_t T);
}  // namespace spice

namespace {

spice_status_t fail(spice_status_t st, const char* fn, const std::string& msg) {
    return spice::set_error(st, (std::string(fn) + ": " + msg).c_str());
}

spice_status_t hip_result(hipError_t e, const char* fn) {
    return e == hipSuccess ? SPICE_OK : fail(SPICE_ERR_HIP, fn, hipGetErrorString(e));
}

bool overlaps(const void* a, size_t an, const void* b, size_t bn) {
    if (!a || !b || an == 0 || bn == 0) return false;
    const uintptr_t a0 = (uintptr_t)a, b0 = (uintptr_t)b;
    return a0 < b0 + bn && b0 < a0 + an;
}

bool aligned16(const void* p) { return (uintptr_t)p % 16 == 0; }

}  // namespace

extern "C" spice_status_t moe_rmsnorm_quant(const spice_moe_cfg_t* cfg, int32_t T, const void* x, const void* resid,
                                            const void* weight, float eps, void* h_out, void* y_out, int8_t* q_out,
                                            float* q_scale, spice_stream_t stream) {
    const char* fn = "moe_rmsnorm_quant";
    try {
        const spice_status_t st = spice::validate(cfg, T);
        if (st != SPICE_OK) return st;
        if (!(eps >= 0.f) || std::isinf(eps)) return fail(SPICE_ERR_INVALID, fn, "eps must be finite and >= 0");
        if (T == 0) return SPICE_OK;
        if (!x) return fail(SPICE_ERR_INVALID, fn, "x is NULL");
        if (!h_out && !y_out && !q_out) return fail(SPICE_ERR_INVALID, fn, "no output");
        if (!q_out != !q_scale) return fail(SPICE_ERR_INVALID, fn, "q_out and q_scale go together");
        if (!aligned16(x) || !aligned16(resid) || !aligned16(weight) || !aligned16(h_out) || !aligned16(y_out) ||
            !aligned16(q_out) || (uintptr_t)q_scale % 4)
            return fail(SPICE_ERR_UNSUPPORTED, fn, "buffers must be 16-byte aligned");
        const size_t es = cfg->dtype == SPICE_BF16 ? 2 : 4, n = (size_t)T * cfg->d, sb = (size_t)T * sizeof(float);
        struct Buf {
            const void* p;
            size_t bytes;
            bool rows;  // [T][d] in the dtype: h_out and y_out may be such an input itself
        };
        const Buf in[3] = {{x, n * es, true}, {resid, n * es, true}, {weight, (size_t)cfg->d * es, false}};
        const Buf out[4] = {{h_out, n * es, true}, {y_out, n * es, true}, {q_out, n, false}, {q_scale, sb, false}};
        for (int i = 0; i < 4; ++i) {
            for (const Buf& b : in)
                if (overlaps(out[i].p, out[i].bytes, b.p, b.bytes) && !(out[i].rows && b.rows && out[i].p == b.p))
                    return fail(SPICE_ERR_INVALID, fn, "an output overlaps an input without being it");
            for (int j = 0; j < i; ++j)
                if (overlaps(out[i].p, out[i].bytes, out[j].p, out[j].bytes))
                    return fail(SPICE_ERR_INVALID, fn, "outputs overlap");
        }
        spice::NormArgs a{};
        a.T = T; a.d = cfg->d; a.dtype = cfg->dtype; a.eps = eps; a.inv_d = 1.0 / cfg->d;
        a.x = x; a.resid = resid; a.weight = weight; a.h = h_out; a.y = y_out; a.q = q_out; a.q_scale = q_scale;
        return hip_result(spice::launch_rmsnorm_quant(a, stream), fn);
    } catch (const std::exception& ex) {
        return spice::set_error(SPICE_ERR_INTERNAL, ex.what());
    } catch (...) {
        return spice::set_error(SPICE_ERR_INTERNAL, "unknown exception");
    }
}

extern "C" spice_status_t moe_expert_ffn_grouped_i8(const spice_moe_cfg_t* cfg, int32_t T, const int8_t* x_q,
                                                    const float* x_scale, const void* x, const int32_t* perm,
                                                    const int32_t* offsets, const int32_t* resident_slot,
                                                    const void* w13_pool, const void* w2_pool, const void* w13_shared,
                                                    const void* w2_shared, const void* w_shared_gate,
                                                    const void* lore_A, const void* lore_B, float* y_slots,
                                                    float* y_shared, void* ws, size_t ws_bytes, spice_stream_t stream) {
    const char* fn = "moe_expert_ffn_grouped_i8";
    try {
        const spice_status_t st = spice::validate(cfg, T);
        if (st != SPICE_OK) return st;
        const spice_moe_cfg_t& c = *cfg;
        if (c.wfmt != SPICE_WFMT_INT8) return fail(SPICE_ERR_UNSUPPORTED, fn, "needs SPICE_WFMT_INT8 expert weights");
        if (T == 0) return SPICE_OK;
        const bool shared = c.shared_inter > 0, gated = shared && w_shared_gate, lore = lore_A && lore_B;
        const struct {
            const void* p;
            const char* name;
            bool needed;
        } need[] = {{x_q, "x_q", true}, {x_scale, "x_scale", true}, {perm, "perm", true}, {offsets, "offsets", true},
                    {resident_slot, "resident_slot", true}, {w13_pool, "w13_pool", c.n_slots > 0},
                    {w2_pool, "w2_pool", c.n_slots > 0}, {w13_shared, "w13_shared", shared},
                    {w2_shared, "w2_shared", shared}, {y_slots, "y_slots", true}, {y_shared, "y_shared", shared},
                    {x, "x", gated || (lore && c.lore_rank > 0)}, {ws, "workspace", true}};
        for (const auto& n : need)
            if (n.needed && !n.p) return fail(SPICE_ERR_INVALID, fn, std::string(n.name) + " is NULL");
        if (!aligned16(x_q) || !aligned16(w13_pool) || !aligned16(w2_pool) || !aligned16(y_slots) || !aligned16(y_shared) ||
            (shared && (!aligned16(w13_shared) || !aligned16(w2_shared))) ||
            (lore && (!aligned16(x) || !aligned16(lore_A) || !aligned16(lore_B))))
            return fail(SPICE_ERR_UNSUPPORTED, fn, "activations, weights and outputs must be 16-byte aligned");
        const spice::WsLayout L = spice::ws_layout(c, T);
        if (ws_bytes < L.base)
            return fail(SPICE_ERR_WORKSPACE, fn, "workspace has " + std::to_string(ws_bytes) + " bytes, needs " +
                                                     std::to_string(L.base));
        const size_t yb = (size_t)T * c.top_k * c.d * sizeof(float), sb = (size_t)T * c.d * sizeof(float);
        const struct {
            const void* p;
            size_t bytes;
        } in[] = {{x_q, (size_t)T * c.d}, {x_scale, (size_t)T * sizeof(float)}, {x, (size_t)T * c.d * 2}};
        bool alias = overlaps(y_slots, yb, y_shared, sb);
        for (const auto& b : in) alias |= overlaps(y_slots, yb, b.p, b.bytes) || overlaps(y_shared, sb, b.p, b.bytes);
        if (alias) return fail(SPICE_ERR_INVALID, fn, "outputs alias each other or the activations");
        char* wsb = static_cast<char*>(ws);
        spice::FfnI8Args a{};
        a.T = T; a.d = c.d; a.N = c.n_experts; a.K = c.top_k; a.C = c.n_slots; a.I = c.inter; a.Is = c.shared_inter;
        a.xq = x_q; a.xs = x_scale; a.perm = perm; a.offsets = offsets; a.resident_slot = resident_slot;
        a.w13_pool = static_cast<const char*>(w13_pool); a.w2_pool = static_cast<const char*>(w2_pool);
        a.w13s = static_cast<const char*>(w13_shared); a.w2s = static_cast<const char*>(w2_shared);
        a.y_slots = y_slots; a.y_shared = y_shared;
        a.h = reinterpret_cast<float*>(wsb + L.h); a.hs = reinterpret_cast<float*>(wsb + L.hs);
        a.hq = reinterpret_cast<int8_t*>(wsb + L.hq); a.hqs = reinterpret_cast<int8_t*>(wsb + L.hqs);
        a.hscale = reinterpret_cast<float*>(wsb + L.hscale); a.hscale_s = reinterpret_cast<float*>(wsb + L.hscale_s);
        a.top = reinterpret_cast<float*>(wsb + L.top); a.top_s = reinterpret_cast<float*>(wsb + L.top_s);
        a.part = L.total > L.part && ws_bytes >= L.total ? reinterpret_cast<int32_t*>(wsb + L.part) : nullptr;
        a.ctrl = static_cast<uint32_t*>(ws);
        if (gated) {
            float* sg = reinterpret_cast<float*>(wsb + L.sgate);
            const hipError_t e = spice::launch_shared_gate(x, w_shared_gate, T, c.d, c.dtype, sg, stream);
            if (e != hipSuccess) return hip_result(e, fn);
            a.sgate = sg;
        }
        if (lore && c.lore_rank > 0) {
            a.r = c.lore_rank;
            a.x = static_cast<const uint16_t*>(x);
            a.lore_A = static_cast<const uint16_t*>(lore_A); a.lore_B = static_cast<const uint16_t*>(lore_B);
            a.u = reinterpret_cast<float*>(wsb + L.u);
        }
        return hip_result(spice::launch_expert_ffn_i8(a, stream), fn);
    } catch (const std::exception& ex) {
        return spice::set_error(SPICE_ERR_INTERNAL, ex.what());
    } catch (...) {
        return spice::set_error(SPICE_ERR_INTERNAL, "unknown exception");
    }
}
