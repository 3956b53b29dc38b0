"""The 8-bit MoE block on the GPU against plain 64-bit forms: the norm with its 8-bit output, the scored
routing, the 8-bit expert FFN, and a layer that runs them one after the other."""
import numpy as np
import pytest
import torch

import block_i8 as R
from block_i8 import EXACT, HIT, LORE, U
from paper_2608_21240_amd import layer as LY, spice, synth, workloads as W

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    spice.lib()
    yield
    torch.cuda.synchronize()


def say(*a):
    print("[block]", *a, flush=True)


def make_cfg(d, N=1, K=1, I=16, Is=0, r=0, C=0, dt=BF, i8=False, **kw):
    s = W.MoEShape(d, N, K, I, Is, r, W.DTYPE_F32 if dt == F32 else W.DTYPE_BF16)
    return spice.make_cfg(s, C, wfmt=spice.SPICE_WFMT_INT8 if i8 else 0, **kw)


def workspace(c, T):
    n = spice.spice_workspace_bytes(c, T)
    assert n, spice.last_error()
    return torch.zeros(n, dtype=torch.uint8, device="cuda"), n


# ---- norm ------------------------------------------------------------------------------------


def norm_inputs(T, d, dt, seed=0, resid=True, weight=True):
    g = R.gen(seed)
    x, r, w = (torch.randn(T, d, generator=g) * 3).to(dt), torch.randn(T, d, generator=g).to(dt), (
        1 + 0.2 * torch.randn(d, generator=g)).to(dt)
    return x.cuda(), r.cuda() if resid else None, w.cuda() if weight else None


def check_norm(x, r, w, eps, h, y, q, qs):
    s, yr, qr, sr = (v.cpu() for v in R.norm_ref(x, r, w, eps))
    half = torch.finfo(x.dtype).eps / 2
    # through fp32 to the dtype: half a step, and fp32's own half step
    for got, ref in ((h, s), (y, yr)):
        if got is not None:
            got = got.double().cpu()
            fine = torch.isfinite(ref)
            assert torch.equal(torch.isnan(ref), torch.isnan(got))
            assert ((got - ref).abs()[fine] <= (ref.abs() * (half + 1.01 * U) + 1e-45)[fine]).all()
    if q is not None:
        assert torch.equal(q.double().cpu(), qr)
        assert torch.equal(torch.isnan(qs.cpu()), torch.isnan(sr))
        fine = ~torch.isnan(sr)
        assert ((qs.double().cpu() - sr).abs()[fine] <= (sr * 1.01 * U + 1e-45)[fine]).all()


@pytest.mark.parametrize("T,d,dt,resid,weight", [
    (1, 2048, BF, True, True), (1, 8, BF, True, True), (3, 8192, BF, True, True), (77, 1504, BF, False, True),
    (5, 4, F32, True, True), (9, 4096, F32, True, False), (130, 1500, F32, True, True), (1031, 104, BF, True, False),
    (2050, 3584, BF, True, True), (600, 520, F32, False, False)])
def test_norm(T, d, dt, resid, weight):
    say("norm", T, d, dt, resid, weight)
    x, r, w = norm_inputs(T, d, dt, T + d, resid, weight)
    h, y = torch.empty_like(x), torch.empty_like(x)
    q, qs = torch.empty(T, d, dtype=torch.int8, device="cuda"), torch.empty(T, device="cuda")
    spice.moe_rmsnorm_quant(make_cfg(d, dt=dt), T, x, r, w, 1e-5, h, y, q, qs)
    check_norm(x, r, w, float(np.float32(1e-5)), h, y, q, qs)


@pytest.mark.parametrize("which", ["h", "y", "q", "hy", "hq", "yq"])
def test_norm_writes_only_what_is_asked_and_may_write_in_place(which):
    T, d = 6, 264
    x, r, w = norm_inputs(T, d, BF, 3)
    x0, r0 = x.clone(), r.clone()
    q, qs = torch.empty(T, d, dtype=torch.int8, device="cuda"), torch.empty(T, device="cuda")
    h, y = (r if "h" in which else None), (x if "y" in which else None)  # the residual stream and the rows in place
    has_q = "q" in which
    spice.moe_rmsnorm_quant(make_cfg(d), T, x, r, w, 1e-6, h, y, q if has_q else None, qs if has_q else None)
    check_norm(x0, r0, w, float(np.float32(1e-6)), h, y, q if has_q else None, qs if has_q else None)
    assert "h" in which or torch.equal(r, r0)
    assert "y" in which or torch.equal(x, x0)


@pytest.mark.parametrize("dt,d", [(BF, 256), (F32, 1028)])
def test_norm_edge_rows(dt, d):
    """Zeros with eps 0, one large value, halves between two codes, NaN, infinities, tiny and huge values."""
    x, _, _ = norm_inputs(9, d, dt, 8)
    x[0] = 0
    x[1] = 0
    x[1, 5] = 1000
    x[2] = torch.arange(d, device="cuda").remainder(255).sub(127).to(dt) * 0.5  # max 63.5: quotients at halves
    x[2, 0] = -127
    x[3, 7] = float("nan")
    x[4, 9] = float("inf")
    x[5, 1] = -float("inf")
    x[6] *= 1e-30
    x[7] *= 1e18
    x[8] = -0.0
    h, y = torch.empty_like(x), torch.empty_like(x)
    q, qs = torch.empty(9, d, dtype=torch.int8, device="cuda"), torch.empty(9, device="cuda")
    spice.moe_rmsnorm_quant(make_cfg(d, dt=dt), 9, x, None, None, 0.0, h, y, q, qs)
    fine = [0, 1, 2, 3, 6, 7, 8]
    check_norm(x[fine], None, None, 0.0, h[fine], y[fine], q[fine], qs[fine])
    assert torch.isnan(qs[4:6]).all() and (q[4:6] == 0).all() and torch.isnan(y[4, 9]) and torch.isnan(y[5, 1])
    assert (y[0] == 0).all() and qs[0] == 0


# ---- scored routing -----------------------------------------------------------------------------


class Routing:
    def __init__(self, T, d, N, K, dt=BF, C=0, seed=0, **cfg):
        g = R.gen(seed)
        self.T, self.N, self.K = T, N, K
        self.x, self.wg = torch.randn(T, d, generator=g).to(dt).cuda(), (0.05 * torch.randn(N, d, generator=g)).to(dt).cuda()
        self.conf = torch.rand(T, K, generator=g).cuda()
        self.balance = (0.05 * torch.randn(N, generator=g)).cuda()
        self.slot = torch.full((N,), -1, dtype=torch.int32)
        self.slot[torch.randperm(N, generator=g)[:C]] = torch.arange(C, dtype=torch.int32)
        self.slot = self.slot.cuda()
        self.bias = None
        self.cfg = make_cfg(d, N, K, C=C, dt=dt, **cfg)
        i32 = dict(dtype=torch.int32, device="cuda")
        self.logits = torch.empty(T, N, dtype=torch.float64, device="cuda")
        self.idx, self.w = torch.full((T, K), -9, **i32), torch.empty(T, K, device="cuda")
        self.cls = torch.empty(T, K, dtype=torch.uint8, device="cuda")
        self.offsets, self.perm, self.inv = torch.empty(3, N + 1, **i32), torch.empty(T * K, **i32), torch.empty(T * K, **i32)
        self.ws, self.wsn = workspace(self.cfg, T)

    def run(self, sigmoid=False, groups=1, keep=1, top=1, balance=False, scale=1.0, logits=True, stream=None, host_out=None):
        sc = spice.route_score(int(sigmoid), groups, keep, top, scale, self.balance if balance else None)
        spice.moe_route_bucket_scored(self.cfg, sc, self.T, self.x, self.wg, self.bias, self.slot, self.conf,
                                      self.logits if logits else None, self.idx, self.w, self.cls, self.offsets,
                                      self.perm, self.inv, host_out, self.ws, self.wsn, stream)

    def check(self, z, sigmoid=False, groups=1, keep=1, top=1, balance=False, scale=1.0):
        idx, w = R.route_ref(z, self.K, sigmoid, groups, keep, top, self.balance.cpu().numpy() if balance else None,
                             bool(self.cfg.norm_topk), scale)
        got = self.idx.cpu().numpy()
        assert np.array_equal(got, idx)
        # fp64 throughout, then one rounding to fp32
        assert np.allclose(self.w.double().cpu().numpy(), w, rtol=1.01 * U, atol=1e-45)
        slot, conf = self.slot.cpu().numpy(), self.conf.cpu().numpy()
        cls = np.where(slot[idx] >= 0, HIT, np.where(conf < self.cfg.tau, LORE, EXACT))
        assert np.array_equal(self.cls.cpu().numpy(), cls)
        self.check_buckets()

    def check_buckets(self):
        perm, inv, off = R.buckets_ref(self.idx.cpu().numpy(), self.cls.cpu().numpy(), self.N)
        assert np.array_equal(self.perm.cpu().numpy(), perm) and np.array_equal(self.inv.cpu().numpy(), inv)
        assert np.array_equal(self.offsets.cpu().numpy(), off)
        assert spice.spice_workspace_flags(self.ws, self.wsn) == 0


RULES = [dict(sigmoid=True), dict(groups=4, keep=2), dict(sigmoid=True, groups=4, keep=2, top=2, balance=True, scale=2.5),
         dict(balance=True, groups=2, keep=1, top=2, scale=16.0)]


@pytest.mark.parametrize("rule", range(len(RULES)))
@pytest.mark.parametrize("T,d,N,K,dt,norm", [
    (1, 64, 8, 2, BF, 0), (1, 2048, 64, 6, BF, 1), (33, 200, 256, 8, BF, 1), (7, 132, 12, 3, F32, 0),
    (230, 2048, 64, 6, BF, 1), (255, 96, 100, 5, F32, 1), (300, 256, 64, 8, BF, 0), (1000, 1440, 36, 4, BF, 1),
    (2000, 64, 252, 12, BF, 1)])
def test_scored_routing(T, d, N, K, dt, norm, rule):
    say("route", T, d, N, K, dt, norm, RULES[rule])
    r = Routing(T, d, N, K, dt, C=N // 3, seed=T + N, norm_topk=norm)
    r.run(**RULES[rule])
    z = r.x.double() @ r.wg.double().t()
    assert torch.allclose(r.logits, z, rtol=0, atol=float(2 * d * 2.0 ** -53 * (r.x.double().abs() @ r.wg.double().abs().t()).max()))
    r.check(r.logits.cpu().numpy(), **RULES[rule])


@pytest.mark.parametrize("T", [3, 240, 400])
@pytest.mark.parametrize("groups,keep,top", [(1, 1, 1), (32, 7, 2), (64, 64, 2), (16, 16, 1)])
def test_group_counts(T, groups, keep, top):
    rule = dict(sigmoid=True, groups=groups, keep=keep, top=top, balance=True)
    r = Routing(T, 256, 64, 6, C=10, seed=groups, norm_topk=1)
    r.run(**rule)
    r.check(r.logits.cpu().numpy(), **rule)


@pytest.mark.parametrize("T", [5, 220, 290])
def test_scored_routing_ties_go_to_the_lower_id(T):
    """Small whole numbers: logits, and with them scores and group values, are exact and often equal."""
    for rule in RULES:
        r = Routing(T, 64, 48, 5, seed=1)
        g = R.gen(2)
        r.x = torch.randint(-1, 2, (T, 64), generator=g).to(BF).cuda()
        r.wg = (torch.randint(-1, 2, (6, 64), generator=g).to(BF) / 8).cuda().repeat(8, 1)
        r.balance = torch.zeros_like(r.balance)
        r.run(**rule)
        r.check((r.x.double() @ r.wg.double().t()).cpu().numpy(), **rule)


@pytest.mark.parametrize("T", [4, 215, 300])
@pytest.mark.parametrize("rule", RULES)
def test_masked_experts(T, rule):
    """-inf logits: single experts, whole groups, all but fewer than K, all."""
    for masked in ([0, 5], list(range(0, 24)), list(range(1, 48)), list(range(46)), list(range(48))):
        r = Routing(T, 64, 48, 5, C=9, seed=4, norm_topk=1)
        r.bias = torch.zeros(48)
        r.bias[masked] = -float("inf")
        r.bias = r.bias.cuda()
        r.run(**rule)
        assert not torch.isnan(r.w).any()
        r.check(r.logits.cpu().numpy(), **rule)


@pytest.mark.parametrize("T", [4, 215, 300])
def test_bad_logits_still_give_valid_experts(T):
    for rule in RULES:
        r = Routing(T, 64, 48, 5, C=9, seed=4, norm_topk=1)
        r.x[1, 3], r.x[2, 5], r.x[3, 6] = float("nan"), float("inf"), -float("inf")
        r.run(**rule)
        idx = r.idx.cpu().numpy()
        assert ((idx >= 0) & (idx < 48)).all() and all(len(set(t)) == 5 for t in idx)
        r.check_buckets()


@pytest.mark.parametrize("T,N,K", [(13, 40, 5), (16, 40, 4), (64, 9, 1), (93, 256, 8), (94, 256, 8), (207, 256, 2),
                                   (187, 128, 2), (188, 128, 64), (300, 191, 3), (300, 130, 3), (256, 93, 3), (256, 94, 3), (257, 16, 2)])
def test_scored_routing_at_the_limits_of_its_variants(T, N, K):
    """64 and 65 slots, 1, 2 and 4 rows per wave, the last and the first calls of the row and tile forms, and of
    the form with separate bucketing."""
    for rule in RULES:
        r = Routing(T, 128, N, K, C=N // 2, seed=T)
        if N % rule.get("groups", 1) or K > rule.get("keep", 1) * (N // rule.get("groups", 1)):
            rule = dict(sigmoid=True)
        r.run(**rule)
        r.check(r.logits.cpu().numpy(), **rule)


def test_scored_routing_of_many_tokens():
    r = Routing(20000, 64, 16, 3, C=5, seed=3, norm_topk=1)
    rule = dict(sigmoid=True, groups=4, keep=2, top=2, balance=True, scale=2.5)
    r.run(**rule)
    r.check(r.logits.cpu().numpy(), **rule)


@pytest.mark.parametrize("T", [120, 300])
@pytest.mark.parametrize("N,K,groups,keep", [(65, 64, 13, 13), (250, 64, 50, 13), (256, 1, 2, 1), (192, 30, 1, 1)])
def test_scored_routing_ranks_of_more_experts_than_lanes(T, N, K, groups, keep):
    """Few distinct scores, masked experts, K up to 64 and groups that leave hardly more: many candidates and ties."""
    rule = dict(sigmoid=True, groups=groups, keep=keep, balance=True)
    r = Routing(T, 64, N, K, seed=N + K)
    g = R.gen(3)
    r.x = torch.randint(-1, 2, (T, 64), generator=g).to(BF).cuda()
    r.wg = (torch.randint(-1, 2, (N, 64), generator=g).to(BF) / 8).cuda()
    r.balance = torch.zeros_like(r.balance)
    r.bias = torch.where(torch.rand(N, generator=g) < 0.3, -float("inf"), 0.0).cuda()
    r.run(**rule)
    r.check(r.logits.cpu().numpy(), **rule)


@pytest.mark.parametrize("T", [5, 300])
def test_scored_routing_copies_to_the_host(T):
    r = Routing(T, 64, 48, 5, C=9, seed=2)
    pin = lambda t: torch.zeros(t.shape, dtype=t.dtype).pin_memory()  # noqa: E731
    x, idx, w, cls = (pin(t) for t in (r.x, r.idx, r.w, r.cls))
    counts, ready = (torch.zeros(n, dtype=torch.int32).pin_memory() for n in (4, 1))
    r.run(sigmoid=True, groups=4, keep=2, host_out=spice.host_out(x, idx, w, cls, counts, ready, 77))
    torch.cuda.synchronize()
    for a, b in ((x, r.x), (idx, r.idx), (w, r.w), (cls, r.cls)):
        assert torch.equal(a, b.cpu())
    assert counts[:3].tolist() == torch.bincount(r.cls.flatten().long(), minlength=3).tolist() and ready.item() == 77


@pytest.mark.parametrize("mode", [spice.SPICE_CONF_GATE, spice.SPICE_CONF_GATE_RENORM])
@pytest.mark.parametrize("T,norm", [(9, 0), (9, 1), (300, 0)])
def test_confidence_from_the_gates(mode, T, norm):
    r = Routing(T, 128, 32, 4, C=4, norm_topk=norm, conf_mode=mode, tau=0.25)
    r.run(sigmoid=True, scale=4.0)
    idx, w = R.route_ref(r.logits.cpu().numpy(), 4, True, renorm=bool(norm))
    conf = w if norm or mode == spice.SPICE_CONF_GATE else w / w.sum(1, keepdims=True)
    sure = np.abs(conf - 0.25) > 1e-6  # the confidence is rounded to fp32
    cls = np.where(r.slot.cpu().numpy()[idx] >= 0, HIT, np.where(conf < 0.25, LORE, EXACT))
    assert sure.mean() > 0.95 and np.array_equal(r.cls.cpu().numpy()[sure], cls[sure])


def test_scored_softmax_without_groups_is_the_plain_call():
    for T in (1, 40, 250, 500):
        r = Routing(T, 256, 64, 6, C=20, seed=T)
        r.run()
        want = [v.clone() for v in (r.idx, r.cls, r.offsets, r.perm, r.inv, r.w)]
        spice.moe_route_bucket(r.cfg, T, r.x, r.wg, None, r.slot, r.conf, None, r.idx, r.w, r.cls, r.offsets, r.perm,
                               r.inv, None, r.ws, r.wsn)
        for a, b in zip(want[:5], (r.idx, r.cls, r.offsets, r.perm, r.inv)):
            assert torch.equal(a, b)
        assert torch.allclose(want[5], r.w, rtol=2 * U, atol=0)


# ---- 8-bit experts -----------------------------------------------------------------------------


class Experts:
    """A layer's 8-bit experts with a routing drawn by the host."""

    def __init__(self, T, d, N, K, I, Is, C, r=0, seed=0, skew=False, lore=False):
        g = R.gen(seed)
        self.T, self.d, self.N, self.K, self.I, self.Is, self.C, self.r = T, d, N, K, I, Is, C, r
        self.cfg = make_cfg(d, N, K, I, Is, r, C, i8=True)
        self.x = torch.randn(T, d, generator=g).to(BF)
        self.xs = (self.x.float().abs().amax(1) / 127).cuda()
        self.x = self.x.cuda()
        self.xq = torch.round(self.x.float() / self.xs[:, None]).to(torch.int8)
        mk = lambda n, a, b: torch.stack([R.blob(0.05 * torch.randn(a, b, generator=g)) for _ in range(n)]).cuda()  # noqa: E731
        self.w13, self.w2 = (mk(C, 2 * I, d), mk(C, d, I)) if C else (None, None)
        self.w13s, self.w2s = (mk(1, 2 * Is, d)[0], mk(1, d, Is)[0]) if Is else (None, None)
        self.w_sg = None
        self.lore_A = (0.05 * torch.randn(N, max(r, 1), d, generator=g)).to(BF).cuda()
        self.lore_B = (0.05 * torch.randn(N, d, max(r, 1), generator=g)).to(BF).cuda()
        slot = torch.full((N,), -1, dtype=torch.int32)
        slot[torch.randperm(N, generator=g)[:C]] = torch.randperm(C, generator=g).to(torch.int32)
        z = torch.rand(T, N, generator=g) ** (1 if not skew else torch.linspace(0.05, 6, N))
        self.idx = torch.topk(z, K, dim=1).indices
        self.cls = torch.where(slot[self.idx] >= 0, HIT, LORE if lore else EXACT)
        perm, inv, off = R.buckets_ref(self.idx.numpy(), self.cls.numpy(), N)
        self.slot = slot.cuda()
        self.perm, self.offsets = torch.from_numpy(perm).int().cuda(), torch.from_numpy(off).int().cuda()
        self.pos = torch.from_numpy(inv).cuda()
        self.y_slots, self.y_shared = torch.full((T * K, d), 7.0, device="cuda"), torch.full((T, d), 7.0, device="cuda")
        self.ws, self.wsn = workspace(self.cfg, T)
        self.ws[spice.SPICE_WS_CONTROL_BYTES:] = 0xA5

    def run(self, lore=False, stream=None):
        la, lb = (self.lore_A, self.lore_B) if lore else (None, None)
        spice.moe_expert_ffn_grouped_i8(self.cfg, self.T, self.xq, self.xs, self.x, self.perm, self.offsets, self.slot,
                                        self.w13, self.w2, self.w13s, self.w2s, self.w_sg, la, lb, self.y_slots,
                                        self.y_shared, self.ws, self.wsn, stream)

    def check(self, lore=False):
        T, K, d, I = self.T, self.K, self.d, self.I
        if self.Is:
            y, tol = R.swiglu_i8_ref(self.xq, self.xs, self.w13s, self.w2s, d, self.Is)
            if self.w_sg is not None:
                gate = torch.sigmoid(self.x.double() @ self.w_sg.double())[:, None]
                y, tol = y * gate, tol * gate + 4 * U * (y * gate).abs()
            self.near(self.y_shared, y, tol)
        else:
            assert (self.y_shared == 7).all()
        idx, cls = self.idx.cuda().reshape(-1), self.cls.cuda().reshape(-1)
        got = self.y_slots[self.pos]  # by slot
        for e in range(self.N):
            s = ((idx == e) & (cls == HIT)).nonzero()[:, 0]
            if s.numel():
                c = int(self.slot[e])
                self.near(got[s], *R.swiglu_i8_ref(self.xq[s // K], self.xs[s // K], self.w13[c], self.w2[c], d, I))
            s = ((idx == e) & (cls == LORE)).nonzero()[:, 0]
            if s.numel() and lore:
                y = R.lore_ref(self.x[s // K], self.lore_A[e], self.lore_B[e])
                self.near(got[s], y, 1e-4 * y.abs().amax(1, keepdim=True))
        rest = (cls == EXACT) if lore else (cls != HIT)
        assert (got[rest] == 7).all()  # rows of other slots stay as they were
        assert spice.spice_workspace_flags(self.ws, self.wsn) == 0

    @staticmethod
    def near(got, ref, tol):
        off = (got.double() - ref).abs() - tol
        assert (off <= 1e-30).all(), float((off / ref.abs().amax()).max())


SIZES = [
    # T, d, N, K, I, Is, C
    (1, 16, 1, 1, 16, 16, 1), (1, 2048, 64, 6, 1408, 2816, 32), (2, 48, 5, 2, 32, 0, 3), (3, 80, 4, 3, 16, 48, 0),
    (17, 272, 7, 3, 112, 208, 7), (33, 1168, 20, 3, 720, 1040, 13), (16, 64, 3, 3, 528, 16, 3), (130, 192, 6, 2, 240, 144, 5),
    (300, 256, 4, 2, 256, 384, 4), (517, 400, 9, 4, 176, 496, 6), (1100, 144, 3, 1, 272, 80, 3)]


@pytest.mark.parametrize("size", SIZES)
@pytest.mark.parametrize("skew", [False, True])
def test_experts(size, skew):
    say("experts", size, skew)
    e = Experts(*size, seed=sum(size), skew=skew)
    e.run()
    e.check()


@pytest.mark.parametrize("size", [s for s, _ in R.SHAPE_CALLS])
def test_experts_in_each_tile_shape(size):
    say("experts", size)
    e = Experts(*size, seed=1, skew=size[0] > 2000)
    e.run()
    e.check()


@pytest.mark.parametrize("size,parts", R.SPLIT_CALLS)
def test_experts_with_a_split_shared_block(size, parts):
    """The split's sums are whole numbers: the same bits with the workspace's optional end and without it, and
    again on the same workspace (its counters are back at zero)."""
    say("experts", size)
    e = Experts(*size, seed=2)
    e.run()
    e.check()
    want = e.y_slots.clone(), e.y_shared.clone()
    for short in (0, 1, 0) if parts > 1 else (0,):
        e.wsn -= short
        e.run()
        e.wsn += short
        assert torch.equal(e.y_slots, want[0]) and torch.equal(e.y_shared, want[1])


def test_split_experts_in_a_graph_beside_an_eager_call():
    """Replays of a captured call, with calls of another workspace on another stream in between."""
    a, b = (Experts(3, 256, 8, 2, 48, 8192, 8, seed=s) for s in (1, 2))
    for e in (a, b):
        e.run()
    torch.cuda.synchronize()
    want = [(e.y_slots.clone(), e.y_shared.clone()) for e in (a, b)]
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph):
        a.run()
    for _ in range(4):
        for e in (a, b):
            e.y_slots.fill_(7), e.y_shared.fill_(7)
        side.wait_stream(torch.cuda.current_stream())
        graph.replay()
        b.run(stream=side)
        torch.cuda.synchronize()
        for e, w in zip((a, b), want):
            assert torch.equal(e.y_slots, w[0]) and torch.equal(e.y_shared, w[1])


@pytest.mark.parametrize("T,K,I,Is", [(1, 6, 256, 512), (2, 4, 1408, 2816), (3, 4, 1408, 2816), (16, 1, 272, 1040),
                                      (16, 2, 272, 0), (17, 2, 272, 16), (1, 8, 2576, 20480), (2, 1, 16, 10752),
                                      (2, 1, 16, 10880)])
@pytest.mark.parametrize("one", [False, True])
def test_experts_of_few_rows(T, K, I, Is, one):
    """Around the limits of down tiles that make H's codes for themselves; one: every slot takes the same expert,
    a bucket of more entries than tokens."""
    e = Experts(T, 64, 9, K, I, Is, 9, seed=T + K)
    if one:
        e.idx = torch.full((T, K), 3)
        perm, inv, off = R.buckets_ref(e.idx.numpy(), e.cls.numpy(), 9)
        e.perm, e.offsets, e.pos = torch.from_numpy(perm).int().cuda(), torch.from_numpy(off).int().cuda(), torch.from_numpy(inv).cuda()
    e.run()
    e.check()


@pytest.mark.parametrize("T", [1, 20, 150, 400])
def test_experts_with_gate_and_surrogates(T):
    e = Experts(T, 256, 8, 3, 96, 160, 4, r=16, seed=T, lore=True)
    e.w_sg = (0.05 * torch.randn(256, generator=R.gen(9))).to(BF).cuda()
    e.run(lore=True)
    e.check(lore=True)


@pytest.mark.parametrize("T", [5, 200])
def test_experts_edge_rows(T):
    """Rows of zeros, scales of zero, NaN scales, codes of -128, experts whose weights are zero."""
    e = Experts(T, 144, 4, 2, 64, 80, 3, seed=2)
    e.xq[0] = 0
    e.xs[1] = 0
    e.xq[2] = -128
    e.w13[0] = 0
    nan = 3
    e.xs[nan] = float("nan")
    e.run()
    idx = e.idx.cuda()
    got = e.y_slots[e.pos].view(T, 2, -1)
    assert torch.isnan(e.y_shared[nan]).all()
    for k in range(2):
        hit = int(e.cls[nan, k]) == HIT
        assert torch.isnan(got[nan, k]).all() == hit
    assert (e.y_shared[:2] == 0).all()
    e.xs[nan], e.xq[nan] = 0.0, 0  # what is left is checked as usual
    e.y_shared[nan] = 0
    for k in range(2):
        if int(e.cls[nan, k]) == HIT:
            e.y_slots[e.pos[2 * nan + k]] = 0
    e.check()
    assert idx.shape == (T, 2)


@pytest.mark.parametrize("T", [40, 300])
def test_experts_bad_indices_raise_a_flag(T):
    """Slots and pool slots out of range are skipped or read as token 0, never followed."""
    e = Experts(T, 64, 4, 2, 48, 32, 4, seed=3)
    e.perm[0], e.perm[1] = -5, T * 2
    e.run()
    assert spice.spice_workspace_flags(e.ws, e.wsn, clear=True) & spice.SPICE_FLAG_BAD_INDEX
    e = Experts(T, 64, 4, 2, 48, 32, 4, seed=3)
    e.slot[2] = 4
    e.run()
    assert spice.spice_workspace_flags(e.ws, e.wsn, clear=True) & spice.SPICE_FLAG_BAD_SLOT
    e = Experts(T, 64, 4, 2, 48, 32, 4, seed=3)
    e.offsets[0, 2:] += T * 2
    e.run()
    torch.cuda.synchronize()


@pytest.mark.parametrize("T", [1, 60])
def test_surrogates_of_every_rank_and_long_buckets(T):
    """All misses are surrogates of one expert or of a few; ranks of one chunk and of several stages."""
    for r, N in ((8, 2), (72, 3), (256, 5)):
        e = Experts(T, 192, N, 1, 32, 48, 1, r=r, seed=r, skew=True, lore=True)
        e.run(lore=True)
        e.check(lore=True)


def test_surrogates_with_bad_indices_raise_a_flag():
    e = Experts(40, 64, 4, 2, 48, 32, 0, r=8, seed=3, lore=True)
    e.perm[0], e.perm[1] = -5, 1000
    e.run(lore=True)
    assert spice.spice_workspace_flags(e.ws, e.wsn, clear=True) & spice.SPICE_FLAG_BAD_INDEX
    e = Experts(40, 64, 4, 2, 48, 32, 0, r=8, seed=3, lore=True)
    e.offsets[1, 2:] += 2 ** 30
    e.run(lore=True)
    torch.cuda.synchronize()


def test_surrogates_alone_after_the_experts():
    """The separate surrogate call takes the 8-bit layer's configuration: the corrections are the same."""
    e = Experts(90, 256, 8, 3, 96, 160, 4, r=16, seed=7, lore=True)
    e.run()
    spice.lore_surrogate_apply(e.cfg, 90, e.x, e.perm, e.offsets, e.lore_A, e.lore_B, e.y_slots, e.ws, e.wsn)
    e.check(lore=True)


def test_experts_give_the_same_bits_each_time():
    for T in (3, 90, 400):
        e = Experts(T, 272, 8, 3, 176, 208, 5, seed=T)
        e.run()
        want = e.y_slots.clone(), e.y_shared.clone()
        for _ in range(3):
            e.run()
            assert torch.equal(e.y_slots, want[0]) and torch.equal(e.y_shared, want[1])


# ---- together ----------------------------------------------------------------------------------


class Block:
    """norm -> scored routing -> 8-bit experts and surrogates -> combine, on one workspace."""

    def __init__(self, T, seed=0, **kw):
        self.e = Experts(T, 256, 16, 4, 96, 160, 9, r=8, seed=seed, lore=True)
        self.r = Routing(T, 256, 16, 4, C=0, seed=seed)
        self.r.slot, self.r.cfg = self.e.slot, self.e.cfg
        self.e.cfg.norm_topk, self.e.cfg.tau = 1, 2.0
        self.x, self.resid, self.w = norm_inputs(T, 256, BF, seed)
        self.out = torch.empty(T, 256, dtype=BF, device="cuda")
        self.h, self.y = torch.empty_like(self.out), torch.empty_like(self.out)
        self.T = T

    def run(self, stream=None):
        e, r = self.e, self.r
        spice.moe_rmsnorm_quant(e.cfg, self.T, self.x, self.resid, self.w, 1e-6, self.h, self.y, e.xq, e.xs, stream)
        sc = spice.route_score(1, 4, 2, 2, 2.5, r.balance)
        spice.moe_route_bucket_scored(e.cfg, sc, self.T, self.y, r.wg, None, e.slot, r.conf, None, r.idx, r.w, r.cls,
                                      r.offsets, r.perm, r.inv, None, e.ws, e.wsn, stream)
        spice.moe_expert_ffn_grouped_i8(e.cfg, self.T, e.xq, e.xs, self.y, r.perm, r.offsets, e.slot, e.w13, e.w2,
                                        e.w13s, e.w2s, None, e.lore_A, e.lore_B, e.y_slots, e.y_shared, e.ws, e.wsn,
                                        stream)
        spice.moe_combine(e.cfg, self.T, r.w, r.cls, r.inv, e.y_slots, e.y_shared, None, self.out, stream)


def block_ref(b):
    """The block's output in 64 bits and how far bf16 and fp32 may be from it."""
    e, r, T = b.e, b.r, b.T
    s, y, q, qs = R.norm_ref(b.x, b.resid, b.w, float(np.float32(1e-6)))
    y = y.float().to(BF)
    z = (y.double() @ r.wg.double().t()).cpu().numpy()
    idx, w = R.route_ref(z, 4, True, 4, 2, 2, r.balance.cpu().numpy(), True, 2.5)
    q, qs = q.to(torch.int8), qs.float()
    ys, tol = R.swiglu_i8_ref(q, qs, e.w13s, e.w2s, 256, 160)
    out, room = ys.clone(), tol.clone()
    for t in range(T):
        for k in range(4):
            ex, g = int(idx[t, k]), w[t, k]
            c = int(e.slot[ex])
            if c >= 0:
                v, tv = R.swiglu_i8_ref(q[t:t + 1], qs[t:t + 1], e.w13[c], e.w2[c], 256, 96)
                v, tv = v[0], tv[0]
            else:
                v = R.lore_ref(y[t:t + 1], e.lore_A[ex], e.lore_B[ex])[0]
                v, tv = v + ys[t], tol[t] + 1e-4 * v.abs().max()
            out[t] += g * v
            room[t] += g * (tv + 16 * U * v.abs())
    return idx, w, out, room + out.abs() * (2.0 ** -8 + 8 * U) + 16 * U * out.abs().amax(1, keepdim=True)


@pytest.mark.parametrize("T", [1, 7, 70, 280])
def test_block(T):
    b = Block(T, seed=T)
    b.run()
    idx, w, out, room = block_ref(b)
    assert np.array_equal(b.r.idx.cpu().numpy(), idx)
    assert np.allclose(b.r.w.double().cpu().numpy(), w, rtol=1.01 * U)
    assert ((b.out.double() - out).abs() <= room).all()


@pytest.mark.parametrize("T", [2, 100, 300])
def test_block_in_a_graph_and_on_another_stream(T):
    """Captured once, replayed on new inputs with eager work between: each replay against an eager run."""
    b, eager = Block(T, seed=1), Block(T, seed=1)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        b.run()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.run()
    for seed in (5, 6, 7):
        x, resid, w = norm_inputs(T, 256, BF, seed)
        for k in (b, eager):
            k.x.copy_(x); k.resid.copy_(resid); k.w.copy_(w)
        graph.replay()
        eager.run()
        torch.cuda.synchronize()
        for name in ("out", "h", "y"):
            assert torch.equal(getattr(b, name), getattr(eager, name)), name
        for name in ("idx", "w", "cls", "offsets", "perm", "inv"):
            assert torch.equal(getattr(b.r, name), getattr(eager.r, name)), name


def test_two_blocks_at_once():
    """Two workspaces, two streams, one GPU."""
    blocks = [Block(150, seed=s) for s in (1, 2)]
    for b in blocks:
        b.run()
    torch.cuda.synchronize()
    want = [b.out.clone() for b in blocks]
    streams = [torch.cuda.Stream() for _ in blocks]
    for _ in range(5):
        for b, s in zip(blocks, streams):
            b.out.zero_()
            s.wait_stream(torch.cuda.current_stream())
            b.run(s)
        torch.cuda.synchronize()
        for b, w in zip(blocks, want):
            assert torch.equal(b.out, w)


@pytest.mark.parametrize("T,gate", [(6, False), (90, True)])
def test_layer_driver(T, gate):
    """LayerRun with 8-bit experts and a scoring rule: norm, routing, GPU experts, the host's exact misses
    (fp32 activations), surrogates and the combine, and the cache that admits 8-bit blobs."""
    s = W.MoEShape(d=256, n_experts=16, top_k=4, inter=96, shared_inter=160, lore_rank=8, dtype=W.DTYPE_BF16)
    wl = W.Workload("i8", s, tokens=T, resident=6, skew=False, wfmt=W.WFMT_INT8, shared_gate=gate)
    host = LY.HostLayer(wl)
    dev = LY.DeviceLayer(host)
    balance = (0.05 * torch.randn(16, generator=R.gen(1))).cuda()
    run = LY.LayerRun(s, T, dev.C, tau=wl.tau, norm_topk=1, wfmt=W.WFMT_INT8,
                      score=spice.route_score(spice.SPICE_SCORE_SIGMOID, 4, 3, 2, 1.5, balance))
    x, resid, w = norm_inputs(T, 256, BF, 3)
    conf = torch.from_numpy(synth.gen_conf(wl)).cuda()
    out = run.forward(dev, x, conf, norm=(resid, w, 1e-6))
    torch.cuda.synchronize()
    check_norm(x, resid, w, float(np.float32(1e-6)), run.h, run.y, run.x_q, run.x_scale)
    z = (run.y.double() @ dev.wg.double().t()).cpu().numpy()
    idx, g = R.route_ref(z, 4, True, 4, 3, 2, balance.cpu().numpy(), True, 1.5)
    assert np.array_equal(run.topk_idx.cpu().numpy(), idx) and run.flags() == 0
    cls = run.slot_class.cpu().numpy()
    assert (np.bincount(cls.ravel(), minlength=3) > 0).all()
    gate_v = torch.sigmoid(run.y.double() @ dev.w_sg.double())[:, None] if gate else 1.0
    ys, tol = R.swiglu_i8_ref(run.x_q, run.x_scale, dev.w13s, dev.w2s, 256, 160)
    ys, tol = ys * gate_v, (tol + 4 * U * ys.abs()) * gate_v
    ref, room = ys.clone(), tol.clone()
    slot = dev.resident_slot.cpu().numpy()
    for t in range(T):
        for k in range(4):
            e = int(idx[t, k])
            if cls[t, k] == HIT:
                v, tv = R.swiglu_i8_ref(run.x_q[t:t + 1], run.x_scale[t:t + 1], dev.w13_pool[slot[e]], dev.w2_pool[slot[e]], 256, 96)
                v, tv = v[0], tv[0]
            elif cls[t, k] == LORE:
                v = R.lore_ref(run.y[t:t + 1], dev.lore_A[e], dev.lore_B[e])[0]
                v, tv = v + ys[t], tol[t] + 1e-4 * v.abs().max()
            else:
                a, sa = R.unblob(dev.host_w13[e].cuda(), 192, 256)
                b2, sb = R.unblob(dev.host_w2[e].cuda(), 256, 96)
                gu = (run.y[t].double() @ a.t()) * sa
                hv = gu[:96] / (1 + torch.exp(-gu[:96])) * gu[96:]
                v = (b2 @ hv) * sb
                tv = 1e-4 * v.abs().max()
            ref[t] += g[t, k] * v
            room[t] += g[t, k] * (tv + 16 * U * v.abs())
    room += ref.abs() * (2.0 ** -8 + 8 * U) + 16 * U * ref.abs().amax(1, keepdim=True)
    assert ((out.double() - ref).abs() <= room).all()


@pytest.mark.parametrize("T", [5, 300])
def test_layer_driver_with_a_scoring_rule_and_bf16_experts(T):
    """The softmax rule without groups is the plain routing: the layer's output is the same bits."""
    s = W.small_shape()
    wl = W.Workload("s", s, tokens=T, resident=s.n_experts // 2, skew=False)
    host = LY.HostLayer(wl)
    x = torch.randn(T, s.d, generator=R.gen(1)).to(BF).cuda()
    conf = torch.from_numpy(synth.gen_conf(wl)).cuda()
    out = []
    for score in (None, spice.route_score()):
        dev = LY.DeviceLayer(host)
        run = LY.LayerRun(s, T, dev.C, tau=wl.tau, layer_call=False, score=score)
        out.append(run.forward(dev, x, conf).clone())
        torch.cuda.synchronize()
        assert run.flags() == 0
    assert torch.equal(out[0], out[1])


def test_cache_admits_8_bit_experts():
    s = W.MoEShape(d=64, n_experts=8, top_k=2, inter=32, shared_inter=0, lore_rank=0, dtype=W.DTYPE_BF16)
    wl = W.Workload("i8c", s, tokens=1, resident=8, skew=False, wfmt=W.WFMT_INT8)
    w = [synth.gen_expert(wl, 0, e) for e in range(8)]
    t13, t2 = ([torch.from_numpy(a[i]).pin_memory() for a in w] for i in (0, 1))
    p13, p2 = (torch.zeros(3, t[0].numel(), dtype=torch.uint8, device="cuda") for t in (t13, t2))
    slot = torch.full((8,), -1, dtype=torch.int32, device="cuda")
    c = spice.ExpertCache(make_cfg(64, 8, 2, 32, 0, 0, 3, i8=True), 1, [[4, 1, 6]], t13, t2, [p13], [p2], [slot], load=True)
    for j, e in enumerate((4, 1, 6)):
        assert torch.equal(p13[j].cpu(), t13[e]) and torch.equal(p2[j].cpu(), t2[e])
    stream = torch.cuda.Stream()
    adm, ev = c.step(0, 0, np.array([[7, 4]], np.int32), np.array([[EXACT, HIT]], np.uint8), 2, copy_stream=stream)
    c.wait(0)
    torch.cuda.synchronize()
    assert adm == [7] and ev == [1]
    assert torch.equal(p13[1].cpu(), t13[7]) and torch.equal(p2[1].cpu(), t2[7])
    assert slot.cpu().tolist() == [-1, -1, -1, -1, 0, -1, 2, 1]
    c.close()


# ---- rows of H that are tiny ---------------------------------------------------------------------


@pytest.mark.parametrize("T,K", [(1, 2), (2, 3), (14, 2), (200, 2)])
def test_experts_tiny_rows(T, K):
    """Rows whose H lies below 127 / the largest fp32 (3.7e-37), down to a few thousand steps of the smallest one:
    their codes are the nearest integers too.  W2's scales lift the outputs back to ordinary sizes."""
    e = Experts(T, 64, 4, K, 96, 80, 4, seed=T)
    e.xs *= 2.0 ** -(56 + (torch.arange(T, device="cuda") + 11) % 14).float()  # from 2^-67 on
    for blob, k in [(b, 96) for b in e.w2] + [(e.w2s, 80)]:
        blob[64 * k:] = (blob[64 * k:].clone().view(F32) * 2.0 ** 110).view(torch.uint8)
    e.run()
    got = e.y_slots[e.pos]
    tops = [R.swiglu_i8_tiny_ref(e.xq, e.xs, e.w13s, e.w2s, 64, 80)[2]]
    e.near(e.y_shared, *R.swiglu_i8_tiny_ref(e.xq, e.xs, e.w13s, e.w2s, 64, 80)[:2])
    for x in range(4):
        s = (e.idx.cuda().reshape(-1) == x).nonzero()[:, 0]
        if s.numel():
            c = int(e.slot[x])
            y, tol, top = R.swiglu_i8_tiny_ref(e.xq[s // K], e.xs[s // K], e.w13[c], e.w2[c], 64, 96)
            e.near(got[s], y, tol)
            tops.append(top)
    tops = torch.cat(tops)
    assert (tops < 3.7e-37).any()
    assert T < 14 or ((tops > 1e-42) & (tops < 1e-40)).any() and ((tops > 1e-38) & (tops < 3.7e-37)).any()
    assert spice.spice_workspace_flags(e.ws, e.wsn) == 0


@pytest.mark.parametrize("T,C", [(1, 2), (3, 2), (17, 1), (60, 2), (400, 3)])
def test_experts_that_share_pool_slots(T, C):
    """More experts than pool slots, all resident: several of them have one slot's weights."""
    e = Experts(T, 80, 40, 4, 48, 32, C, seed=T)
    e.slot = (torch.arange(40, dtype=torch.int32) % C).cuda()
    e.cls = torch.full_like(e.cls, HIT)
    perm, inv, off = R.buckets_ref(e.idx.numpy(), e.cls.numpy(), 40)
    e.perm, e.offsets, e.pos = torch.from_numpy(perm).int().cuda(), torch.from_numpy(off).int().cuda(), torch.from_numpy(inv).cuda()
    e.run()
    e.check()


@pytest.mark.parametrize("T", [1, 40, 300])
@pytest.mark.parametrize("c", [HIT, LORE])
@pytest.mark.parametrize("bad", [1 << 30, -1, -(1 << 31)])
@pytest.mark.parametrize("at", [3, 6])
def test_a_bucket_of_impossible_size_raises_a_flag(T, c, bad, at):
    """A start that gives one bucket more than T K slots, or the one before it fewer than none: the flag is raised,
    the two are skipped and every other bucket's rows are right."""
    N, K, r = 6, 4, 8
    e = Experts(T, 64, N, K, 48, 32, N if c == HIT else 0, r=r, seed=T, lore=True)
    e.offsets[c, at] = bad  # the end of a bucket and the start of the next (or the class's end)
    e.run(lore=True)
    assert spice.spice_workspace_flags(e.ws, e.wsn, clear=True) == spice.SPICE_FLAG_BAD_INDEX
    e.near(e.y_shared, *R.swiglu_i8_ref(e.xq, e.xs, e.w13s, e.w2s, 64, 32))
    got = e.y_slots[e.pos]
    for x in range(N):
        s = (e.idx.cuda().reshape(-1) == x).nonzero()[:, 0]
        if s.numel() == 0:
            continue
        if x in (at - 1, at):
            assert (got[s] == 7).all()
        elif c == HIT:
            i = int(e.slot[x])
            e.near(got[s], *R.swiglu_i8_ref(e.xq[s // K], e.xs[s // K], e.w13[i], e.w2[i], 64, 48))
        else:
            y = R.lore_ref(e.x[s // K], e.lore_A[x], e.lore_B[x])
            e.near(got[s], y, 1e-4 * y.abs().amax(1, keepdim=True))


@pytest.mark.parametrize("T", [1, 40, 300])
def test_bad_starts_raise_a_flag(T):
    """Buckets of right sizes past the end of the slots."""
    for c in (HIT, LORE):
        e = Experts(T, 64, 4, 2, 48, 32, 4 if c == HIT else 0, r=8, seed=3, lore=True)
        e.offsets[c, 1:] += T * 2
        e.run(lore=True)
        assert spice.spice_workspace_flags(e.ws, e.wsn, clear=True) == spice.SPICE_FLAG_BAD_INDEX


# ---- scored routing in tiles: contractions and experts split over a group's blocks -----------------


@pytest.mark.parametrize("rule", [0, 2])
@pytest.mark.parametrize("size,tiles", R.SCORED_TILES)
def test_scored_routing_in_split_tiles(size, tiles, rule):
    """Long rows and many experts, on the whole workspace (twice: its counters are back at zero) and on the smallest
    one, which leaves no room for partial logits."""
    T, d, N, K, f32 = size
    say("route", size, tiles)
    rule = RULES[rule] if N % 4 == 0 and K <= N // 2 else dict(RULES[rule], groups=1, keep=1)
    r = Routing(T, d, N, K, F32 if f32 else BF, C=N // 3, seed=T + N, norm_topk=1)
    z = r.x.double() @ r.wg.double().t()
    room = float(2 * d * 2.0 ** -53 * (r.x.double().abs() @ r.wg.double().abs().t()).max())
    full, r.wsn = r.wsn, 1024
    with pytest.raises(spice.SpiceError) as e:
        r.run(**rule)
    base = int(str(e.value).split("needs ")[1].split()[0].rstrip(")"))
    assert base < full
    for r.wsn in (full, full, base):
        r.logits.fill_(9), r.idx.fill_(-9), r.perm.fill_(-9)
        r.run(**rule)
        assert torch.allclose(r.logits, z, rtol=0, atol=room)
        r.check(r.logits.cpu().numpy(), **rule)


@pytest.mark.parametrize("T", [4, 215, 300])
@pytest.mark.parametrize("rule", [RULES[2], RULES[3]])
def test_infinite_balance_biases(T, rule):
    """-inf: chosen only where a token's kept groups have fewer than K others, in no group value, the weight its
    score; +inf: first."""
    r = Routing(T, 64, 48, 5, C=9, seed=4)
    for low in ([0, 5, 30], list(range(0, 24)), list(range(1, 48)), list(range(48))):
        r.balance = (0.05 * torch.randn(48, generator=R.gen(8)))
        r.balance[low] = -float("inf")
        if len(low) == 3:
            r.balance[[7, 8, 40]] = float("inf")
        r.balance = r.balance.cuda()
        r.run(**rule)
        r.check(r.logits.cpu().numpy(), **rule)


@pytest.mark.parametrize("T,N,d", [(40, 48, 64), (230, 64, 2048), (250, 16, 2048), (120, 256, 1024), (250, 256, 2048)])
def test_scored_routing_copies_to_the_host_in_one_launch(T, N, d):
    """Rows of many slots, and the one-launch tiles, whole and split."""
    r = Routing(T, d, N, 5, C=9, seed=2)
    pin = lambda t: torch.zeros(t.shape, dtype=t.dtype).pin_memory()  # noqa: E731
    x, idx, w, cls = (pin(t) for t in (r.x, r.idx, r.w, r.cls))
    counts, ready = (torch.zeros(n, dtype=torch.int32).pin_memory() for n in (4, 1))
    rule = dict(sigmoid=True, groups=4, keep=2)
    r.run(**rule, host_out=spice.host_out(x, idx, w, cls, counts, ready, 78))
    torch.cuda.synchronize()
    r.check(r.logits.cpu().numpy(), **rule)
    for a, b in ((x, r.x), (idx, r.idx), (w, r.w), (cls, r.cls)):
        assert torch.equal(a, b.cpu())
    assert counts[:3].tolist() == torch.bincount(r.cls.flatten().long(), minlength=3).tolist() and ready.item() == 78


@pytest.mark.parametrize("size,parts", [R.SPLIT_CALLS[0], R.SPLIT_CALLS[1]])
def test_gate_of_a_split_shared_block(size, parts):
    e = Experts(*size, seed=5)
    e.w_sg = (0.05 * torch.randn(e.d, generator=R.gen(9))).to(BF).cuda()
    e.run()
    e.check()


@pytest.mark.parametrize("T", [1, 40])
def test_longest_contraction(T):
    """inter and shared_inter at their limit, every product of W2's at its largest: the sums stay in 32 bits."""
    I = 131056
    e = Experts(T, 16, 1, 1, I, I, 1, seed=1)
    e.xq[:] = 127
    for w13, w2 in ((e.w13[0], e.w2[0]), (e.w13s, e.w2s)):
        w13[:2 * I * 16] = 127  # codes
        w13[2 * I * 16:] = torch.full((2 * I,), 1e-3).cuda().view(torch.uint8)
        w2[:I * 16] = 128  # code -128
    e.run()
    e.check()
