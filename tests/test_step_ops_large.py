"""The steps around the LoRA linears where sizes pass 32 bits, launch grids, or the caches (the accesses past them are variants of their own).
References in 64 bits of the rows that hold something; tolerances as in tests/test_step_ops.py: a bf16 step of the value, fp32 sums in
units of their largest term."""

import pytest

from paper_2509_01193_amd import binding as bd
from test_step_ops import act64, near, ref_block_norm, ref_block_norm_rest, ref_gated_projections, test_gated as check_gated

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_logits_rows_beyond_32_bits():
    T, V, ld, k = 4, 1003, (1 << 30) + 8, 3
    mem = torch.empty(3 * ld + V, dtype=torch.bfloat16, device=DEV)
    z = mem.as_strided((T, V), (ld, 1))
    z.copy_((torch.randn(T, V, generator=torch.Generator().manual_seed(1)) * 3).bfloat16())
    target = torch.tensor([0, 1002, -1, 77], dtype=torch.int32, device=DEV)
    desc = bd.make_logprob_desc("bf16", T, V, ld, k)
    logp, lse, rest, ent = (torch.empty(T, device=DEV) for _ in range(4))
    top_logp, top_id = torch.empty(T, k, device=DEV), torch.empty(T, k, dtype=torch.int32, device=DEV)
    before = z.double().cpu()
    bd.lobra_token_logprob_fwd(desc, z, target, logp, lse, rest, ent, top_logp, top_id)
    w = torch.tensor([1.0, -2.0, 3.0, 0.5], device=DEV)
    bd.lobra_token_logprob_bwd(desc, z, target, lse, rest, None, w, None, z)
    torch.cuda.synchronize()
    p = torch.softmax(before, dim=1)
    lp = torch.log_softmax(before, dim=1)
    tgt = target.cpu().long()
    has = (tgt >= 0).double()
    near(logp, lp.gather(1, tgt.clamp(min=0)[:, None])[:, 0] * has, "f32", "logp")
    near(ent, -(p * lp).sum(dim=1), "f32", "entropy")
    assert torch.equal(top_id.cpu().long(), torch.sort(before, dim=1, descending=True, stable=True).indices[:, :k])
    one = torch.nn.functional.one_hot(tgt.clamp(min=0), V).double()
    near(z, (w.double().cpu() * has)[:, None] * (one - p), "bf16", "gradient", scale=2.0)


@pytest.mark.parametrize("T,d", [(540000, 4096), (9000, 4096), (2200000, 8)])
def test_block_norm_of_many_rows(T, d):
    """(540000 x 4096: 2.2e9 elements; 9000 x 4096: the backward pass past the caches; 2200000 rows: two launches forward.)  Gradients
    arrive at a few rows only, which make the sums."""
    n, eps, alpha = 3, 1e-5, 0.7
    off, task = [0, T // 3, T // 2 + 5, T - 4, T], [1, -1, 2, 0]
    rows = torch.tensor([0, 1, T // 3 - 1, T // 3, T // 2 + 5, T - 5, T - 4, T - 1])
    of = torch.tensor([next(t for k, t in enumerate(task) if off[k] <= r < off[k + 1]) for r in rows.tolist()])
    gen = torch.Generator(device=DEV).manual_seed(d)
    mk = lambda *s: torch.randn(*s, generator=gen, device=DEV, dtype=torch.bfloat16)
    dv = dict(r=mk(T, d), b=mk(T, d), w_post=mk(d), gate=mk(n, d), w_pre=mk(d), dr_out=None, dx=None)
    for k in ("dr_out", "dx"):
        dv[k] = torch.zeros(T, d, dtype=torch.bfloat16, device=DEV)
        dv[k][rows.to(DEV)] = mk(len(rows), d)
    v = {k: (t[rows.to(DEV)] if t.shape[0] == T else t).cpu() for k, t in dv.items()}
    plan = bd.Plan("bf16", T, d, 8, [0, 8, 16, 24], off, task)
    cfg = bd.BlockNormConfig(eps, alpha)
    r_out, x = torch.empty_like(dv["r"]), torch.empty_like(dv["r"])
    post, pre = torch.empty(T, device=DEV), torch.empty(T, device=DEV)
    bd.lobra_mlora_block_norm_fwd(plan, cfg, dv["r"], dv["b"], dv["w_post"], dv["gate"], dv["w_pre"], r_out, x, post, pre)
    ref, _, gate = ref_block_norm(d, v, eps, alpha, of)
    at = rows.to(DEV)
    near(r_out[at], ref["r_out"], "bf16", "r_out")
    rest = ref_block_norm_rest(d, v, eps, alpha, of, gate, r_out[at].cpu(), n)
    near(x[at], rest["x"], "bf16", "x")
    ws = torch.empty(bd.lobra_mlora_block_norm_workspace_bytes(plan), dtype=torch.uint8, device=DEV)
    dgate, dpost, dpre = torch.empty(n, d, device=DEV), torch.empty(d, device=DEV), torch.empty(d, device=DEV)
    dr, db = dv["dr_out"], dv["dx"]
    bd.lobra_mlora_block_norm_bwd(plan, cfg, r_out, dv["b"], dv["w_post"], dv["gate"], dv["w_pre"], post, pre, dr, db, dr, db, dgate, dpost, dpre, 0, ws)
    torch.cuda.synchronize()
    near(dr[at], rest["dr"], "bf16", "dr", fp32=4e-6)
    near(db[at], rest["db"], "bf16", "db", fp32=8e-6)
    for got, k in ((dgate, "dgate"), (dpost, "dw_post"), (dpre, "dw_pre")):
        near(got, rest[k], "f32", k, fp32=1e-5)
    dr[at], db[at] = 0, 0
    assert not bool(dr.any()) and not bool(db.any())


def test_gates_of_more_tasks_than_a_grid_has_rows():
    n, d = 70000, 4
    off, task = list(range(n + 11)), list(range(n)) + [-1] * 10
    of = torch.tensor(task)
    gen = torch.Generator().manual_seed(2)
    mk = lambda *s: torch.randn(*s, generator=gen)
    T = n + 10
    v = dict(r=mk(T, d), b=mk(T, d), w_post=None, gate=mk(n, d), w_pre=None, dr_out=mk(T, d), dx=None)
    dv = {k: (t.to(DEV) if t is not None else None) for k, t in v.items()}
    plan = bd.Plan("f32", T, d, 8, list(range(n + 1)), off, task)
    cfg = bd.BlockNormConfig(1e-5, 0.5)
    dr, db, dgate = torch.empty_like(dv["r"]), torch.empty_like(dv["r"]), torch.empty(n, d, device=DEV)
    ws = torch.empty(bd.lobra_mlora_block_norm_workspace_bytes(plan), dtype=torch.uint8, device=DEV)
    bd.lobra_mlora_block_norm_bwd(plan, cfg, dv["r"], dv["b"], None, dv["gate"], None, None, None, dv["dr_out"], None, dr, db, dgate, None, None, 0, ws)
    torch.cuda.synchronize()
    near(dgate, 0.5 * (v["dr_out"].double() * v["b"].double())[:n], "f32", "dgate")
    gate = torch.cat([v["gate"], torch.ones(1, d)])[of].double()
    near(db, 0.5 * gate * v["dr_out"].double(), "f32", "db")


def test_gradients_of_more_bytes_than_the_caches_hold():
    n, ranks, D = 3, [0, 33, 33, 80], 1 << 20
    gen = torch.Generator(device=DEV).manual_seed(3)
    g = torch.randn(ranks[-1], D, generator=gen, device=DEV)
    odd = torch.randn(7, 1001, generator=gen, device=DEV)
    for joint in (False, True):
        gset = bd.GradSet([(g, None, ranks), (odd, odd, [0, 1, 4, 7])], n)
        scale, most = torch.tensor([0.5, 2.0, -1.0], device=DEV), torch.tensor([1.0, 1e9, -1.0], device=DEV)
        norm, factor = torch.empty(n, device=DEV), torch.empty(n, device=DEV)
        ws = torch.empty(gset.ws_bytes, dtype=torch.uint8, device=DEV)
        sq = torch.tensor([sum(float(t[o[k]:o[k + 1]].double().square().sum()) for t, o in ((g, ranks), (odd, [0, 1, 4, 7]))) for k in range(n)])
        bd.lobra_grad_clip(gset, most, scale, None, norm, factor, None, bd.FLAG_JOINT_NORM if joint else 0, ws)
        torch.cuda.synchronize()
        ref = (sq.double() * scale.double().cpu() ** 2)
        ref = torch.sqrt(ref.sum().expand(n) if joint else ref)
        assert torch.all((norm.double().cpu() - ref).abs() <= 2.0 ** -23 * ref)
        want = scale.double().cpu() * torch.where(torch.tensor([True, joint, False]) & (ref > most.double().cpu()), most.double().cpu() / ref, 1.0)
        assert torch.all((factor.double().cpu() - want).abs() <= 2.0 ** -22 * want.abs())


@pytest.mark.parametrize("T,f", [(140000, 8192), (300000, 4104)])
def test_gated_projections_beyond_32_bits(T, f):
    d, ranks = 64, [8, 16]
    off, task = [0, T // 2, T - 3, T], [1, -1, 0]
    rows = torch.tensor([0, T // 2 - 1, T // 2, T - 4, T - 3, T - 1])
    of = torch.tensor([next(t for k, t in enumerate(task) if off[k] <= r < off[k + 1]) for r in rows.tolist()])
    gen = torch.Generator(device=DEV).manual_seed(f)
    mk = lambda std, *s: torch.randn(*s, generator=gen, device=DEV, dtype=torch.bfloat16) * std
    R = 2 * sum(ranks)
    w = dict(x=mk(1.0, T, d), W=mk(0.125, d, 2 * f), A=mk(0.125, R, d), B=mk(0.25, R, f), s=torch.tensor([0.5, 1.5], device=DEV))
    plan = bd.Plan("bf16", T, d, 2 * f, [0, 16, 48], off, task, n_proj=2)
    at = rows.to(DEV)
    small = {k: (t[at] if k == "x" else t).cpu() for k, t in w.items()}
    y = ref_gated_projections(small, f, ranks, of)
    a, _ = act64(0, y[:, :f])
    h_ref = a * y[:, f:]
    gu, h = torch.empty(T, 2 * f, dtype=torch.bfloat16, device=DEV), torch.empty(T, f, dtype=torch.bfloat16, device=DEV)
    hs = torch.empty(plan.h_save_bytes, dtype=torch.uint8, device=DEV)
    ws = torch.empty(max(bd.lobra_mlora_gated_workspace_bytes(plan, True), plan.bwd_ws_bytes, 16), dtype=torch.uint8, device=DEV)
    bd.lobra_mlora_gated_fwd(plan, 0, *w.values(), gu, h, hs, ws)
    torch.cuda.synchronize()
    # (2^-7 of the largest: the rounding of the projected activations and of [g | u], as in tests/test_step_ops.py)
    for got, ref, what in ((gu[at], y, "projections"), (h[at], h_ref, "h")):
        assert float((got.double().cpu() - ref).abs().max() / ref.abs().max()) <= 2.0 ** -7, what
    # gradients arrive at these rows alone
    dh = torch.zeros(T, f, dtype=torch.bfloat16, device=DEV)
    dh[at] = mk(1.0, len(rows), f)
    gk, dk = gu[at].double().cpu(), dh[at].double().cpu()
    a, da = act64(0, gk[:, :f])
    dy = torch.cat([dk * gk[:, f:] * da, dk * a], dim=1)
    dx, dA, dB = torch.empty(T, d, dtype=torch.bfloat16, device=DEV), torch.empty(R, d, device=DEV), torch.empty(R, f, device=DEV)
    bd.lobra_mlora_gated_bwd(plan, 0, *w.values(), gu, dh, hs, gu, dx, dA, dB, 0, ws)
    torch.cuda.synchronize()
    near(gu[at], dy, "bf16", "dgu", fp32=4e-6)
    from test_step_ops import ref_gated_back
    for got, ref, what in zip((dx[at], dA, dB), ref_gated_back(small, f, ranks, of, gu[at].double().cpu()), ("dx", "dA", "dB")):
        assert float((got.double().cpu() - ref).abs().max() / ref.abs().max()) <= 2e-2, what
    gu[at] = 0
    assert not bool(gu.any())


@pytest.mark.parametrize("T,d,f,ranks,batch,act", [
    (80, 264, 72, [8, 8], "tokens", 0), (97, 1000, 136, [24], "tokens", 1), (112, 64, 264, [8], "mixed", 0), (113, 136, 8200, [8], "bare", 0),
    (128, 4096, 64, [16, 64, 8], "tokens", 1), (128, 512, 1376, [16] * 9, "tokens", 0), (127, 2056, 520, [64, 8], "mixed", 0),
    (129, 520, 192, [16], "tokens", 0),
])
def test_gated_few_tokens(T, d, f, ranks, batch, act):
    """(up to 128 tokens are one stream over the weights)"""
    check_gated("bf16", T, d, f, ranks, batch, act)


@pytest.mark.parametrize("T,d,f,ranks,batch,act", [
    (167, 2176, 1432, [8] * 16, "mixed", 0), (200, 4096, 512, [16, 8], "tokens", 1), (300, 4096, 256, [64, 8], "mixed", 0), (150, 2048, 264, [8], "bare", 0),
    (500, 1032, 64, [16], "one", 0), (140, 8192, 128, [8], "mixed", 1),
])
def test_gated_sums_of_a_split_product(T, d, f, ranks, batch, act):
    check_gated("bf16", T, d, f, ranks, batch, act)


def test_gated_workspace_without_room_for_sums():
    """What a smaller workspace takes: the product rounds [g | u], as where it is not split."""
    T, d, f = 200, 4096, 512
    gen = torch.Generator().manual_seed(1)
    mk = lambda std, *s: (torch.randn(*s, generator=gen) * std).bfloat16().to(DEV)
    plan = bd.Plan("bf16", T, d, 2 * f, [0, 16], [0, T], [0], n_proj=2)
    w = mk(1.0, T, d), mk(1 / 64, d, 2 * f), mk(1 / 64, 16, d), mk(0.3, 16, f), torch.ones(1, device=DEV)
    hs = torch.empty(plan.h_save_bytes, dtype=torch.uint8, device=DEV)
    gu, h, h1 = torch.empty(T, 2 * f, dtype=torch.bfloat16, device=DEV), *(torch.empty(T, f, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    ws = torch.empty(bd.lobra_mlora_gated_workspace_bytes(plan, True), dtype=torch.uint8, device=DEV)
    bd.lobra_mlora_gated_fwd(plan, 0, *w, gu, h, hs, ws)
    bd.lobra_mlora_gated_fwd(plan, 0, *w, gu, h1, hs, ws[:256])
    torch.cuda.synchronize()
    assert float((h.double() - h1.double()).abs().max() / h.double().abs().max()) <= 2.0 ** -7


@pytest.mark.parametrize("T,d,f,ranks,batch,act", [
    (1, 1, 8, [8], "one", 0), (2, 15, 64, [8], "bare", 1), (16, 16, 72, [8, 8], "tokens", 0), (17, 17, 136, [24], "tokens", 1), (33, 63, 8, [8], "mixed", 0),
    (28, 919, 256, [16] * 8, "tokens", 0), (48, 4097, 64, [64, 8], "tokens", 1), (64, 130, 2056, [8, 16], "mixed", 0), (65, 130, 200, [8], "tokens", 0),
])
def test_gated_few_tokens_fp32(T, d, f, ranks, batch, act):
    check_gated("f32", T, d, f, ranks, batch, act)
