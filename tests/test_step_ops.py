"""The steps around the LoRA linears: gated feed-forward block, norms around a residual block, log probabilities, gradient norms.

Each operator against a plain implementation in 64 bits, at the sizes and masks where it can go wrong; gradients also against differences of
the operator's own forward; refusals.  Tolerances: a result rounded to bf16 is off by half a step, 2^-9 of its value, and 2^-8 allows for
fp32 sums that fall on the other side of a rounding; fp32 results are held to a few units in the last place of the largest term of their
sum, which grows with the square root of its length (2e-6 of the tensor's largest for the lengths here).
"""
import ctypes
import math

import numpy as np
import pytest

from paper_2509_01193_amd import binding as bd

torch = pytest.importorskip("torch")
DEV = "cuda:0"
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def near(got, ref, dtype, what, scale=None, fp32=2e-6):
    """|got - ref| <= one bf16 step of the value (bf16), or fp32 * the largest (fp32 results)."""
    got, ref = got.detach().double().cpu(), ref.double().cpu()
    assert got.shape == ref.shape, what
    top = float(ref.abs().max()) if scale is None else scale
    bound = fp32 * top * torch.ones_like(ref)
    if dtype == "bf16":
        bound = ref.abs() * 2.0 ** -8 + 2 * fp32 * top
    off = (got - ref).abs() - bound
    bad = ~((off <= 0) | (torch.isnan(got) & torch.isnan(ref)) | (got == ref))
    assert not bool(bad.any()), "%s: %d of %d, e.g. %r for %r" % (what, int(bad.sum()), bad.numel(), got[bad][:3].tolist(), ref[bad][:3].tolist())


def guarded(*shape, dtype, fill=0xC3):
    """A device tensor between two margins; the second result says whether the margins are as they were."""
    n = int(np.prod(shape)) * torch.empty(0, dtype=dtype).element_size()
    buf = torch.full(((n + 15) // 16 * 16 + 512,), fill, dtype=torch.uint8, device=DEV)
    view = buf[256:256 + n].view(dtype).view(*shape)
    return view, lambda: bool((buf[:256] == fill).all()) and bool((buf[256 + n:] == fill).all())


# ------------------------------------------------------------------------------------------------------------------
# log probabilities
# ------------------------------------------------------------------------------------------------------------------
def ref_logprob(z, target, k):
    z = z.double().cpu()
    T, V = z.shape
    m = z.max(dim=1).values
    m0 = torch.where(torch.isinf(m) & (m < 0), torch.zeros_like(m), m)
    e = torch.exp(z - m0[:, None])
    s = e.sum(dim=1)
    none = s == 0
    lse = torch.where(none, -math.inf, m0 + torch.log(s))
    lp = (z - m0[:, None]) - torch.log(s)[:, None]
    p = torch.where(none[:, None], torch.zeros_like(e), e / s[:, None])
    ent = torch.where(none, 0.0, -torch.where(p > 0, p * torch.where(p > 0, lp, torch.zeros_like(lp)), torch.zeros_like(p)).sum(dim=1))
    ent = torch.where(torch.isnan(lse), lse, ent)
    tgt = target.cpu().long()
    has = (tgt >= 0) & (tgt < V)
    at = z.gather(1, tgt.clamp(0, V - 1)[:, None])[:, 0]
    # (not z - lse, which a row of the type's lowest value would lose its ln V in)
    logp = torch.where(has, torch.where(none, torch.full_like(at, -math.inf), (at - m0) - torch.log(s)), torch.zeros_like(at))
    top_id = torch.full((T, k), -1, dtype=torch.int64)
    top_lp = torch.full((T, k), -math.inf, dtype=torch.float64)
    if k:
        number = ~torch.isnan(z)
        order = torch.sort(torch.where(number, z, -math.inf), dim=1, descending=True, stable=True).indices
        for i in range(T):
            ids = [j for j in order[i, :k + int((~number[i]).sum())].tolist() if number[i, j]][:k]
            top_id[i, :len(ids)] = torch.tensor(ids, dtype=torch.int64)
            top_lp[i, :len(ids)] = -math.inf if none[i] else (z[i, ids] - m0[i]) - torch.log(s[i])
    return dict(lse=lse, logp=logp, ent=ent, p=p, top_id=top_id, top_lp=top_lp, has=has, none=none)


def ref_logprob_grad(z, target, r, w, v):
    z, V = z.double().cpu(), z.shape[1]
    w, v = w.double().cpu() * r["has"], v.double().cpu()
    x = torch.where(r["p"] > 0, torch.log(r["p"]), torch.zeros_like(z))
    g = -r["p"] * (w[:, None] + v[:, None] * (x + r["ent"][:, None]))
    rows = torch.arange(z.shape[0])[r["has"]]
    g[rows, target.cpu().long()[r["has"]]] += w[r["has"]]
    g[((w == 0) & (v == 0)) | r["none"]] = 0
    return g


def logits_of(kind, T, V, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    z = torch.randn(T, V, generator=g) * 3
    if kind == "offset":                     # a common offset that exp alone would not survive
        z += 1000
    elif kind == "masked":                   # type's infinity in most places, rows of one token, a row of none
        z[torch.rand(T, V, generator=g) < 0.9] = -math.inf
        z[0] = -math.inf
        if T > 1:
            z[1] = -math.inf
            z[1, V // 2] = 4.0
    elif kind == "lowest":                   # masks of the type's lowest value, a row of nothing else
        low = torch.finfo(DT[dtype]).min
        z[torch.rand(T, V, generator=g) < 0.5] = low
        z[0] = low
    elif kind == "equal":                    # ties everywhere
        z = torch.round(z / 4)
        z[0] = 0.25
    elif kind == "one_stride":               # all the large ones where one thread of a workgroup looks
        z[:, ::2048] += 40
        z[:, 1::2048] += 40
    elif kind == "nan":
        z[0, V // 3] = math.nan
        if T > 1:
            z[1, 0] = math.inf
    return z.to(DT[dtype])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,V,k,kind", [
    (1, 1, 1, "plain"), (3, 7, 32, "plain"), (5, 64, 5, "plain"), (2, 1000, 32, "plain"), (7, 4099, 20, "offset"), (3, 32000, 20, "plain"),
    (700, 9001, 3, "plain"), (4, 5000, 20, "masked"), (6, 257, 32, "masked"), (4, 20001, 8, "lowest"), (5, 9000, 32, "equal"),
    (2, 40960, 32, "equal"), (2, 65536, 32, "one_stride"), (520, 8200, 32, "one_stride"), (3, 3000, 4, "nan"), (1, 131072, 32, "plain"),
])
def test_logprob_forward(dtype, T, V, k, kind):
    z = logits_of(kind, T, V, dtype, T + V)
    target = torch.randint(0, V, (T,), generator=torch.Generator().manual_seed(V))
    target[T // 2] = -1 if T > 1 else target[0]
    if T > 2:
        target[2] = V                        # beyond the vocabulary: none either
    r = ref_logprob(z, target, k)
    zd, tg = z.to(DEV), target.to(torch.int32).to(DEV)
    for ent in (True, False):
        o = {n: guarded(T, dtype=torch.float32) for n in ("logp", "lse", "ent")}
        tl, ti = guarded(T, k, dtype=torch.float32), guarded(T, k, dtype=torch.int32)
        bd.lobra_token_logprob_fwd(bd.make_logprob_desc(dtype, T, V, top_k=k), zd, tg, o["logp"][0], o["lse"][0], None,
                                   o["ent"][0] if ent else None, tl[0], ti[0])
        torch.cuda.synchronize()
        assert all(ok() for _, ok in list(o.values()) + [tl, ti])
        # a difference z - lse of a few ulp of its larger term
        tol = 4e-6 + 2.0 ** -22 * max([0.0] + [abs(v) for v in r["lse"].tolist() if abs(v) < 1e30])
        for name, ref in (("logp", r["logp"]), ("lse", r["lse"])) + ((("ent", r["ent"]),) if ent else ()):
            got = o[name][0].double().cpu()
            same = (got == ref) | (torch.isnan(got) & torch.isnan(ref)) | ((got - ref).abs() <= tol + 2.0 ** -22 * ref.abs())
            # (+inf in a row: lse is NaN here, by definition)
            same |= torch.isnan(got) & torch.isinf(z.double()).logical_and(z.double() > 0).any(dim=1)
            assert bool(same.all()), (name, got[~same][:4], ref[~same][:4])
        clean = ~torch.isnan(r["lse"]) & ~(torch.isinf(z.double()) & (z.double() > 0)).any(dim=1)
        assert torch.equal(ti[0].long().cpu()[clean], r["top_id"][clean])
        got, ref = tl[0].double().cpu()[clean], r["top_lp"][clean]
        assert bool(((got == ref) | ((got - ref).abs() <= tol + 2.0 ** -22 * ref.abs())).all())
        ids = ti[0].cpu()
        assert int(ids.max()) < V and int(ids.min()) >= -1
        for row in ids.tolist():             # no token twice
            real = [j for j in row if j >= 0]
            assert len(set(real)) == len(real)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("T,V,pad,kind,with_ent", [
    (1, 1, 0, "plain", True), (3, 7, 1, "plain", False), (9, 1000, 0, "plain", True), (4, 4099, 5, "offset", False), (5, 3001, 7, "masked", True),
    (4, 2048, 0, "lowest", True), (2500, 520, 0, "plain", False), (2, 50001, 0, "plain", True),
])
def test_logprob_backward(dtype, in_place, T, V, pad, kind, with_ent):
    z = logits_of(kind, T, V, dtype, T * V + pad)
    g = torch.Generator().manual_seed(T)
    target = torch.randint(-1, V, (T,), generator=g)
    w, v = torch.randn(T, generator=g), torch.randn(T, generator=g) if with_ent else torch.zeros(T)
    w[T // 2] = 0
    if T > 3:
        w[3], v[3] = 0, 0
    r = ref_logprob(z, target, 0)
    ref = ref_logprob_grad(z, target, r, w, v)
    wide, ok = guarded(T, V + pad, dtype=DT[dtype])
    wide[:, V:] = 7.0
    wide[:, :V] = z.to(DEV)
    zd = wide[:, :V]
    out, ok2 = (zd, ok) if in_place else guarded(T, V + pad, dtype=DT[dtype])
    if not in_place:
        out[:, V:] = 7.0
        whole, out = out, out[:, :V]
    else:
        whole = wide
    desc = bd.make_logprob_desc(dtype, T, V, ld=V + pad)
    lse, ent, rest = (torch.empty(T, device=DEV) for _ in range(3))
    tg, wd, vd = target.to(torch.int32).to(DEV), w.to(DEV), v.to(DEV) if with_ent else None
    bd.lobra_token_logprob_fwd(desc, zd, tg, None, lse, rest, ent)
    bd.lobra_token_logprob_bwd(desc, zd, tg, lse, rest, ent if with_ent else None, wd, vd, out)
    torch.cuda.synchronize()
    assert ok() and ok2() and (pad == 0 or bool((whole[:, V:] == 7.0).all()))
    # p = exp(z - lse) with lse in fp32: relative error of an ulp of lse, next to fp32 products
    top = float((w.abs() + v.abs() * 20).max())
    near(out, ref, dtype, "dlogits", scale=top, fp32=2e-6 + 2.0 ** -23 * max([0.0] + [abs(x) for x in r["lse"].tolist() if abs(x) < 1e30]))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_logprob_of_a_barred_target(dtype):
    """logp is -inf; the gradient is dlogp at the target, -dlogp p elsewhere, 0 at the other barred tokens."""
    T, V = 3, 1000
    z = torch.randn(T, V, generator=torch.Generator().manual_seed(2))
    z[:, 100:200] = -math.inf
    z = z.to(DT[dtype])
    target, w = torch.tensor([150, 199, 5], dtype=torch.int32), torch.tensor([0.75, -2.0, 1.0])
    desc, zd = bd.make_logprob_desc(dtype, T, V), z.to(DEV)
    logp, lse, rest, dz = torch.empty(T, device=DEV), torch.empty(T, device=DEV), torch.empty(T, device=DEV), torch.empty_like(zd)
    bd.lobra_token_logprob_fwd(desc, zd, target.to(DEV), logp, lse, rest)
    bd.lobra_token_logprob_bwd(desc, zd, target.to(DEV), lse, rest, None, w.to(DEV), None, dz)
    torch.cuda.synchronize()
    assert logp[:2].tolist() == [-math.inf, -math.inf] and math.isfinite(float(logp[2]))
    ref = -w.double()[:, None] * torch.softmax(z.double(), dim=1)
    ref[torch.arange(T), target.long()] += w.double()
    assert dz[0, 150].item() == 0.75 and dz[1, 199].item() == -2.0
    others = dz[:, 100:200].clone()
    others[0, 50], others[1, 99] = 0, 0
    assert not bool(others.any())
    near(dz, ref, dtype, "dlogits", scale=2.0)


@pytest.mark.gpu
def test_logprob_gradient_against_differences():
    T, V, eps = 6, 777, 2e-2
    g = torch.Generator(device=DEV).manual_seed(5)
    z = torch.randn(T, V, device=DEV, generator=g) * 2
    dirn = torch.randn(T, V, device=DEV, generator=g)
    target = torch.randint(0, V, (T,), device=DEV, generator=g).int()
    w, v = torch.randn(T, device=DEV, generator=g), torch.randn(T, device=DEV, generator=g)
    desc = bd.make_logprob_desc("f32", T, V)

    def loss(x):
        logp, ent = torch.empty(T, device=DEV), torch.empty(T, device=DEV)
        bd.lobra_token_logprob_fwd(desc, x.contiguous(), target, logp, None, None, ent)
        return float((w.double() * logp.double() + v.double() * ent.double()).sum())

    lse, ent, dz = torch.empty(T, device=DEV), torch.empty(T, device=DEV), torch.empty(T, V, device=DEV)
    bd.lobra_token_logprob_fwd(desc, z, target, None, lse, None, ent)
    bd.lobra_token_logprob_bwd(desc, z, target, lse, None, ent, w, v, dz)
    slope = float((dz.double() * dirn.double()).sum())
    # fourth-order differences: the fifth derivative times eps^4, and 1e-6 of each of four values over eps
    got = (8 * (loss(z + eps * dirn) - loss(z - eps * dirn)) - (loss(z + 2 * eps * dirn) - loss(z - 2 * eps * dirn))) / (12 * eps)
    assert abs(got - slope) <= 1e-3 * max(1.0, abs(slope)), (got, slope)


def test_logprob_refusals():
    L = bd.lib()
    desc = lambda **kw: ctypes.byref(bd.LogprobDesc(*[{**dict(dtype=bd.BF16, V=100, T=4, ld=0, top_k=0), **kw}[n] for n in ("dtype", "V", "T", "ld", "top_k")]))
    p, f = ctypes.c_void_p(4096), ctypes.c_void_p(8192)
    fwd = lambda d, z=p, o=f: L.lobra_token_logprob_fwd(d, z, f, o, f, f, f, None, None, None)
    bwd = lambda d, z=p, lse=f, ent=f, dent=f, dz=p: L.lobra_token_logprob_bwd(d, z, f, lse, f, ent, f, dent, dz, None)
    SHAPE, NULL, ALIGN, DTYPE = -2, -1, -8, -3
    for call in (fwd, bwd):
        assert call(None) == NULL
        assert call(desc(dtype=5)) == DTYPE
        for bad in (dict(V=0), dict(V=(1 << 24) + 1), dict(T=-1), dict(T=1 << 31), dict(ld=99), dict(ld=-1), dict(top_k=-1), dict(top_k=33),
                    dict(ld=1 << 59)):
            assert call(desc(**bad)) == SHAPE, bad
        assert call(desc(T=0)) == bd.OK
        assert call(desc(), z=None) == NULL
        assert call(desc(), z=ctypes.c_void_p(4098)) == ALIGN
    assert fwd(desc(), o=ctypes.c_void_p(8194)) == ALIGN
    assert bwd(desc(), lse=None) == NULL and bwd(desc(), dz=None) == NULL and bwd(desc(), ent=None) == NULL
    assert bwd(desc(), dz=ctypes.c_void_p(4104)) == ALIGN
    z = torch.zeros(4, 100)
    with pytest.raises(AssertionError):
        bd.lobra_token_logprob_fwd(bd.make_logprob_desc("bf16", 4, 100), z, None, stream=0)
    with pytest.raises(AssertionError):
        bd.lobra_token_logprob_fwd(bd.make_logprob_desc("f32", 4, 100, ld=104), z, None, stream=0)


def test_logprob_refuses_other_types_and_short_rows():
    """fp16 logits are no bf16 ones, int64 targets no int32 ones, and every array of the rows has a number for each: what is refused is not
    read as what it is not.  (On the CPU: a call that goes through has no rows.)"""
    T, V, k = 4, 100, 3
    f, i = torch.zeros(T), torch.zeros(T, dtype=torch.int32)
    top = dict(top_logp=torch.zeros(T, k), top_id=torch.zeros(T, k, dtype=torch.int32))
    z = torch.zeros(T, V, dtype=torch.bfloat16)
    desc, wide = bd.make_logprob_desc("bf16", T, V, top_k=k), bd.make_logprob_desc("f32", T, V)

    def fwd(**kw):
        a = {**dict(desc=desc, logits=z, target=i, logp=f, lse=f, lse_rest=f, entropy=f), **top, **kw}
        bd.lobra_token_logprob_fwd(**a, stream=0)

    def bwd(**kw):
        a = {**dict(desc=desc, logits=z, target=i, lse=f, lse_rest=f, entropy=f, dlogp=f, dentropy=f, dlogits=z), **kw}
        bd.lobra_token_logprob_bwd(**a, stream=0)

    for call, names in ((fwd, ("logp", "lse", "lse_rest", "entropy")), (bwd, ("lse", "lse_rest", "entropy", "dlogp", "dentropy"))):
        for bad in (z.half(), z.float(), z.short()):
            with pytest.raises(AssertionError):
                call(logits=bad)
        for bad in (z.float().int(), z.float().double()[:, :V]):
            with pytest.raises(AssertionError):
                call(desc=wide, logits=bad)
        for bad in (i.long(), i.float(), i[:T - 1]):
            with pytest.raises(AssertionError):
                call(target=bad)
        for name in names:
            for bad in (f.double(), f.bfloat16(), f.int(), f[:T - 1]):
                with pytest.raises(AssertionError):
                    call(**{name: bad})
    with pytest.raises(AssertionError):
        bwd(dlogits=z.half())
    for bad in (dict(top_id=top["top_id"].long()), dict(top_id=top["top_id"][:, :2].contiguous()), dict(top_logp=top["top_logp"].double()),
                dict(top_logp=top["top_logp"][1:])):
        with pytest.raises(AssertionError):
            fwd(**bad)
    none = bd.make_logprob_desc("bf16", 0, V, top_k=k)
    bd.lobra_token_logprob_fwd(none, z[:0], i[:0], f[:0], f[:0], f[:0], f[:0], top["top_logp"][:0], top["top_id"][:0], stream=0)
    bd.lobra_token_logprob_bwd(none, z[:0], i[:0], f[:0], f[:0], f[:0], f[:0], f[:0], z[:0], stream=0)


# ------------------------------------------------------------------------------------------------------------------
# gradient norms and clipping
# ------------------------------------------------------------------------------------------------------------------
def ref_clip(grads, ranks, gs, most, step, joint):
    n = len(gs)
    sq = np.zeros(n)
    for g, off in zip(grads, ranks):
        for t in range(n):
            with np.errstate(over="ignore", invalid="ignore"):
                sq[t] += np.square(g[off[t]:off[t + 1]].astype(np.float64)).sum()
    with np.errstate(invalid="ignore"):
        total = gs.astype(np.float64) ** 2 * sq
    norm = np.sqrt(np.full(n, total.sum()) if joint else total)
    fine = norm <= np.finfo(np.float32).max
    f = np.where((most >= 0) & (norm > most), most / np.where(norm > 0, norm, 1), 1.0) * gs
    f = np.where(fine, f, 0.0)
    return norm, f, np.where(fine, step, 0)


@pytest.mark.gpu
@pytest.mark.parametrize("joint", [False, True])
@pytest.mark.parametrize("scaled,limited", [(True, True), (False, True), (True, False)])
@pytest.mark.parametrize("case", ["one", "layers", "odd", "empty", "none", "huge", "bad"])
def test_grad_clip(case, joint, scaled, limited):
    rng = np.random.default_rng(len(case))
    n = {"one": 1, "none": 3}.get(case, 4)
    layers = {"one": [([0, 8], 64)], "layers": [([0, 16, 32, 40, 48], 4096), ([0, 16, 32, 40, 48], 1376), ([0, 3, 4, 100, 101], 5000)],
              "odd": [([0, 1, 4, 5, 12], 37), ([0, 3, 6, 9, 12], 1), ([0, 5, 6, 7, 8], 40001)], "empty": [([0, 0, 7, 7, 9], 100)], "none": [],
              "huge": [([0, 2, 4, 6, 8], 100)], "bad": [([0, 2, 4, 6, 8], 1000), ([0, 2, 4, 6, 8], 77)]}[case]
    ranks = [np.asarray(r) for r, _ in layers]
    grads = [rng.standard_normal((r[-1], d)).astype(np.float32) for r, d in layers]
    if case == "huge":                        # squares that fp32 does not hold, and squares that vanish in it
        grads[0][:2] *= 1e30
        grads[0][2:4] *= 1e-30
        grads[0][4:6] = 3e38
    if case == "bad":
        grads[0][3, 500] = np.inf
        grads[1][7, 76] = np.nan
    gs = (rng.random(n) + 0.5).astype(np.float32) * np.float32([1, -1, 1, 1][:n])
    if not scaled:
        gs = np.ones(n, np.float32)
    most = np.asarray([1.0, 1e9, -1.0, np.nan][:n], np.float32)
    step = np.arange(1, n + 1, dtype=np.int32)
    lim = most if limited else np.full(n, -1.0)
    norm, f, so = ref_clip(grads, ranks, gs, lim.astype(np.float64), step, joint)
    up = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(DEV)
    gd = [up(g) for g in grads]
    outs = [guarded(*g.shape, dtype=torch.float32) for g in gd]
    for device_mem in (False, True):
        tensors = [(g, o[0], r) for g, o, r in zip(gd, outs, ranks)]
        mem = torch.empty(bd.grad_set_device_bytes(tensors, n), dtype=torch.uint8, device=DEV) if device_mem else None
        gset = bd.GradSet(tensors, n, device_mem=mem)
        ws, ws_ok = guarded(gset.ws_bytes, dtype=torch.uint8)
        nd, cd, sd = (guarded(n, dtype=t) for t in (torch.float32, torch.float32, torch.int32))
        bd.lobra_grad_clip(gset, up(most) if limited else None, up(gs) if scaled else None, up(step), nd[0], cd[0], sd[0],
                           bd.FLAG_JOINT_NORM if joint else 0, ws)
        torch.cuda.synchronize()
        assert ws_ok() and all(o[1]() for o in outs + [nd, cd, sd])
        got = nd[0].double().cpu().numpy()
        with np.errstate(over="ignore"):
            ref32 = norm.astype(np.float32).astype(np.float64)
        ok = (got == ref32) | (np.isnan(got) & np.isnan(ref32)) | (np.abs(got - ref32) <= 2.0 ** -23 * np.abs(ref32))
        assert ok.all(), (got, ref32)
        assert np.allclose(cd[0].cpu().numpy(), f, rtol=2.0 ** -22, atol=0), (cd[0], f)
        assert np.array_equal(sd[0].cpu().numpy(), so)
        scale = cd[0].cpu().numpy()
        for g, o, r in zip(grads, outs, ranks):
            per = np.repeat(scale, np.diff(r))[:, None]
            with np.errstate(invalid="ignore"):
                assert np.array_equal(o[0].cpu().numpy(), np.where(per == 0, np.float32(0), g * per))
    if case in ("layers", "odd"):
        # in place, the scale over the gradient scale, nothing else wanted
        gset = bd.GradSet([(g, g, r) for g, r in zip(gd, ranks)], n)
        ws, both = torch.empty(gset.ws_bytes, dtype=torch.uint8, device=DEV), up(gs)
        bd.lobra_grad_clip(gset, up(most) if limited else None, both, None, None, both, None, bd.FLAG_JOINT_NORM if joint else 0, ws)
        torch.cuda.synchronize()
        assert torch.equal(both, cd[0])
        assert all(torch.equal(g, o[0]) for g, o in zip(gd, outs))


def test_grad_set_refusals():
    L = bd.lib()
    g16, g4 = ctypes.c_void_p(4096).value, 4100
    off = np.asarray([0, 4, 8], np.int32)
    ptr = off.ctypes.data_as(ctypes.POINTER(ctypes.c_int32))
    n = ctypes.c_size_t()

    def size(grad=g16, out=None, D=16, ro=ptr, n_tensors=1, n_tasks=2, arr=True):
        t = (bd.GradTensor * 1)(bd.GradTensor(grad, out, D, ro))
        return L.lobra_grad_set_device_bytes(t if arr else None, n_tensors, n_tasks, ctypes.byref(n))

    assert size() == bd.OK and n.value > 0
    assert size(grad=None) == -1 and size(ro=None) == -1 and size(arr=False) == -1
    assert size(D=0) == -2 and size(D=(1 << 20) + 1) == -2 and size(n_tensors=-1) == -2 and size(n_tasks=-1) == -2
    assert size(grad=g4) == -8 and size(out=g4) == -8
    for bad in ([1, 4, 8], [0, 5, 4]):
        b = np.asarray(bad, np.int32)
        assert size(ro=b.ctypes.data_as(ctypes.POINTER(ctypes.c_int32))) == -6
    assert L.lobra_grad_set_create(None, 0, 1, None) == -1
    assert L.lobra_grad_set_workspace_bytes(None, ctypes.byref(n)) == -10
    assert L.lobra_grad_clip(None, None, None, None, None, None, None, 0, None, 0, None) == -10
    assert L.lobra_grad_set_destroy(None) == bd.OK


@pytest.mark.parametrize("use", [lambda t, n: bd.GradSet(t, n), lambda t, n: bd.grad_set_device_bytes(t, n)], ids=["set", "bytes"])
def test_grad_set_refuses_other_types_and_tables(use):
    """What the library would read or write beyond its end: elements of two bytes, and a table of fewer tasks.  Nothing is launched or looked up."""
    f32, short = torch.zeros(8, 16), [0, 4, 8]
    for other in (torch.bfloat16, torch.float16, torch.float64, torch.int32):
        with pytest.raises(AssertionError, match="fp32"):
            use([(f32, None, short), (torch.zeros(8, 16, dtype=other), None, short)], 2)
        with pytest.raises(AssertionError, match="fp32"):
            use([(f32, torch.zeros(8, 16, dtype=other), short)], 2)
    for n_tasks, table in ((3, [0, 4, 8]), (1, [0, 4, 8]), (2, [0, 8]), (2, [0])):
        with pytest.raises(AssertionError, match="rank_off"):
            use([(f32, None, table)], n_tasks)
    assert bd.grad_set_device_bytes([(f32, f32, short)], 2) > 0


@pytest.mark.gpu
def test_grad_clip_refusals():
    g = torch.zeros(8, 16, device=DEV)
    gset = bd.GradSet([(g, None, [0, 4, 8])], 2)
    ws, v, st = torch.empty(gset.ws_bytes, dtype=torch.uint8, device=DEV), torch.ones(2, device=DEV), torch.ones(2, dtype=torch.int32, device=DEV)
    call = lambda **kw: bd.lobra_grad_clip(gset, v, v, kw.get("step"), v.clone(), None, kw.get("step_out"), ws=kw.get("ws", ws), check=False)
    assert call() == bd.OK
    assert call(step=st) == -1 and call(step_out=st) == -1
    assert call(ws=None) == -7 and call(ws=ws[:gset.ws_bytes - 1]) == -7 and call(ws=torch.empty(gset.ws_bytes + 16, dtype=torch.uint8, device=DEV)[4:]) == -8


def test_grad_clip_refuses_other_types_and_fewer_tasks():
    """Per-task arrays of another type, or of fewer tasks than the set has.  (On the CPU: the set has no tensors and is never made.)"""
    n = 3
    gset = bd.GradSet.__new__(bd.GradSet)
    gset.handle, gset.n_tasks, gset.ws_bytes = ctypes.c_void_p(), n, 16
    f, i = torch.zeros(n), torch.zeros(n, dtype=torch.int32)

    def clip(**kw):
        a = {**dict(max_norm=f, grad_scale=f, step=i, norm=f, clip_scale=f, step_out=i), **kw}
        return bd.lobra_grad_clip(gset, **a, stream=0, check=False)

    assert clip() == -10                     # (no set: the library's own refusal)
    for name in ("max_norm", "grad_scale", "norm", "clip_scale"):
        for bad in (f.double(), f.bfloat16(), f.int(), f[:n - 1]):
            with pytest.raises(AssertionError):
                clip(**{name: bad})
    for name in ("step", "step_out"):
        for bad in (i.long(), i.float(), i[:n - 1]):
            with pytest.raises(AssertionError):
                clip(**{name: bad})


# ------------------------------------------------------------------------------------------------------------------
# norms around a residual block
# ------------------------------------------------------------------------------------------------------------------
def batch_of(kind, T, n):
    """(segment offsets, tasks)"""
    if kind == "one":
        return [0, T], [0]
    if kind == "bare":
        return [0, T], [-1]
    rng = np.random.default_rng(T)
    off, task = [0], []
    while off[-1] < T:
        k = 1 if kind == "tokens" else int(rng.integers(0, 60))
        off.append(min(off[-1] + k, T))
        task.append(int(rng.integers(-1, n)))
    return off, task


def ref_block_norm(d, v, eps, alpha, of):
    """r', x, and from the stored r' everything of backward."""
    q = {k: (t.double().cpu() if t is not None else None) for k, t in v.items()}
    gate = torch.ones_like(q["r"])
    if q["gate"] is not None:
        gate = torch.where((of >= 0)[:, None], q["gate"][of.clamp(min=0)], gate)
    o = {}
    if q["b"] is None:
        rp = v["r"]
    else:
        n = 1 / torch.sqrt((q["b"] ** 2).mean(dim=1, keepdim=True) + eps) if q["w_post"] is not None else torch.ones(len(of), 1, dtype=torch.float64)
        bh = q["b"] * n
        wp = q["w_post"] if q["w_post"] is not None else torch.ones(d, dtype=torch.float64)
        o["r_out"] = q["r"] + alpha * gate * wp * bh
        rp = o["r_out"].to(v["r"].dtype)
        o["rstd_post"] = n[:, 0]
    return o, rp, gate


def ref_block_norm_rest(d, v, eps, alpha, of, gate, rp, n_tasks):
    q = {k: (t.double().cpu() if t is not None else None) for k, t in v.items()}
    o, rp = {}, rp.double().cpu()
    g = q["dr_out"] if q["dr_out"] is not None else torch.zeros_like(rp)
    if q["w_pre"] is not None:
        m = 1 / torch.sqrt((rp ** 2).mean(dim=1, keepdim=True) + eps)
        rh = rp * m
        o["x"], o["rstd_pre"] = q["w_pre"] * rh, m[:, 0]
        if q["dx"] is not None:
            u = q["w_pre"] * q["dx"]
            g = g + m * (u - rh * (u * rh).mean(dim=1, keepdim=True))
            o["dw_pre"] = (q["dx"] * rh).sum(dim=0)
    o["dr"] = g
    if q["b"] is not None:
        n = 1 / torch.sqrt((q["b"] ** 2).mean(dim=1, keepdim=True) + eps) if q["w_post"] is not None else 1.0
        bh = q["b"] * n
        wp = q["w_post"] if q["w_post"] is not None else torch.ones(d, dtype=torch.float64)
        o["dgate"] = torch.stack([(alpha * wp * (g * bh)[of == t]).sum(dim=0) for t in range(n_tasks)])
        e = alpha * gate * g
        if q["w_post"] is not None:
            o["dw_post"] = (e * bh).sum(dim=0)
            e = e * wp
            e = n * (e - bh * (e * bh).mean(dim=1, keepdim=True))
        o["db"] = e
    return o


NORM_FORMS = {"all": "b w_post gate w_pre dr_out dx", "no_gate": "b w_post w_pre dr_out dx", "no_post": "b gate w_pre dr_out dx",
              "plain": "b w_pre dr_out dx", "first": "w_pre dr_out dx", "last": "b w_post gate dr_out", "no_dr": "b w_post gate w_pre dx"}


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,T,d,batch,form", [
    ("bf16", 1, 8, "one", "all"), ("bf16", 40, 4096, "tokens", "all"), ("bf16", 300, 512, "mixed", "all"), ("bf16", 333, 1024, "mixed", "no_gate"),
    ("bf16", 77, 2048, "bare", "all"), ("bf16", 200, 1032, "mixed", "no_post"), ("bf16", 65, 8192, "mixed", "all"), ("bf16", 19, 16384, "mixed", "all"),
    ("bf16", 130, 3000, "mixed", "plain"), ("bf16", 130, 520, "mixed", "first"), ("bf16", 130, 640, "mixed", "last"), ("bf16", 64, 64, "mixed", "no_dr"),
    ("bf16", 5000, 256, "mixed", "all"), ("f32", 100, 1, "mixed", "all"), ("f32", 90, 257, "mixed", "all"), ("f32", 50, 1025, "mixed", "all"),
    ("f32", 33, 2051, "mixed", "no_gate"), ("f32", 9, 9001, "tokens", "all"), ("f32", 70, 256, "mixed", "all"), ("f32", 70, 1024, "mixed", "plain"),
    ("f32", 40, 4096, "mixed", "all"), ("f32", 40, 6000, "mixed", "no_post"), ("f32", 12, 16384, "mixed", "all"), ("f32", 45, 1540, "mixed", "last"),
    ("f32", 45, 300, "mixed", "no_dr"), ("f32", 45, 300, "mixed", "first"),
])
def test_block_norm(dtype, T, d, batch, form):
    n, eps, alpha = 3, 1e-5, 0.7
    off, task = batch_of(batch, T, n)
    of = torch.from_numpy(np.repeat(np.asarray(task), np.diff(np.asarray(off))))
    g = torch.Generator().manual_seed(T * d)
    has = NORM_FORMS[form].split()
    mk = lambda *s: torch.randn(*s, generator=g).to(DT[dtype])
    v = dict(r=mk(T, d) * 2, b=mk(T, d) if "b" in has else None, w_post=mk(d) if "w_post" in has else None, gate=mk(n, d) if "gate" in has else None,
             w_pre=mk(d) if "w_pre" in has else None, dr_out=mk(T, d) if "dr_out" in has else None, dx=mk(T, d) if "dx" in has else None)
    if T > 2 and v["b"] is not None:
        v["b"][1] = 0                         # a row that the norm has nothing of
    dv = {k: (t.to(DEV) if t is not None else None) for k, t in v.items()}
    plan = bd.Plan(dtype, T, d, max(d // 8 * 8, 8), [0, 4, 8, 12], off, task)
    cfg = bd.BlockNormConfig(eps, alpha)
    G = {}
    new = lambda k, *s, dt=torch.float32: G.setdefault(k, guarded(*s, dtype=dt))[0]
    post, pre = v["w_post"] is not None, v["w_pre"] is not None
    r_out = new("r_out", T, d, dt=DT[dtype]) if v["b"] is not None else None
    x = new("x", T, d, dt=DT[dtype]) if pre else None
    rp_, rr_ = new("rstd_post", T) if post else None, new("rstd_pre", T) if pre else None
    bd.lobra_mlora_block_norm_fwd(plan, cfg, dv["r"], dv["b"], dv["w_post"], dv["gate"], dv["w_pre"], r_out, x, rp_, rr_)
    torch.cuda.synchronize()
    ref, _, gate = ref_block_norm(d, v, eps, alpha, of)
    if v["b"] is not None:
        near(r_out, ref["r_out"], dtype, "r_out")
        if post:
            near(rp_, ref["rstd_post"], "f32", "rstd_post")
    kept = r_out if r_out is not None else dv["r"]
    rest = ref_block_norm_rest(d, v, eps, alpha, of, gate, kept, n)
    if pre:
        near(x, rest["x"], dtype, "x")
        near(rr_, rest["rstd_pre"], "f32", "rstd_pre")
    # backward: separate outputs, then in place with sums that are added to
    want = [k for k in ("dgate", "dw_post", "dw_pre") if k in rest and (k != "dgate" or v["gate"] is not None)]
    shapes = dict(dgate=(n, d), dw_post=(d,), dw_pre=(d,))
    ws, ws_ok = guarded(bd.lobra_mlora_block_norm_workspace_bytes(plan), dtype=torch.uint8)
    grads = {k: new(k, *shapes[k]) for k in want}
    dr, db = new("dr", T, d, dt=DT[dtype]), new("db", T, d, dt=DT[dtype]) if v["b"] is not None else None
    args = (plan, cfg, kept, dv["b"], dv["w_post"], dv["gate"], dv["w_pre"], rp_, rr_, dv["dr_out"], dv["dx"])
    bd.lobra_mlora_block_norm_bwd(*args, dr, db, grads.get("dgate"), grads.get("dw_post"), grads.get("dw_pre"), ws=ws)
    torch.cuda.synchronize()
    assert ws_ok() and all(ok() for _, ok in G.values())
    near(dr, rest["dr"], dtype, "dr", fp32=4e-6)
    if db is not None:
        near(db, rest["db"], dtype, "db", fp32=8e-6)      # (a difference of terms of its size, with fp32's 1 / rms of either)
    for k in want:
        near(grads[k], rest[k], "f32", k, fp32=1e-5, scale=max(float(rest[k].abs().max()), 1e-3))
    first = {k: t.clone() for k, t in grads.items()}
    dr1, db1 = dr.clone(), None if db is None else db.clone()
    # the gradient of the residual over dr_out and of the block over dx: the same bits, and the sums twice
    dro, dxo = dv["dr_out"], dv["dx"]
    bd.lobra_mlora_block_norm_bwd(*args, dro if dro is not None else dr, dxo if dxo is not None and db is not None else db,
                                  grads.get("dgate"), grads.get("dw_post"), grads.get("dw_pre"), flags=bd.FLAG_ACCUMULATE_GRADS, ws=ws)
    torch.cuda.synchronize()
    assert torch.equal(dro if dro is not None else dr, dr1)
    if db is not None:
        assert torch.equal(dxo if dxo is not None else db, db1)
    for k in want:
        assert torch.equal(grads[k], first[k] + first[k]), k
    # frozen gains and gates: the activations' gradients alone, without a workspace
    dv["dr_out"], dv["dx"] = (t.to(DEV) if t is not None else None for t in (v["dr_out"], v["dx"]))
    args = args[:9] + (dv["dr_out"], dv["dx"])
    bd.lobra_mlora_block_norm_bwd(*args, dr, db)
    torch.cuda.synchronize()
    assert torch.equal(dr, dr1) and (db is None or torch.equal(db, db1))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,T,d,batch,form", [
    ("bf16", 120, 2560, "mixed", "all"), ("bf16", 75, 4608, "mixed", "plain"), ("bf16", 75, 5120, "mixed", "all"), ("bf16", 40, 6144, "tokens", "all"),
    ("bf16", 33, 6152, "mixed", "no_gate"), ("bf16", 20, 12288, "mixed", "all"), ("f32", 30, 2560, "mixed", "plain"), ("f32", 30, 5121, "mixed", "all"),
    ("f32", 15, 12289, "mixed", "no_dr"),
])
def test_block_norm_between_the_widths_of_whole_teams(dtype, T, d, batch, form):
    """Rows that leave lanes or whole waves of their team without a packet."""
    test_block_norm(dtype, T, d, batch, form)


@pytest.mark.gpu
def test_block_norm_gradient_against_differences():
    T, d, n, eps = 20, 96, 2, 1e-2
    g = torch.Generator(device=DEV).manual_seed(3)
    mk = lambda *s: torch.randn(*s, device=DEV, generator=g)
    off, task = [0, 7, 12, 20], [1, -1, 0]
    plan, cfg = bd.Plan("f32", T, d, d, [0, 4, 8], off, task), bd.BlockNormConfig(1e-5, 0.6)
    v = dict(r=mk(T, d), b=mk(T, d), w_post=mk(d), gate=mk(n, d), w_pre=mk(d))
    cr, cx = mk(T, d), mk(T, d)               # the loss is linear in r' and x

    def forward(v):
        r_out, x, rp, rr = torch.empty(T, d, device=DEV), torch.empty(T, d, device=DEV), torch.empty(T, device=DEV), torch.empty(T, device=DEV)
        bd.lobra_mlora_block_norm_fwd(plan, cfg, v["r"], v["b"], v["w_post"], v["gate"], v["w_pre"], r_out, x, rp, rr)
        return r_out, x, rp, rr

    r_out, x, rp, rr = forward(v)
    gr = dict(r=torch.empty(T, d, device=DEV), b=torch.empty(T, d, device=DEV), gate=torch.empty(n, d, device=DEV), w_post=torch.empty(d, device=DEV),
              w_pre=torch.empty(d, device=DEV))
    ws = torch.empty(bd.lobra_mlora_block_norm_workspace_bytes(plan), dtype=torch.uint8, device=DEV)
    bd.lobra_mlora_block_norm_bwd(plan, cfg, r_out, v["b"], v["w_post"], v["gate"], v["w_pre"], rp, rr, cr, cx, gr["r"], gr["b"], gr["gate"],
                                  gr["w_post"], gr["w_pre"], ws=ws)
    for k in v:
        dirn = mk(*v[k].shape)

        def loss(e):
            r_out, x, _, _ = forward({**v, k: v[k] + e * dirn})
            return float((cr.double() * r_out.double() + cx.double() * x.double()).sum())

        got = (8 * (loss(eps) - loss(-eps)) - (loss(2 * eps) - loss(-2 * eps))) / (12 * eps)
        slope = float((gr[k].double() * dirn.double()).sum())
        # values of some 4e3 terms of size one, each off by 1e-7, over eps; slopes of some tens
        assert abs(got - slope) <= 2e-3 * max(10.0, abs(slope)), (k, got, slope)


@pytest.mark.gpu
def test_block_norm_refusals():
    T, d = 16, 64
    plan, cfg = bd.Plan("bf16", T, d, 64, [0, 8], [0, T], [0]), bd.BlockNormConfig(1e-5, 1.0)
    t = lambda *s: torch.zeros(*s, dtype=torch.bfloat16, device=DEV)
    r, b, w, gt, st = t(T, d), t(T, d), t(d), t(1, d), torch.ones(T, device=DEV)
    fwd = lambda plan=plan, cfg=cfg, r=r, b=b, r_out=b.clone(), x=b.clone(): bd.lobra_mlora_block_norm_fwd(plan, cfg, r, b, w, gt, w, r_out, x, st, st.clone(), check=False)
    assert fwd() == bd.OK
    assert fwd(r=None) == -1 and fwd(r_out=None) == -1 and fwd(x=None) == -1
    assert fwd(r=t(T * d + 8)[4:4 + T * d]) == -8
    for bad in (bd.BlockNormConfig(-1.0, 1.0), bd.BlockNormConfig(math.nan, 1.0), bd.BlockNormConfig(math.inf, 1.0), bd.BlockNormConfig(0.0, math.nan)):
        assert fwd(cfg=bad) == -2
    assert fwd(plan=bd.Plan("bf16", T, d, 64, [0, 8], [0, T], [0], bd.PLAN_HOST_ONLY)) == -10
    wide = bd.Plan("bf16", 1, 16392, 64, [0, 8], [0, 1], [0])
    assert fwd(plan=wide) == -2
    with pytest.raises(bd.LobraError):
        bd.lobra_mlora_block_norm_workspace_bytes(wide)
    gr, ws = torch.zeros(1, d, device=DEV), torch.empty(bd.lobra_mlora_block_norm_workspace_bytes(plan), dtype=torch.uint8, device=DEV)

    def bwd(**kw):
        a = dict(r_out=r, b=b, w_post=w, gate=gt, w_pre=w, rstd_post=st, rstd_pre=st, dr_out=r, dx=b, dr=r.clone(), db=b.clone(), dgate=gr, dw_post=None,
                 dw_pre=None, ws=ws)
        a.update(kw)
        return bd.lobra_mlora_block_norm_bwd(plan, cfg, *[a[k] for k in ("r_out", "b", "w_post", "gate", "w_pre", "rstd_post", "rstd_pre", "dr_out", "dx",
                                                                         "dr", "db", "dgate", "dw_post", "dw_pre")], 0, a["ws"], check=False)

    assert bwd() == bd.OK
    for bad in (dict(dr=None), dict(db=None), dict(rstd_pre=None), dict(rstd_post=None), dict(r_out=None), dict(gate=None), dict(b=None),
                dict(w_post=None, dw_post=gr), dict(dx=None, dw_pre=gr)):
        assert bwd(**bad) == -1, bad
    assert bwd(ws=None) == -7 and bwd(ws=ws[:ws.numel() - 1]) == -7


@pytest.mark.gpu
def test_block_norm_of_no_tokens():
    plan, cfg = bd.Plan("f32", 0, 32, 32, [0, 8], [0], []), bd.BlockNormConfig(1e-5, 1.0)
    e = torch.empty(0, 32, device=DEV)
    w, gt = torch.ones(32, device=DEV), torch.ones(1, 32, device=DEV)
    dg, dp, dq = (torch.full(s, 5.0, device=DEV) for s in ((1, 32), (32,), (32,)))
    ws = torch.empty(max(bd.lobra_mlora_block_norm_workspace_bytes(plan), 16), dtype=torch.uint8, device=DEV)
    some = torch.zeros(4, 32, device=DEV)
    bd.lobra_mlora_block_norm_fwd(plan, cfg, some, some, w, gt, w, some.clone(), some.clone())
    bd.lobra_mlora_block_norm_bwd(plan, cfg, some, some, w, gt, w, None, None, None, some, some.clone(), some.clone(), dg, dp, dq, ws=ws)
    torch.cuda.synchronize()
    assert not bool(dg.any()) and not bool(dp.any()) and not bool(dq.any())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("accumulate", [False, True])
def test_block_norm_of_an_empty_batch(dtype, accumulate):
    """A chunk without tokens, its tensors those of no rows (which have no address) and no byte of workspace: gradients of 0, or as they were."""
    n, d = 3, 72
    plan, cfg = bd.Plan(dtype, 0, d, 64, [0, 4, 8, 12], [0, 0, 0], [2, -1]), bd.BlockNormConfig(1e-5, 0.5)
    e, st = torch.empty(0, d, dtype=DT[dtype], device=DEV), torch.empty(0, device=DEV)
    assert e.data_ptr() == 0
    w, gate = torch.ones(d, dtype=DT[dtype], device=DEV), torch.ones(n, d, dtype=DT[dtype], device=DEV)
    ws = torch.empty(bd.lobra_mlora_block_norm_workspace_bytes(plan), dtype=torch.uint8, device=DEV)
    bd.lobra_mlora_block_norm_fwd(plan, cfg, e, e, w, gate, w, e, e, st, st)
    for want in ("dgate dw_post dw_pre", "dgate", "dw_post", "dw_pre", ""):
        G = {k: guarded(*s, dtype=torch.float32) for k, s in (("dgate", (n, d)), ("dw_post", (d,)), ("dw_pre", (d,))) if k in want.split()}
        for t, _ in G.values():
            t.fill_(5.0)
        for scratch in (ws, None):
            bd.lobra_mlora_block_norm_bwd(plan, cfg, e, e, w, gate, w, st, st, e, e, e, e, *[G[k][0] if k in G else None for k in ("dgate", "dw_post", "dw_pre")],
                                          flags=bd.FLAG_ACCUMULATE_GRADS if accumulate else 0, ws=scratch)
        torch.cuda.synchronize()
        for k, (t, ok) in G.items():
            assert ok() and bool((t == (5.0 if accumulate else 0.0)).all()), k
    # what a gradient needs apart from the batch is still asked for
    back = lambda *frozen, **kw: bd.lobra_mlora_block_norm_bwd(plan, cfg, e, e, *frozen, st, st, e, e, e, e, **kw, ws=ws, check=False)
    g1 = torch.zeros(n, d, device=DEV)
    assert back(w, None, w, dgate=g1) == -1 and back(None, gate, w, dw_post=g1) == -1 and back(w, gate, None, dw_pre=g1) == -1


# ------------------------------------------------------------------------------------------------------------------
# gated feed-forward block
# ------------------------------------------------------------------------------------------------------------------
def act64(code, g):
    if code == bd.ACT_SILU:
        q = torch.sigmoid(g)
        return g * q, q * (1 + g * (1 - q))
    c = math.sqrt(2 / math.pi)
    t = torch.tanh(c * (g + 0.044715 * g ** 3))
    return 0.5 * g * (1 + t), 0.5 * (1 + t) + 0.5 * g * (1 - t ** 2) * c * (1 + 3 * 0.044715 * g ** 2)


def gated_inputs(dtype, T, d, f, ranks, seed):
    g = torch.Generator().manual_seed(seed)
    mk = lambda std, *s: (torch.randn(*s, generator=g) * std).to(DT[dtype])
    R = 2 * sum(ranks)
    return dict(x=mk(1.0, T, d), W=mk(1 / math.sqrt(d), d, 2 * f), A=mk(1 / math.sqrt(d), R, d), B=mk(0.3, R, f),
                s=torch.rand(len(ranks), generator=g) + 0.5, dh=mk(1.0, T, f))


def ref_gated_projections(v, f, ranks, of):
    x, W, A, B = (v[k].double() for k in ("x", "W", "A", "B"))
    y, row = x @ W, 0
    for t, r in enumerate(ranks):
        idx = (of == t).nonzero().flatten()
        for j in (0, 1):
            w = slice(row + j * r, row + (j + 1) * r)
            y[idx, j * f:(j + 1) * f] += float(v["s"][t]) * (x[idx] @ A[w].T) @ B[w]
        row += 2 * r
    return y


def ref_gated_back(v, f, ranks, of, dy):
    x, W, A, B = (v[k].double() for k in ("x", "W", "A", "B"))
    dx, dA, dB, row = dy @ W.T, torch.zeros_like(A), torch.zeros_like(B), 0
    for t, r in enumerate(ranks):
        idx, s = (of == t).nonzero().flatten(), float(v["s"][t])
        for j in (0, 1):
            w, part = slice(row + j * r, row + (j + 1) * r), dy[idx, j * f:(j + 1) * f]
            dx[idx] += s * (part @ B[w].T) @ A[w]
            dA[w], dB[w] = s * (part @ B[w].T).T @ x[idx], s * (x[idx] @ A[w].T).T @ part
        row += 2 * r
    return dx, dA, dB


GATED = [
    # dtype, T, d, f, ranks, batch, activation
    ("f32", 1, 33, 8, [8], "one", 0), ("f32", 150, 100, 72, [8, 16], "mixed", 1), ("f32", 700, 96, 200, [8, 8, 8], "mixed", 0),
    ("bf16", 16, 264, 72, [8, 8], "tokens", 0), ("bf16", 17, 1000, 8, [24], "tokens", 1), ("bf16", 33, 8, 136, [8], "mixed", 0),
    ("bf16", 64, 4096, 64, [16, 64, 8], "tokens", 1), ("bf16", 64, 136, 8200, [8], "bare", 0), ("bf16", 5, 2056, 520, [64, 8], "tokens", 0),
    ("bf16", 65, 512, 192, [16], "mixed", 0),
    ("bf16", 1, 64, 64, [8], "one", 0), ("bf16", 40, 512, 1376, [16, 8], "tokens", 1), ("bf16", 300, 256, 128, [16], "mixed", 0),
    ("bf16", 300, 264, 136, [8, 16], "mixed", 1), ("bf16", 600, 1024, 640, [16, 32, 8], "mixed", 0), ("bf16", 300, 256, 512, [8], "bare", 0),
    ("bf16", 2100, 512, 1160, [64, 8], "mixed", 0), ("bf16", 4500, 256, 1024, [8, 24, 16], "mixed", 1), ("bf16", 3000, 640, 2048, [40], "one", 0),
    ("bf16", 2049, 1024, 4096, [16] * 5, "mixed", 1),
    ("bf16", 16000, 128, 128, [8, 16], "mixed", 0), ("bf16", 9000, 256, 264, [64, 8, 24], "mixed", 0), ("bf16", 5000, 256, 1160, [8], "bare", 1),
    ("bf16", 6000, 128, 1000, [16] * 9, "tokens", 0),
]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,T,d,f,ranks,batch,act", GATED)
def test_gated(dtype, T, d, f, ranks, batch, act):
    n = len(ranks)
    off, task = batch_of(batch, T, n)
    of = torch.from_numpy(np.repeat(np.asarray(task), np.diff(np.asarray(off))))
    v = gated_inputs(dtype, T, d, f, ranks, T + d + f)
    plan = bd.Plan(dtype, T, d, 2 * f, np.concatenate([[0], np.cumsum([2 * r for r in ranks])]), off, task, n_proj=2)
    y = ref_gated_projections(v, f, ranks, of)
    a, _ = act64(act, y[:, :f])
    h_ref = a * y[:, f:]
    # storage bf16: the projected activations are rounded to bf16 between the adapter's factors (2^-9 of the adapter term, which is of the
    # size of y here), and h may start from the rounded projections: 2^-7 of h's largest in all.  fp32: sums of up to d products
    tol = dict(f32=4e-6, bf16=2.0 ** -7)[dtype]
    dv = {k: t.to(DEV) for k, t in v.items()}
    w = [dv[k] for k in ("x", "W", "A", "B", "s")]
    edt = DT[dtype]
    for save in (False, True):
        h, h_ok = guarded(T, f, dtype=edt)
        gu, gu_ok = guarded(T, 2 * f, dtype=edt)
        hs, hs_ok = guarded(max(plan.h_save_bytes, 16), dtype=torch.uint8)
        ws, ws_ok = guarded(max(bd.lobra_mlora_gated_workspace_bytes(plan, save), 16), dtype=torch.uint8)
        bd.lobra_mlora_gated_fwd(plan, act, *w, gu if save else None, h, hs if save else None, ws)
        torch.cuda.synchronize()
        assert h_ok() and gu_ok() and hs_ok() and ws_ok()
        off_h = float((h.double().cpu() - h_ref).abs().max() / h_ref.abs().max())
        assert off_h <= tol, (save, off_h)
    off_y = float((gu.double().cpu() - y).abs().max() / y.abs().max())
    assert off_y <= tol, off_y
    # backward from the projections as they were kept
    gk = gu.double().cpu()
    a, da = act64(act, gk[:, :f])
    dh = v["dh"].double()
    dy = torch.cat([dh * gk[:, f:] * da, dh * a], dim=1)
    wsb, wsb_ok = guarded(max(plan.bwd_ws_bytes, 16), dtype=torch.uint8)
    dgu, dgu_ok = guarded(T, 2 * f, dtype=edt)
    dx, dx_ok = guarded(T, d, dtype=edt)
    dA, dA_ok = guarded(2 * sum(ranks), d, dtype=torch.float32)
    dB, dB_ok = guarded(2 * sum(ranks), f, dtype=torch.float32)
    bd.lobra_mlora_gated_bwd(plan, act, *w, gu, dv["dh"], hs, dgu, dx, dA, dB, 0, wsb)
    torch.cuda.synchronize()
    assert wsb_ok() and dgu_ok() and dx_ok() and dA_ok() and dB_ok()
    near(dgu, dy, dtype, "dgu", fp32=4e-6)
    dx_ref, dA_ref, dB_ref = ref_gated_back(v, f, ranks, of, dgu.double().cpu())
    for got, ref, name in ((dx, dx_ref, "dx"), (dA, dA_ref, "dA"), (dB, dB_ref, "dB")):
        top = float(ref.abs().max())
        if top == 0:
            assert not bool(got.any()), name
            continue
        assert float((got.double().cpu() - ref).abs().max()) / top <= (1e-5 if dtype == "f32" else 2e-2), name
    # in place of the projections: the same bits
    keep = dgu.clone()
    bd.lobra_mlora_gated_bwd(plan, act, *w, gu, dv["dh"], hs, gu, dx, dA, dB, bd.FLAG_NO_DX, wsb)
    torch.cuda.synchronize()
    assert torch.equal(gu, keep)


@pytest.mark.gpu
@pytest.mark.parametrize("T", [40, 200, 4500])
def test_gated_adapter_of_no_finite_value_stays_with_its_task(T):
    """Tasks side by side in a tile: NaN and inf in one's adapters (both projections) reach its own tokens alone - and, as in the layer's own
    products, whose matrix instructions take 16 rows at a time, at most rows that share a block of 16 with those.  The few-token kernels share
    nothing."""
    d, f, ranks = 256, 1024, [8, 16, 24]
    off, task = batch_of("mixed", T, 3)
    of = torch.from_numpy(np.repeat(np.asarray(task), np.diff(np.asarray(off))))
    v = gated_inputs("bf16", T, d, f, ranks, T)
    for row in (16, 20, 31, 32, 47):                  # task 1: stacked rows 16 .. 47, gate's then up's
        v["B"][row, ::3] = math.nan
        v["A"][row, ::5] = math.inf
    plan = bd.Plan("bf16", T, d, 2 * f, [0, 16, 48, 96], off, task, n_proj=2)
    y = ref_gated_projections({**v, "A": torch.nan_to_num(v["A"], posinf=0.0), "B": torch.nan_to_num(v["B"])}, f, ranks, of)
    h_ref = act64(0, y[:, :f])[0] * y[:, f:]
    w = [v[k].to(DEV) for k in ("x", "W", "A", "B", "s")]
    gu, h = torch.empty(T, 2 * f, dtype=torch.bfloat16, device=DEV), torch.empty(T, f, dtype=torch.bfloat16, device=DEV)
    ws = torch.empty(bd.lobra_mlora_gated_workspace_bytes(plan, True), dtype=torch.uint8, device=DEV)
    bd.lobra_mlora_gated_fwd(plan, 0, *w, gu, h, None, ws)
    torch.cuda.synchronize()
    others = of != 1
    got = h.double().cpu()
    assert bool(torch.isnan(got[of == 1]).any())
    if T > 64:
        blocks = torch.zeros((T + 31) // 16 * 16, dtype=torch.bool)
        blocks[:T] = of == 1
        # (the last row of tiles may begin anywhere: blocks of 16 from any row)
        others &= torch.tensor([not bool(blocks[max(0, i - 15):i + 16].any()) for i in range(T)])
        assert int(others.sum()) > 20
    assert bool(torch.isfinite(got[others]).all())
    assert float((got - h_ref)[others].abs().max() / h_ref[others].abs().max()) <= 2.0 ** -7


@pytest.mark.gpu
@pytest.mark.parametrize("act", [bd.ACT_SILU, bd.ACT_GELU_TANH])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gated_activation_at_the_ends(act, dtype):
    """Values at which exp overflows, squares overflow, and zeros; W is a choice of columns, so that g and u are the inputs themselves."""
    vals = [0.0, -0.0, 1e-30, 1.0, -1.0, 12.0, -12.0, 90.0, -90.0, 1e4, -1e4, 1e20, -1e20, 1e25, -1e25, 3e38, -3e38]
    T, d, f = len(vals), 16, 8
    x = torch.zeros(T, d)
    x[:, 0], x[:, 1] = torch.tensor(vals), 0.5
    W = torch.zeros(d, 2 * f)
    W[0, :f], W[1, f:] = 1.0, 1.0
    x, W = x.to(DT[dtype]).to(DEV), W.to(DT[dtype]).to(DEV)
    plan = bd.Plan(dtype, T, d, 2 * f, None, [0, T], [-1], n_proj=2)
    gu, h, dgu = (torch.empty(T, c, dtype=DT[dtype], device=DEV) for c in (2 * f, f, 2 * f))
    dh, dx = torch.ones(T, f, dtype=DT[dtype], device=DEV), torch.empty(T, d, dtype=DT[dtype], device=DEV)
    ws = torch.empty(max(bd.lobra_mlora_gated_workspace_bytes(plan, True), plan.bwd_ws_bytes, 16), dtype=torch.uint8, device=DEV)
    bd.lobra_mlora_gated_fwd(plan, act, x, W, None, None, None, gu, h, None, ws)
    bd.lobra_mlora_gated_bwd(plan, act, x, W, None, None, None, gu, dh, None, dgu, dx, None, None, 0, ws)
    torch.cuda.synchronize()
    g = gu[:, 0].double().cpu()
    assert torch.equal(g, x[:, 0].double().cpu())
    a, da = act64(act, g.clamp(-1e6, 1e6))            # (beyond: a = g or 0, a' = 1 or 0)
    a = torch.where(g.abs() > 1e6, torch.where(g > 0, g, torch.zeros_like(g)), a)
    rel = 2.0 ** -8 if dtype == "bf16" else 2e-6
    for got, ref in ((h[:, 3], a * 0.5), (dgu[:, 2], 0.5 * da), (dgu[:, f + 1], a)):
        got = got.double().cpu()
        assert bool(torch.isfinite(got).all()) and bool(((got - ref).abs() <= rel * ref.abs() + 1e-30 * (dtype == "f32") + 1e-30).all()), (got, ref)


@pytest.mark.gpu
def test_gated_refusals():
    T, d, f = 64, 64, 64
    p2 = bd.Plan("bf16", T, d, 2 * f, [0, 16], [0, T], [0], n_proj=2)
    p1 = bd.Plan("bf16", T, d, 2 * f, [0, 16], [0, T], [0])
    v = gated_inputs("bf16", T, d, f, [8], 1)
    w = [v[k].to(DEV) for k in ("x", "W", "A", "B", "s")]
    t = lambda *s: torch.zeros(*s, dtype=torch.bfloat16, device=DEV)
    ws = torch.empty(bd.lobra_mlora_gated_workspace_bytes(p2, False), dtype=torch.uint8, device=DEV)
    fwd = lambda plan=p2, act=0, x=w[0], gu=None, h=t(T, f), ws=ws: bd.lobra_mlora_gated_fwd(plan, act, x, *w[1:], gu, h, None, ws, check=False)
    assert fwd() == bd.OK
    assert fwd(plan=p1) == -2 and fwd(act=2) == -2 and fwd(act=-1) == -2
    assert fwd(h=None) == -1 and fwd(x=None) == -1
    assert fwd(ws=None) == -7 and fwd(ws=ws[:T * 2 * f * 2]) == -7 and fwd(ws=ws[:100]) == -7
    assert fwd(h=t(T * f + 8)[1:1 + T * f]) == -8
    with pytest.raises(bd.LobraError):
        bd.lobra_mlora_gated_workspace_bytes(p1, True)
    wsb = torch.empty(max(p2.bwd_ws_bytes, 16), dtype=torch.uint8, device=DEV)
    dA, dB = torch.zeros(16, d, device=DEV), torch.zeros(16, f, device=DEV)
    dgu = torch.full((T, 2 * f), 3.0, dtype=torch.bfloat16, device=DEV)

    def bwd(plan=p2, act=0, gu=t(T, 2 * f), dh=t(T, f), out=dgu, dx=t(T, d), ws=wsb):
        return bd.lobra_mlora_gated_bwd(plan, act, *w, gu, dh, None, out, dx, dA, dB, 0, ws, check=False)

    for bad, st in ((dict(gu=None), -1), (dict(dh=None), -1), (dict(out=None), -1), (dict(dx=None), -1), (dict(act=9), -2), (dict(plan=p1), -2),
                    (dict(ws=None), -7)):
        assert bwd(**bad) == st, bad
    torch.cuda.synchronize()
    assert bool((dgu == 3.0).all())                   # nothing was launched
    assert bwd() == bd.OK


@pytest.mark.gpu
@pytest.mark.parametrize("act", [bd.ACT_SILU, bd.ACT_GELU_TANH])
@pytest.mark.parametrize("T,d,f,keep", [(1, 512, 72, False), (40, 512, 1376, True), (128, 1000, 264, False), (192, 4096, 1376, False), (192, 4096, 1376, True),
                                        (2100, 512, 1160, False), (4500, 256, 1024, True)])
def test_gated_output_starts_from_unrounded_projections(T, d, f, keep, act):
    """bf16, no adapters: one rounding of h (2^-8 of it at most) next to fp32 sums, in the forms that have the projections in fp32.  From [g | u] as
    rounded it would be off by up to 2^-8 (1 + |g a' / a|) more, which the same bound does not hold."""
    v = gated_inputs("bf16", T, d, f, [8], T * f)
    plan = bd.Plan("bf16", T, d, 2 * f, None, [0, T], [-1], n_proj=2)
    y = v["x"].double() @ v["W"].double()
    h_of = lambda y: act64(act, y[:, :f])[0] * y[:, f:]
    ref = h_of(y)
    gu = torch.empty(T, 2 * f, dtype=torch.bfloat16, device=DEV) if keep else None
    h = torch.empty(T, f, dtype=torch.bfloat16, device=DEV)
    ws = torch.empty(max(bd.lobra_mlora_gated_workspace_bytes(plan, keep), 16), dtype=torch.uint8, device=DEV)
    bd.lobra_mlora_gated_fwd(plan, act, v["x"].to(DEV), v["W"].to(DEV), None, None, None, gu, h, None, ws)
    torch.cuda.synchronize()
    near(h, ref, "bf16", "h")
    if gu is not None:
        near(gu, y, "bf16", "gu")
    with pytest.raises(AssertionError):               # (the bound can tell)
        near(h_of(y.bfloat16().double()).bfloat16(), ref, "bf16", "h")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gated_block_and_loss_of_an_empty_batch(dtype):
    """Tensors of no rows, which have no address: the adapters' gradients are 0, or stay as they are where they are added to."""
    d, f, edt = 64, 72, DT[dtype]
    plan = bd.Plan(dtype, 0, d, 2 * f, [0, 16, 48], [0, 0], [1], n_proj=2)
    v = gated_inputs(dtype, 0, d, f, [8, 16], 1)
    w = [v[k].to(DEV) for k in ("x", "W", "A", "B", "s")]
    e = lambda c, dt=edt: torch.empty(0, c, dtype=dt, device=DEV)
    for save in (False, True):
        ws = torch.empty(bd.lobra_mlora_gated_workspace_bytes(plan, save), dtype=torch.uint8, device=DEV)
        bd.lobra_mlora_gated_fwd(plan, 0, *w, e(2 * f) if save else None, e(f), e(0, torch.uint8) if save else None, ws)
    for flags, want in ((0, 0.0), (bd.FLAG_ACCUMULATE_GRADS, 5.0), (bd.FLAG_NO_DX, 0.0)):
        (dA, okA), (dB, okB) = guarded(48, d, dtype=torch.float32), guarded(48, f, dtype=torch.float32)
        dA.fill_(5.0)
        dB.fill_(5.0)
        ws = torch.empty(plan.bwd_ws_bytes, dtype=torch.uint8, device=DEV)
        bd.lobra_mlora_gated_bwd(plan, 0, *w, e(2 * f), e(f), None, e(2 * f), e(d), dA, dB, flags, ws)
        torch.cuda.synchronize()
        assert okA() and okB() and bool((dA == want).all()) and bool((dB == want).all())
    desc, row, ids = bd.make_logprob_desc(dtype, 0, 100, top_k=3), torch.empty(0, device=DEV), torch.empty(0, dtype=torch.int32, device=DEV)
    bd.lobra_token_logprob_fwd(desc, e(100), ids, row, row, row, row, e(3, torch.float32), e(3, torch.int32))
    bd.lobra_token_logprob_bwd(desc, e(100), ids, row, row, row, row, row, e(100))
    torch.cuda.synchronize()


def _typed_calls():
    """name -> (call with keyword arguments in the place of its own, names of tensors of the plan's type, names of fp32 ones); plans of the
    host alone, which the library itself refuses."""
    T, d, f, n = 4, 16, 8, 2
    plan = lambda dt: bd.Plan(dt, T, d, 2 * f, [0, 16, 32], [0, 1, T], [0, 1], bd.PLAN_HOST_ONLY, n_proj=2)
    cfg = bd.BlockNormConfig(1e-5, 1.0)

    def calls(dt):
        e, g = (lambda *s: torch.zeros(*s, dtype=DT[dt])), torch.zeros
        p = plan(dt)
        norm = dict(r=e(T, d), b=e(T, d), w_post=e(d), gate=e(n, d), w_pre=e(d), r_out=e(T, d), x=e(T, d), rstd_post=g(T), rstd_pre=g(T))
        back = dict(r_out=e(T, d), b=e(T, d), w_post=e(d), gate=e(n, d), w_pre=e(d), rstd_post=g(T), rstd_pre=g(T), dr_out=e(T, d), dx=e(T, d),
                    dr=e(T, d), db=e(T, d), dgate=g(n, d), dw_post=g(d), dw_pre=g(d))
        layer = dict(x=e(T, d), W=e(d, 2 * f), A=e(32, d), B=e(32, f), s=g(n))
        gated = {**layer, "gu": e(T, 2 * f), "h": e(T, f)}
        gback = {**layer, "gu": e(T, 2 * f), "dh": e(T, f), "h_saved": None, "dgu": e(T, 2 * f), "dx": e(T, d), "dA": g(32, d), "dB": g(32, f)}
        return [(bd.lobra_mlora_block_norm_fwd, (p, cfg), norm, ("rstd_post", "rstd_pre")),
                (bd.lobra_mlora_block_norm_bwd, (p, cfg), back, ("rstd_post", "rstd_pre", "dgate", "dw_post", "dw_pre")),
                (bd.lobra_mlora_gated_fwd, (p, 0), gated, ("s",)), (bd.lobra_mlora_gated_bwd, (p, 0), gback, ("s", "dA", "dB"))]
    return calls


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("which", range(4), ids=["norm_fwd", "norm_bwd", "gated_fwd", "gated_bwd"])
def test_norms_and_gated_block_refuse_other_types(dtype, which):
    """The plan's element type and fp32 differ in their bytes: a gradient of a gain made like the gain, for one, is written to twice its length."""
    call, head, args, fp32 = _typed_calls()(dtype)[which]
    assert call(*head, **args, stream=0, check=False) == -10
    for name, t in args.items():
        if t is None:
            continue
        own = torch.float32 if name in fp32 else DT[dtype]
        for other in (torch.float32, torch.bfloat16, torch.float16, torch.float64):
            if other is not own:
                with pytest.raises(AssertionError):
                    call(*head, **{**args, name: t.to(other)}, stream=0, check=False)


@pytest.mark.gpu
def test_on_another_stream_and_in_a_graph():
    """The calls run on the stream that they are given, allocate nothing and can be captured; a replay sees new inputs."""
    T, V, d = 64, 5000, 512
    z, tgt = torch.randn(T, V, device=DEV), torch.randint(0, V, (T,), device=DEV).int()
    desc = bd.make_logprob_desc("f32", T, V)
    logp, lse, dz = torch.empty(T, device=DEV), torch.empty(T, device=DEV), torch.empty(T, V, device=DEV)
    w = torch.randn(T, device=DEV)
    grads = [torch.randn(8, 100, device=DEV), torch.randn(8, 64, device=DEV)]
    gset = bd.GradSet([(g, None, [0, 4, 8]) for g in grads], 2)
    ws, norm = torch.empty(gset.ws_bytes, dtype=torch.uint8, device=DEV), torch.empty(2, device=DEV)
    plan, cfg = bd.Plan("f32", T, d, d, [0, 4, 8], [0, 30, T], [0, 1]), bd.BlockNormConfig(1e-5, 1.0)
    r, b, wp, x, ro = torch.randn(T, d, device=DEV), torch.randn(T, d, device=DEV), torch.randn(d, device=DEV), torch.empty(T, d, device=DEV), torch.empty(T, d, device=DEV)

    def work():
        bd.lobra_token_logprob_fwd(desc, z, tgt, logp, lse)
        bd.lobra_token_logprob_bwd(desc, z, tgt, lse, None, None, w, None, dz)
        bd.lobra_grad_clip(gset, None, None, None, norm, None, None, ws=ws)
        bd.lobra_mlora_block_norm_fwd(plan, cfg, r, b, wp, None, wp, ro, x)

    outs = (logp, lse, dz, norm, ro, x)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        work()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        work()
    for k in range(3):
        z.mul_(0.9).add_(0.01 * k)
        b.mul_(1.1)
        grads[1].mul_(1.5)
        work()
        torch.cuda.synchronize()
        ref = [o.clone() for o in outs]
        for o in outs:
            o.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(o, q) for o, q in zip(outs, ref)), k


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,T,d,f,form", [("bf16", 40, 512, 264, "few tokens"), ("bf16", 192, 4096, 136, "split product"), ("bf16", 2304, 512, 1024, "persistent"),
                                              ("f32", 40, 260, 72, "few tokens"), ("f32", 300, 96, 200, "the layer's product")])
def test_passes_with_their_gradients_on_another_stream_and_in_a_graph(dtype, T, d, f, form):
    """Gated block and norms, both passes, and clipped gradients written: on a stream of their own, captured, and replayed on new inputs."""
    n, edt = 2, DT[dtype]
    g = torch.Generator(device=DEV).manual_seed(T)
    mk = lambda *s, std=1.0: (torch.randn(*s, device=DEV, generator=g) * std).to(edt)
    new = lambda *s, dt=edt: torch.empty(*s, dtype=dt, device=DEV)
    off, task = [0, T // 3, T - 5, T], [1, -1, 0]
    plan, cfg = bd.Plan(dtype, T, d, 2 * f, [0, 16, 48], off, task, n_proj=2), bd.BlockNormConfig(1e-5, 0.5)
    r, b, w_post, gate, w_pre, dh, dro = mk(T, d), mk(T, d), mk(d), mk(n, d), mk(d), mk(T, f), mk(T, d)
    W, A, B, s = mk(d, 2 * f, std=d ** -0.5), mk(48, d, std=d ** -0.5), mk(48, f, std=0.3), torch.ones(n, device=DEV)
    ro, x, h, h0, gu, dgu, dx, dr, db = new(T, d), new(T, d), new(T, f), new(T, f), new(T, 2 * f), new(T, 2 * f), new(T, d), new(T, d), new(T, d)
    f32 = torch.float32
    rp, rr, dA, dB, dgate, dwo, dwr = new(T, dt=f32), new(T, dt=f32), new(48, d, dt=f32), new(48, f, dt=f32), new(n, d, dt=f32), new(d, dt=f32), new(d, dt=f32)
    cA, cB, norm, scale, limit = new(48, d, dt=f32), new(48, f, dt=f32), new(n, dt=f32), new(n, dt=f32), torch.full((n,), 0.1, device=DEV)
    gset = bd.GradSet([(dA, cA, [0, 16, 48]), (dB, cB, [0, 16, 48]), (dgate, None, [0, 1, 2])], n)
    hs = new(max(plan.h_save_bytes, 16), dt=torch.uint8)
    ws = new(max(bd.lobra_mlora_gated_workspace_bytes(plan, True), bd.lobra_mlora_gated_workspace_bytes(plan, False), plan.bwd_ws_bytes,
                 bd.lobra_mlora_block_norm_workspace_bytes(plan), gset.ws_bytes), dt=torch.uint8)

    def work():
        bd.lobra_mlora_block_norm_fwd(plan, cfg, r, b, w_post, gate, w_pre, ro, x, rp, rr)
        bd.lobra_mlora_gated_fwd(plan, 0, x, W, A, B, s, None, h0, None, ws)
        bd.lobra_mlora_gated_fwd(plan, 0, x, W, A, B, s, gu, h, hs, ws)
        bd.lobra_mlora_gated_bwd(plan, 0, x, W, A, B, s, gu, dh, hs, dgu, dx, dA, dB, 0, ws)
        bd.lobra_mlora_block_norm_bwd(plan, cfg, ro, b, w_post, gate, w_pre, rp, rr, dro, dx, dr, db, dgate, dwo, dwr, 0, ws)
        bd.lobra_grad_clip(gset, limit, None, None, norm, scale, None, ws=ws)

    outs = (ro, x, rp, rr, h0, gu, h, dgu, dx, dA, dB, dr, db, dgate, dwo, dwr, norm, scale, cA, cB)
    work()
    torch.cuda.synchronize()
    ref = [o.clone() for o in outs]
    assert all(bool(torch.isfinite(o).all()) for o in ref)
    for o in outs:
        o.fill_(float("nan"))
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        work()
    side.synchronize()
    assert all(torch.equal(o, q) for o, q in zip(outs, ref))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        work()
    for k in range(3):
        b.mul_(1.25).add_(0.01 * k)
        dh.mul_(0.5)
        work()
        torch.cuda.synchronize()
        ref = [o.clone() for o in outs]
        for o in outs:
            o.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(o, q) for o, q in zip(outs, ref)), k
