"""Rows of logits beyond their own tokens: the loss against a teacher's likeliest tokens and its gradient, the selection of beam search, and the
reordering of what is kept per sequence.

Against plain implementations in 64 bits.  Tolerances: a loss comes from sums of exponentials in fp32, a few units in the last place of 1 (4e-6, and
2^-22 of what it is itself); a gradient is off by 2e-6 of the row's weight, and in bf16 by half a step, 2^-8 of its value.  A beam's score is rounded once to
fp32, from a sum in 64 bits whose lse has the losses' error.  Tokens, beams and moved bytes are compared as they are.
"""
import ctypes
import math

import numpy as np
import pytest

from paper_2509_01193_amd import binding as bd

torch = pytest.importorskip("torch")
from test_step_ops import DEV, DT, guarded, logits_of  # noqa: E402


# ------------------------------------------------------------------------------------------------------------------
# a teacher's likeliest tokens
# ------------------------------------------------------------------------------------------------------------------
def ref_distill(z, tl, ids, tail, temperature):
    """(loss [T], gradient of each row's loss [T, V], teacher [T]) in 64 bits, row by row."""
    T, V = z.shape
    loss, grad, taught = torch.zeros(T, dtype=torch.float64), torch.zeros(T, V, dtype=torch.float64), torch.zeros(T, dtype=torch.bool)
    for i in range(T):
        x = z[i].double() / temperature
        places = [(int(j), float(l)) for j, l in zip(ids[i], tl[i]) if 0 <= int(j) < V]
        if not places or (not tail and all(l == -math.inf for _, l in places)):
            continue
        taught[i] = True
        m = float(x.max())
        if bool(torch.isnan(x).any()) or m == math.inf or any(math.isnan(l) or l == math.inf for _, l in places):
            loss[i], grad[i] = math.nan, math.nan
            continue
        if m == -math.inf:
            loss[i] = math.inf                       # (and no gradient)
            continue
        e = (x - m).exp()
        S = e.sum()
        p = e / S
        if tail:
            qs = [math.exp(l) for _, l in places]
            ln_q = [l for _, l in places]
        else:
            top = max(l for _, l in places) / temperature
            own = sum(math.exp(l / temperature - top) for _, l in places)
            ln_q = [l / temperature - top - math.log(own) for _, l in places]
            qs = [math.exp(v) for v in ln_q]
        total, mass = 0.0, sum(qs)
        g = mass * p
        for (j, _), q, lq in zip(places, qs, ln_q):
            if q > 0:
                lp = float(x[j]) - m - float(S.log())
                total += q * (lq - lp)
            g[j] -= q
        qr = 1 - mass if tail else 0.0
        if qr > 2.0 ** -20:
            rest = x.clone()
            rest[[j for j, _ in places]] = -math.inf
            mr = float(rest.max())
            if mr == -math.inf:
                total = math.inf
                g += qr * p
            else:
                er = (rest - mr).exp()
                total += qr * (math.log(qr) - (mr - m + float(er.sum().log()) - float(S.log())))
                g += qr * (p - er / er.sum())
        loss[i], grad[i] = total, g / temperature
    return loss, grad, taught


def teacher_of(kind, z, k, tail, temperature, seed):
    """Log probabilities and ids [T, k] of another model's likeliest tokens, as `kind` has them."""
    T, V = z.shape
    g = torch.Generator().manual_seed(seed)
    t = torch.nan_to_num(z.float(), nan=0.0, posinf=5.0)
    t = torch.where(t < -1e30, torch.full_like(t, -30.0), t) + torch.randn(T, V, generator=g)
    kk = min(k, V)
    lp, ids = torch.log_softmax(t.double() / (temperature if tail else 1.0), dim=1).topk(kk, dim=1)
    lp = torch.nn.functional.pad(lp, (0, k - kk), value=-math.inf).float()
    ids = torch.nn.functional.pad(ids, (0, k - kk), value=-1).int()
    order = torch.randperm(k, generator=g)           # (no order is asked for)
    lp, ids = lp[:, order].contiguous(), ids[:, order].contiguous()
    if kind == "short" or kind == "odd":
        ids[torch.rand(T, k, generator=g) < 0.5] = -1
    if kind == "odd":
        ids[0] = -1                                  # a row without a teacher
        if T > 1:
            ids[1] = V + 3
        if T > 2:
            ids[2] = 0
            lp[2] = math.log(0.5 / k)                # one token in every place
        if T > 3:
            lp[3] = -math.inf
            ids[3] = torch.arange(k) % V
        if T > 4:
            lp[4, k // 2], ids[4, k // 2] = math.nan, 0
    return lp, ids


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("T,V,k,temperature,kind,teacher,pad", [
    (1, 1, 1, 1.0, "plain", "full", 0), (3, 7, 8, 2.0, "plain", "full", 0), (5, 64, 64, 1.0, "plain", "short", 0), (6, 1000, 128, 0.7, "plain", "odd", 5),
    (7, 4099, 20, 1.0, "offset", "odd", 0), (40, 32000, 8, 1.0, "plain", "full", 0), (9, 32000, 65, 2.0, "lowest", "odd", 8), (5, 5000, 20, 1.0, "masked", "full", 0),
    (6, 257, 32, 1.0, "equal", "odd", 1), (4, 20001, 100, 4.0, "sure", "full", 0), (4, 3000, 4, 1.0, "nan", "full", 0), (3, 300001, 40, 1.0, "plain", "odd", 0),
    (300, 9001, 3, 1.0, "plain", "odd", 0), (2, 131072, 128, 1.0, "one_stride", "full", 0),
])
def test_distill(dtype, tail, T, V, k, temperature, kind, teacher, pad):
    z = logits_of("plain" if kind == "sure" else kind, T, V, dtype, T + V + k)
    if kind == "sure":                               # the listed tokens have all of the student's probability but 1e-15
        z[:, :2] += 60
        z = z.to(DT[dtype])
    tl, ids = teacher_of(teacher, z, k, tail, temperature, V)
    if kind == "sure":
        ids[:, :2] = torch.tensor([0, 1], dtype=torch.int32)
        ids[:, 2:] = torch.where(ids[:, 2:] < 2, torch.full_like(ids[:, 2:], -1), ids[:, 2:])
        tl[:, :2] = math.log(0.1)
    loss, grad, taught = ref_distill(z, tl, ids, tail, temperature)
    w = torch.rand(T, generator=torch.Generator().manual_seed(T)) + 0.5
    if T > 5:
        w[5] = 0
    wide = torch.full((T, V + pad), 3.0, dtype=DT[dtype], device=DEV)
    wide[:, :V] = z.to(DEV)
    zd = wide[:, :V]
    desc = bd.make_distill_desc(dtype, T, V, k, tail=tail, temperature=temperature, ld=V + pad)
    ld, lok = guarded(T, dtype=torch.float32)
    st, sok = guarded(T, 4, dtype=torch.float32)
    t_args = tl.to(DEV), ids.to(DEV)
    bd.lobra_token_distill_fwd(desc, zd, *t_args, ld, st)
    torch.cuda.synchronize()
    assert lok() and sok()
    got = ld.double().cpu()
    # (a term takes the rounding of its logit's distance from the maximum: 2^-23 of it)
    far = torch.where(torch.isfinite(loss), loss.abs(), torch.zeros_like(loss))
    good = (got == loss) | (torch.isnan(got) & torch.isnan(loss)) | ((got - loss).abs() <= 4e-6 + 2.0 ** -22 * far)
    if kind == "lowest":                             # distances of 1e38: only relative
        good |= (got - loss).abs() <= 1e-6 * far
    assert bool(good.all()), [(i, float(got[i]), float(loss[i])) for i in (~good).nonzero().flatten().tolist()[:4]]
    only, ook = guarded(T, dtype=torch.float32)
    bd.lobra_token_distill_fwd(desc, zd, *t_args, only)
    assert torch.equal(torch.nan_to_num(only), torch.nan_to_num(ld)) and ook()
    want = grad * w.double()[:, None]
    want[w == 0] = 0
    scale = (w.double() / temperature)[:, None]

    def check(out, want, extra, what):
        out = out.double().cpu()
        bound = 2e-6 * scale + extra + (want.abs() * 2.0 ** -8 if dtype == "bf16" else 0)
        bad = ~(((out - want).abs() <= bound) | (torch.isnan(out) & torch.isnan(want)))
        assert not bool(bad.any()), (what, int(bad.sum()), bad.nonzero()[:3].tolist(), out[bad][:3].tolist(), want[bad][:3].tolist())

    base = torch.full((T, V + pad), 9.0, dtype=DT[dtype], device=DEV)
    dz = base[:, :V]
    wd = w.to(DEV)
    bd.lobra_token_distill_bwd(desc, zd, *t_args, st, wd, dz)
    torch.cuda.synchronize()
    check(dz, want, 0, "apart")
    assert bool((base[:, V:] == 9.0).all()) and bool((wide[:, V:] == 3.0).all())
    # added to another loss's gradient, in which rows without a weight stay as they are
    other = (torch.randn(T, V, generator=torch.Generator().manual_seed(7)) * 0.1).to(DT[dtype])
    base[:, :V] = other.to(DEV)
    bd.lobra_token_distill_bwd(desc, zd, *t_args, st, wd, dz, flags=bd.FLAG_ACCUMULATE_GRADS)
    check(dz, want + other.double(), 2.0 ** -23 * other.double().abs(), "added")
    # over the logits
    bd.lobra_token_distill_bwd(desc, zd, *t_args, st, wd, zd)
    torch.cuda.synchronize()
    check(zd, want, 0, "in place")
    assert bool((wide[:, V:] == 3.0).all())


@pytest.mark.gpu
def test_distill_of_the_own_tokens_is_none():
    """The student as its own teacher, through the log probabilities as they are written: no loss, no gradient."""
    T, V, k = 30, 5000, 20
    z = torch.randn(T, V, generator=torch.Generator().manual_seed(1)).to(DEV) * 4
    f = lambda *s, dt=torch.float32: torch.empty(*s, dtype=dt, device=DEV)
    tl, ti = f(T, k), f(T, k, dt=torch.int32)
    bd.lobra_token_logprob_fwd(bd.make_logprob_desc("f32", T, V, top_k=k), z, None, top_logp=tl, top_id=ti)
    desc = bd.make_distill_desc("f32", T, V, k, tail=True)
    loss, st, dz = f(T), f(T, 4), f(T, V)
    bd.lobra_token_distill_fwd(desc, z, tl, ti, loss, st)
    bd.lobra_token_distill_bwd(desc, z, tl, ti, st, torch.ones(T, device=DEV), dz)
    assert float(loss.abs().max()) < 4e-6 and float(dz.abs().max()) < 4e-6


@pytest.mark.gpu
@pytest.mark.parametrize("tail", [False, True])
def test_distill_gradient_against_differences(tail):
    T, V, k, t = 4, 50, 6, 1.5
    g = torch.Generator().manual_seed(4)
    z = torch.randn(T, V, generator=g).to(DEV)
    tl, ids = (x.to(DEV) for x in teacher_of("short", z.cpu(), k, tail, t, 3))
    desc = bd.make_distill_desc("f32", T, V, k, tail=tail, temperature=t)
    loss, st, dz = torch.empty(T, device=DEV), torch.empty(T, 4, device=DEV), torch.empty(T, V, device=DEV)
    w = (torch.rand(T, generator=g) + 0.5).to(DEV)
    bd.lobra_token_distill_fwd(desc, z, tl, ids, loss, st)
    bd.lobra_token_distill_bwd(desc, z, tl, ids, st, w, dz)

    def value(x):
        bd.lobra_token_distill_fwd(desc, x, tl, ids, loss)
        return float((loss.double() * w.double()).sum())

    for _ in range(5):
        step = torch.randn(T, V, generator=g).to(DEV)
        h = 2.0 ** -6
        # central differences: h^2 / 6 times a third derivative of a few; the losses' own error over 2 h
        slope = (value(z + h * step) - value(z - h * step)) / (2 * h)
        want = float((dz.double() * step.double()).sum())
        assert abs(slope - want) < 20 * h * h / 6 + T * 1.5 * 8e-6 / h, (slope, want)


def test_distill_refusals():
    L, p = bd.lib(), 4096
    mk = lambda dtype="bf16", T=3, V=100, k=5, **kw: bd.make_distill_desc(dtype, T, V, k, **kw)
    F = lambda d, z=p, l=p, i=p, loss=p, st=p: L.lobra_token_distill_fwd(ctypes.byref(d) if d else None, z, l, i, loss, st, None)
    B = lambda d, z=p, l=p, i=p, st=p, w=p, dz=p, flags=0: L.lobra_token_distill_bwd(ctypes.byref(d) if d else None, z, l, i, st, w, dz, flags, None)
    for call in (F, B):
        assert call(None) == -1 and call(mk(dtype=2)) == -3
        for bad in (mk(V=0), mk(V=(1 << 24) + 1), mk(T=-1), mk(T=1 << 31), mk(k=0), mk(k=129), mk(ld=99), mk(ld=1 << 59), mk(temperature=0.0), mk(temperature=-1.0),
                    mk(temperature=math.inf), mk(temperature=math.nan), mk(temperature=1e-40), mk(tail=2), mk(tail=-1)):
            assert call(bad) == -2
        assert call(mk(), z=None) == -1 and call(mk(), l=None) == -1 and call(mk(), i=None) == -1
        assert call(mk(), z=p + 2) == -8 and call(mk(), l=p + 2) == -8 and call(mk(), i=p + 1) == -8 and call(mk(), st=p + 4) == -8
        assert call(mk(T=0), z=None) == 0
    assert F(mk(), loss=None, st=None) == 0 and F(mk(), loss=p + 1) == -8
    assert B(mk(), st=None) == -1 and B(mk(), w=None) == -1 and B(mk(), dz=None) == -1 and B(mk(), w=p + 2) == -8 and B(mk(), dz=p + 8) == -8
    assert B(mk(), flags=bd.FLAG_ACCUMULATE_GRADS) == -2                 # (dlogits is logits)
    z, f, i = torch.zeros(3, 100).bfloat16(), torch.zeros(3, 5), torch.zeros(3, 5, dtype=torch.int32)
    loss, st = torch.zeros(3), torch.zeros(3, 4)
    for bad in (dict(logits=z.float()), dict(logits=z[:2]), dict(teacher_logp=f[:2]), dict(teacher_logp=f.double()), dict(teacher_id=i.long()), dict(teacher_id=i[:, :4]),
                dict(loss=loss[:2]), dict(loss=loss.half()), dict(stat=st[:2]), dict(stat=st.double())):
        with pytest.raises(AssertionError):
            bd.lobra_token_distill_fwd(mk(), **{**dict(logits=z, teacher_logp=f, teacher_id=i, loss=loss, stat=st), **bad}, stream=0)
    for bad in (dict(dlogits=z.float()), dict(dlogits=z[:, :99]), dict(dloss=loss[:2]), dict(dloss=loss.bfloat16())):
        with pytest.raises(AssertionError):
            bd.lobra_token_distill_bwd(mk(), **{**dict(logits=z, teacher_logp=f, teacher_id=i, stat=st, dloss=loss, dlogits=z), **bad}, stream=0)


# ------------------------------------------------------------------------------------------------------------------
# beam search
# ------------------------------------------------------------------------------------------------------------------
def ref_select(z, score, done, done_token, k):
    """Scores, beams, tokens [n, k], from all continuations sorted in 64 bits; equal ones stay in order."""
    n, b = score.shape
    V = z.shape[1]
    out = [], [], []
    for i in range(n):
        total = torch.full((b, V + 1), -math.inf, dtype=torch.float64)       # (the last column: a beam that is done)
        for j in range(b):
            s = float(score[i, j])
            if not s > -math.inf:
                continue
            if done is not None and int(done[i, j]):
                total[j, V] = s
                continue
            x = z[i * b + j].double()
            m = float(x.max())
            if bool(torch.isnan(x).any()) or not abs(m) < math.inf:
                continue
            total[j, :V] = (s - (m + math.log(float((x - m).exp().sum())))) + x
        v, at = torch.sort(total.flatten(), descending=True, stable=True)
        v, at = v[:k], at[:k]
        some = v > -math.inf
        tok = torch.where(at % (V + 1) == V, done_token, at % (V + 1))
        pad = (0, k - len(v))
        out[0].append(torch.nn.functional.pad(v, pad, value=-math.inf))
        out[1].append(torch.nn.functional.pad(torch.where(some, at // (V + 1), -1), pad, value=-1))
        out[2].append(torch.nn.functional.pad(torch.where(some, tok, -1), pad, value=-1))
    return tuple(torch.stack(o) for o in out)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,b,V,k,kind,pad", [
    (1, 1, 1, 1, "plain", 0), (2, 3, 2, 8, "plain", 0), (1, 4, 32000, 4, "plain", 0), (3, 5, 4099, 10, "plain", 3), (40, 2, 8192, 4, "plain", 0), (2, 4, 8193, 8, "plain", 1),
    (3, 8, 20001, 16, "offset", 0), (2, 16, 1000, 32, "plain", 0), (2, 32, 30, 32, "plain", 2), (2, 4, 5000, 32, "masked", 0), (2, 3, 9000, 8, "lowest", 0),
    (2, 4, 20000, 32, "equal", 0), (2, 2, 40960, 32, "constant", 0), (3, 4, 3001, 8, "twins", 0), (2, 4, 3000, 4, "nan", 0), (5, 4, 50257, 8, "first", 0),
    (7, 4, 500, 4, "done", 0), (2, 3, 70, 8, "none", 0), (1, 2, 300000, 32, "one_stride", 0), (2, 16, 70000, 32, "plain", 0), (1, 32, 40000, 32, "ahead", 1),
    (1, 16, 90000, 17, "ahead", 0), (1, 16, 70000, 32, "equal", 0),
])
def test_beam_select(dtype, n, b, V, k, kind, pad):
    z = logits_of(kind if kind in ("offset", "masked", "lowest", "equal", "nan", "one_stride") else "plain", n * b, V, dtype, n + b + V)
    g = torch.Generator().manual_seed(k)
    score = -10 * torch.rand(n, b, generator=g)
    done = None
    if kind == "constant":                           # nothing but equals
        z[:] = 0.5
        score[:] = -1.0
    elif kind == "twins":                            # beams of the same logits and score, whose rows begin at other alignments
        z = z[::b].repeat_interleave(b, dim=0).contiguous()
        score[:] = score[:, :1]
    elif kind == "first":
        score[:, 1:] = -math.inf
    elif kind == "ahead":                            # one beam far in front of the others
        score -= 30 * (torch.arange(b) != b // 2)
    elif kind == "done":
        done = (torch.rand(n, b, generator=g) < 0.6).int()
        done[0] = 1
        score[1, 2], score[2, 0] = math.nan, -math.inf
        z[0] = math.nan                              # (of a beam that is done)
    elif kind == "none":
        score[0] = -math.inf
        z[b:] = -math.inf
    want = ref_select(z, score, done, 2, k)
    wide = torch.full((n * b, V + pad), 1e4, dtype=DT[dtype], device=DEV)
    wide[:, :V] = z.to(DEV)
    desc = bd.make_beam_desc(dtype, n, b, V, k, ld=V + pad)
    ws, wok = guarded(bd.lobra_beam_workspace_bytes(desc), dtype=torch.uint8)
    os_, ob, ot = guarded(n, k, dtype=torch.float32), guarded(n, k, dtype=torch.int32), guarded(n, k, dtype=torch.int32)
    sd, dd = score.to(DEV), None if done is None else done.to(DEV)
    bd.lobra_beam_select(desc, wide[:, :V], sd, dd, 2, os_[0], ob[0], ot[0], ws)
    torch.cuda.synchronize()
    assert wok() and os_[1]() and ob[1]() and ot[1]()
    got, ref = os_[0].double().cpu(), want[0]
    assert bool(((got == ref) | ((got - ref).abs() <= 4e-6 + 2.0 ** -23 * ref.abs())).all()), (got, ref)
    assert torch.equal(ob[0].cpu().long(), want[1]), (ob[0], want[1])
    assert torch.equal(ot[0].cpu().long(), want[2]), (ot[0], want[2])
    if k == b:                                       # over the scores
        bd.lobra_beam_select(desc, wide[:, :V], sd, dd, 2, sd, ob[0], ot[0], ws)
        assert torch.equal(sd, os_[0])


@pytest.mark.gpu
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("n,b,shapes,dtype,limited", [
    (1, 1, [(3,)], torch.float32, False), (3, 4, [(5, 8), (7, 33), (1, 1)], torch.bfloat16, True), (2, 5, [(77, 33)], torch.float32, True),
    (5, 8, [(64, 512)] * 3, torch.bfloat16, True), (2, 32, [(11, 7)], torch.uint8, True), (2, 16, [(2000, 64), (3, 5), (2, 16)], torch.bfloat16, False),
    (3, 2, [(4, 6)] * 150, torch.float32, True), (2, 3, [(0, 4), (6, 0), (9, 4)], torch.float32, True), (70, 3, [(5,)], torch.int64, False),
])
def test_beam_reorder(in_place, n, b, shapes, dtype, limited):
    g = torch.Generator().manual_seed(n + b)
    parent = torch.randint(0, b, (n, b + 2), generator=g, dtype=torch.int32)
    parent[0, :b] = torch.arange(1, b + 1) % b       # a cycle
    if n > 1:
        parent[1, 0] = -1
        parent[1, b - 1] = b
    used = None
    if limited:
        used = torch.randint(0, 12, (n,), generator=g, dtype=torch.int32)
        used[0] = 1 << 30
        if n > 2:
            used[2] = -5
    src = [torch.randint(-100, 100, (n * b, *s), generator=g).to(dtype) for s in shapes]
    want, states, checks = [], [], []
    for s in src:
        d = s.clone() if in_place else torch.full_like(s, 99)
        for i in range(n):
            rows = s[i * b:(i + 1) * b].clone()
            for j in range(b):
                p = int(parent[i, j])
                if not 0 <= p < b:
                    continue
                if used is None:
                    d[i * b + j] = rows[p]
                else:
                    u = min(max(int(used[i]), 0), s.shape[1])
                    d[i * b + j, :u] = rows[p, :u]
        want.append(d)
        dev, ok = guarded(*s.shape, dtype=dtype)
        dev.copy_(s)
        out, ok2 = (dev, ok) if in_place else guarded(*s.shape, dtype=dtype)
        if not in_place:
            out.fill_(99)
        states.append((dev, out))
        checks += [ok, ok2]
    bd.lobra_beam_reorder(states, n, b, parent.to(DEV), None if used is None else used.to(DEV))
    torch.cuda.synchronize()
    assert all(ok() for ok in checks)
    for (s0, d), s, ref in zip(states, src, want):
        assert torch.equal(d.cpu(), ref)
        assert in_place or torch.equal(s0.cpu(), s)


@pytest.mark.gpu
def test_beam_reorder_beyond_32_bits():
    """Rows of 1.5 GB: offsets that 32 bits do not hold."""
    n, b, L = 1, 3, 3 * 2 ** 28
    s = torch.empty(n * b, L, dtype=torch.int16, device=DEV)
    for i in range(b):
        s[i].fill_(i + 1)
        s[i, -1] = 100 + i
    bd.lobra_beam_reorder([(s, s)], n, b, torch.tensor([[2, 1, 0]], dtype=torch.int32, device=DEV))
    torch.cuda.synchronize()
    assert [int(v) for v in s[:, -1]] == [102, 101, 100]
    for i, v in enumerate((3, 2, 1)):
        assert bool((s[i, :-1] == v).all())


def test_beam_refusals():
    L, p, n = bd.lib(), 4096, ctypes.c_size_t()
    mk = lambda dtype="bf16", n=2, b=3, V=100, k=4, **kw: bd.make_beam_desc(dtype, n, b, V, k, **kw)
    size = lambda d: L.lobra_beam_workspace_bytes(ctypes.byref(d) if d else None, ctypes.byref(n))
    S = lambda d, z=p, s=p, done=p, os=p + 64, ob=p, ot=p, ws=p, nb=1 << 30: L.lobra_beam_select(ctypes.byref(d) if d else None, z, s, done, 2, os, ob, ot, ws, nb, None)
    for call in (size, S):
        assert call(None) == -1 and call(mk(dtype=2)) == -3
        for bad in (mk(V=0), mk(V=(1 << 24) + 1), mk(n=-1), mk(b=0), mk(b=33), mk(k=0), mk(k=33), mk(ld=99), mk(ld=1 << 58), mk(n=1 << 23), mk(n=1 << 17, V=1 << 20)):
            assert call(bad) == -2
    assert size(mk()) == 0 and n.value == 6 * (4 * 8 + 8) and L.lobra_beam_workspace_bytes(ctypes.byref(mk()), None) == -1
    assert S(mk(n=0), z=None) == 0
    assert S(mk(), z=None) == -1 and S(mk(), s=None) == -1 and S(mk(), os=None) == -1 and S(mk(), ob=None) == -1 and S(mk(), ot=None) == -1
    assert S(mk(), z=p + 2) == -8 and S(mk(), s=p + 2) == -8 and S(mk(), done=p + 2) == -8 and S(mk(), ws=p + 8) == -8 and S(mk(), ot=p + 1) == -8
    assert S(mk(), ws=None) == -7 and S(mk(), nb=6 * 40 - 1) == -7
    assert S(mk(), os=p) == -2                       # (over the scores, of which there are fewer)
    z, f, i = torch.zeros(6, 100).bfloat16(), torch.zeros(2, 3), torch.zeros(2, 3, dtype=torch.int32)
    of, oi, ws = torch.zeros(2, 4), torch.zeros(2, 4, dtype=torch.int32), torch.zeros(512, dtype=torch.uint8)
    ok = dict(logits=z, score=f, done=i, done_token=2, out_score=of, out_beam=oi, out_token=oi, ws=ws)
    for bad in (dict(logits=z.float()), dict(logits=z[:5]), dict(score=f[:1]), dict(score=f.double()), dict(done=i.bool()), dict(done=i[:1]), dict(out_score=of[:1]),
                dict(out_beam=oi.long()), dict(out_token=oi[:, :2])):
        with pytest.raises(AssertionError):
            bd.lobra_beam_select(mk(), **{**ok, **bad}, stream=0)


def test_reorder_refusals():
    L, p = bd.lib(), 1 << 20

    def R(src=p, dst=p, row=64, unit=8, n_states=1, n=2, b=3, parent=p, ld=3, used=p, arr=True):
        t = (bd.BeamState * 1)(bd.BeamState(src, dst, row, unit))
        return L.lobra_beam_reorder(t if arr else None, n_states, n, b, parent, ld, used, None)

    for bad in (dict(n_states=-1), dict(n=-1), dict(b=0), dict(b=33), dict(ld=2), dict(ld=1 << 40), dict(n=1 << 23), dict(row=-1), dict(unit=-1), dict(row=1 << 58)):
        assert R(**bad) == -2, bad
    assert R(arr=False) == -1 and R(src=None) == -1 and R(dst=None) == -1 and R(parent=None) == -1
    assert R(parent=p + 2) == -8 and R(used=p + 1) == -8
    for shift in (1, 64, 383, -1, -383):             # six rows of 64 bytes
        assert R(dst=p + shift) == -2
    assert R(n_states=0) == 0 and R(n=0) == 0 and R(row=0, src=None, dst=None) == 0
    s, par = torch.zeros(6, 4, 5), torch.zeros(2, 3, dtype=torch.int32)
    for bad in (dict(states=[(s, s.half())]), dict(states=[(s, s[:, :3].contiguous())]), dict(states=[(s[:5], s[:5])]), dict(parent=par.long()), dict(parent=par[:1]),
                dict(parent=par[:, :2]), dict(used=par[0, :1]), dict(states=[(s[:, 0, 0].contiguous(),) * 2]), dict(states=[(s[:, :, 1:],) * 2])):
        with pytest.raises(AssertionError):
            bd.lobra_beam_reorder(**{**dict(states=[(s, s)], n_req=2, beams=3, parent=par, used=torch.zeros(2, dtype=torch.int32)), **bad}, stream=0)


# ------------------------------------------------------------------------------------------------------------------
@pytest.mark.gpu
def test_on_another_stream_and_in_a_graph():
    """A teacher's tokens from the library's own log probabilities, loss and gradient; a step of beam search with its states."""
    n, b, V, k, L = 3, 4, 5003, 4, 20
    g = torch.Generator().manual_seed(2)
    teacher, z = (torch.randn(n * b, V, generator=g).bfloat16().to(DEV) * 3 for _ in range(2))
    score, hist = -torch.rand(n, b, generator=g).to(DEV), torch.randint(0, V, (n * b, L), generator=g, dtype=torch.int32).to(DEV)
    w = torch.rand(n * b, generator=g).to(DEV)
    ld, dd, bdsc = bd.make_logprob_desc("bf16", n * b, V, top_k=20), bd.make_distill_desc("bf16", n * b, V, 20, tail=True), bd.make_beam_desc("bf16", n, b, V, k)
    ws = torch.empty(bd.lobra_beam_workspace_bytes(bdsc), dtype=torch.uint8, device=DEV)

    def outputs():
        f = lambda *s, dt=torch.float32: torch.zeros(*s, dtype=dt, device=DEV)
        return dict(tl=f(n * b, 20), ti=f(n * b, 20, dt=torch.int32), loss=f(n * b), st=f(n * b, 4), dz=torch.zeros_like(z), s=f(n, k), bm=f(n, k, dt=torch.int32),
                    tk=f(n, k, dt=torch.int32), next=torch.zeros_like(hist))

    def go(o):
        bd.lobra_token_logprob_fwd(ld, teacher, None, top_logp=o["tl"], top_id=o["ti"])
        bd.lobra_token_distill_fwd(dd, z, o["tl"], o["ti"], o["loss"], o["st"])
        bd.lobra_token_distill_bwd(dd, z, o["tl"], o["ti"], o["st"], w, o["dz"])
        bd.lobra_beam_select(bdsc, z, score, None, 2, o["s"], o["bm"], o["tk"], ws)
        bd.lobra_beam_reorder([(hist, o["next"])], n, b, o["bm"])

    eager, other, graphed = outputs(), outputs(), outputs()
    go(eager)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        go(other)
    torch.cuda.synchronize()
    assert all(torch.equal(eager[i], other[i]) for i in eager)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        go(graphed)
    for r in range(3):
        z.mul_(1.0 if r == 0 else 0.7)
        graph.replay()
        torch.cuda.synchronize()
        go(eager)
        torch.cuda.synchronize()
        assert all(torch.equal(eager[i], graphed[i]) for i in eager), r


def test_reorder_of_tensors_that_meet():
    """Two tensors of a list where one writes what is the other's too; six rows of 64 bytes."""
    L, p = bd.lib(), 1 << 20

    def R(*pairs):
        t = (bd.BeamState * len(pairs))(*(bd.BeamState(a, b, 64, 8) for a, b in pairs))
        return L.lobra_beam_reorder(t, len(pairs), 2, 3, None, 3, None, None)

    for pairs in (((p, p), (p, p)), ((p, p), (p + 383, p + 383)), ((p, p + 4096), (p + 8192, p + 4096)), ((p, p + 4096), (p + 4096 + 64, p + 8192)),
                  ((p, p), (p + 4096, p + 4096), (p, p + 8192)), ((p + 4096, p + 8192), (p, p + 4096 + 383))):
        assert R(*pairs) == -2, pairs
    # (as far as the missing parents)
    assert R((p, p), (p + 384, p + 384)) == -1 and R((p, p + 4096), (p, p + 8192)) == -1 and R((p, p + 384), (p + 768, p + 1152)) == -1


def test_host_tensors():
    """What lies in host memory is refused before anything is launched."""
    z, f, i = torch.zeros(3, 100).bfloat16(), torch.zeros(3, 5), torch.zeros(3, 5, dtype=torch.int32)
    dd, bm = bd.make_distill_desc("bf16", 3, 100, 5), bd.make_beam_desc("bf16", 1, 3, 100)
    one, par, ws = torch.zeros(1, 3), torch.zeros(1, 3, dtype=torch.int32), torch.zeros(4096, dtype=torch.uint8)
    for call in (lambda: bd.lobra_token_distill_fwd(dd, z, f, i, torch.zeros(3), torch.zeros(3, 4), stream=0),
                 lambda: bd.lobra_token_distill_bwd(dd, z, f, i, torch.zeros(3, 4), torch.zeros(3), z, stream=0),
                 lambda: bd.lobra_beam_select(bm, z, one, None, 2, one, par, par.clone(), ws, stream=0),
                 lambda: bd.lobra_beam_reorder([(z, z)], 1, 3, par, stream=0)):
        with pytest.raises(AssertionError, match="host tensor"):
            call()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("noise", [0.05, 0.7])
@pytest.mark.parametrize("T,V,k,temperature", [(60, 16064, 4, 2.0), (9, 20099, 32, 2.0), (30, 70528, 1, 2.0), (3, 108864, 1, 2.0), (50, 3001, 64, 0.7), (40, 2048, 10, 1.0)])
def test_distill_of_nearly_the_same_model(dtype, noise, T, V, k, temperature):
    """A loss far below 1, terms near 1 that cancel, with a tail.  Only the sum over what is not listed is in fp32.  A relative error e of it moves
    ln S by p_r e and ln p_r by (1 - p_r) e, so the loss by (sum q p_r - q_r (1 - p_r)) e = (p_r - q_r) e; the loss itself is rounded once more, by 2^-24.  e, in units of 2^-24: 4 for
    each unit of the exponents, weighted as the sum weighs them (difference, scale's own two roundings, product), 2 for the exponential, one an addition (up to 64 or V / 512 in a
    thread, 14 behind it), 24 for rescaling on the way."""
    g = torch.Generator().manual_seed(V)
    z = (torch.randn(T, V, generator=g) * 2.5).to(DT[dtype])
    z[torch.arange(T), torch.randint(0, V, (T,), generator=g)] += (torch.rand(T, generator=g) * 16).to(DT[dtype])
    teacher = (z.double() + noise * torch.randn(T, V, generator=g)) / temperature
    tl, ids = torch.log_softmax(teacher, dim=1).topk(k, dim=1)
    tl, ids = tl.float(), ids.int()
    held = float(np.float32(temperature))            # (what the descriptor holds)
    want, _, _ = ref_distill(z, tl, ids, True, held)
    x = z.double() / held * math.log2(math.e)
    x = x - x.max(dim=1, keepdim=True).values
    e = torch.exp2(x)
    rest = e.scatter(1, ids.long(), 0.0)
    p_r, q_r = rest.sum(dim=1) / e.sum(dim=1), 1 - tl.double().exp().sum(dim=1)
    size = (rest * x.abs()).sum(dim=1) / rest.sum(dim=1)
    off = 2.0 ** -24 * (want.abs() + (4 * size + 2 + max(64, V / 512) + 14 + 24) * (p_r - q_r).abs()) + 4e-13          # (in 64 bits: some hundred terms of up to 30)
    loss = torch.empty(T, device=DEV)
    bd.lobra_token_distill_fwd(bd.make_distill_desc(dtype, T, V, k, tail=True, temperature=temperature), z.to(DEV), tl.to(DEV), ids.to(DEV), loss)
    got = loss.double().cpu()
    print("%s V %d noise %g: losses of %.1e, off by %.1e of themselves, allowed %.1e" % (
        dtype, V, noise, float(want.abs().median()), float((got - want).norm() / want.norm()), float(off.norm() / want.norm())))
    assert bool(((got - want).abs() <= off).all()), ((got - want).abs() / off).max()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("far", [-1e9, -1e30, "lowest", 1e30, math.inf])
def test_scores_that_swallow_the_logits(dtype, far):
    """Scores next to which logits are lost even in 64 bits (the type's lowest value for a beam that is none, for one): a beam's continuations still come by its logits."""
    n, b, V, k = 2, 4, 20000, 8
    far = -3.4028234663852886e38 if far == "lowest" else far
    g = torch.Generator().manual_seed(11)
    z = (torch.randn(n * b, V, generator=g) * (1e-7 if far == -1e9 else 3)).to(DT[dtype])
    z[:, 5000:5200] = -math.inf
    score = torch.tensor([[-1.0, far / 2, far, -math.inf], [far, -math.inf, far, math.nan]])
    few = [17, 900, 19000]
    z[0] = -math.inf                                 # the beam of an ordinary score has three continuations
    z[0, few] = torch.tensor([1.0, 3.0, 2.0]).to(DT[dtype])
    z[6] = z[4]                                      # equal beams: the lower one's, one of its own behind the other
    desc = bd.make_beam_desc(dtype, n, b, V, k)
    f = lambda dt: torch.empty(n, k, dtype=dt, device=DEV)
    os_, ob, ot = f(torch.float32), f(torch.int32), f(torch.int32)
    ws = torch.empty(bd.lobra_beam_workspace_bytes(desc), dtype=torch.uint8, device=DEV)
    bd.lobra_beam_select(desc, z.to(DEV), score.to(DEV), None, 2, os_, ob, ot, ws)
    own = lambda row: torch.sort(z[row].float(), descending=True, stable=True).indices[:k].tolist()
    first = [(0, t) for t in (900, 19000, 17)]
    rest = [(1, t) for t in own(1)]
    # (half of infinity is infinity: the lower beam)
    want0 = (first + rest)[:k] if far < 0 else rest if far == math.inf else [(2, t) for t in own(2)]
    got = [list(zip(ob[i].tolist(), ot[i].tolist())) for i in range(n)]
    assert got[0] == want0, (got[0], want0)
    if far == -1e9:                                  # (the two beams' continuations of equal value alternate)
        assert [t for bb, t in got[1] if bb == 0] == own(4)[:sum(bb == 0 for bb, _ in got[1])]
        assert [t for bb, t in got[1] if bb == 2] == own(4)[:sum(bb == 2 for bb, _ in got[1])]
    else:
        assert got[1] == [(0, t) for t in own(4)], (got[1], own(4))
    assert bool((os_[1] == far).all()) or far == -1e9


def peaks(dtype, V, b, k):
    """Logits [b, V] with one peak in every part of 16 KB, each reaching far over what the k-th largest of a part has elsewhere, and their scores."""
    part, g = 4096 if dtype == "f32" else 8192, torch.Generator().manual_seed(V)
    z = torch.randn(b, V, generator=g)
    at = torch.arange(0, V, part)
    at = at + torch.randint(0, V - int(at[-1]), (len(at),), generator=g)
    z[:, at] = 20 + 0.01 * torch.randperm(b * len(at), generator=g).view(b, -1)
    return z.to(DT[dtype]), -1 - 0.003 * torch.arange(b)[None, :], len(at) * b


PARTS = [("f32", 131072, 1024), ("f32", 131073, 1056), ("f32", 151000, 1184), ("bf16", 262144, 1024), ("bf16", 300000, 1184)]


def test_peaks_are_far_enough_apart():
    """Of the inputs below: no two continuations that are wanted, or next to those, lie nearer to each other than the kernel's sums are exact, but those of one beam."""
    for dtype, V, parts in PARTS:
        z, score, n = peaks(dtype, V, 32, 32)
        assert n == parts
        v, beam, _ = (t[0] for t in ref_select(z, score, None, 2, 40))
        assert bool(((v[:-1] - v[1:] > 2e-5) | (beam[:-1] == beam[1:])).all())


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["peaks", "constant"])
@pytest.mark.parametrize("dtype,V,parts", PARTS)
def test_more_parts_than_the_merge_lists(dtype, V, parts, kind):
    """32 beams, all of whose parts reach the merge's first threshold, with more candidates than its list holds: up to 1024 parts are listed in their turn, more are looked at
    as they lie; the counts leave 32 peaks, or all candidates, which are equal."""
    b = k = 32
    z, score, _ = peaks(dtype, V, b, k)
    if kind == "constant":
        z[:], score[:] = 0.5, -1.0
    want = ref_select(z, score, None, 2, k)
    desc = bd.make_beam_desc(dtype, 1, b, V, k)
    ws, wok = guarded(bd.lobra_beam_workspace_bytes(desc), dtype=torch.uint8)
    o = [guarded(1, k, dtype=dt) for dt in (torch.float32, torch.int32, torch.int32)]
    bd.lobra_beam_select(desc, z.to(DEV), score.to(DEV), None, 2, *(t for t, _ in o), ws)
    torch.cuda.synchronize()
    assert wok() and all(ok() for _, ok in o)
    assert bool(((o[0][0].double().cpu() - want[0]).abs() <= 4e-6 + 2.0 ** -23 * want[0].abs()).all())
    assert torch.equal(o[1][0].cpu().long(), want[1]) and torch.equal(o[2][0].cpu().long(), want[2]), (o[1][0], want[1], o[2][0], want[2])


def meet(pairs, size):
    """Whether a tensor of the list writes what another one reads or writes, pair by pair; pairs of addresses, sizes of the tensors."""
    over = lambda p, n, q, m: p < q + m and q < p + n
    return any(size[i] and size[j] and (over(b, size[i], d, size[j]) or over(b, size[i], c, size[j]) or over(a, size[i], d, size[j]))
               for i, (a, b) in enumerate(pairs) for j, (c, d) in enumerate(pairs[:i]))


@pytest.mark.parametrize("n", [1, 2, 3, 7, 40, 255, 256, 257, 300, 700])
def test_which_lists_of_states_meet(n):
    """Lists that do and lists that don't, of every length around what is sorted at a time, against pair by pair; six rows a tensor."""
    L, rng, seen = bd.lib(), np.random.default_rng(n), set()
    for trial in range(60 if n < 100 else 12):
        row = rng.choice([0, 16, 32, 48], size=n, p=[0.05, 0.35, 0.3, 0.3])
        # places of their own, some of which are given up for one that another tensor has, or one next to it
        place = (1 << 20) + 288 * rng.permutation(2 * n)
        src, dst = place[:n].copy(), np.where(rng.random(n) < 0.4, place[:n], place[n:])
        for _ in range(int(rng.integers(0, 3))):
            i, j, shift = int(rng.integers(n)), int(rng.integers(n)), int(rng.choice([0, 16, 272, -272, 288]))
            k = rng.integers(4)
            if k == 0:
                src[i] = src[j]                      # (read twice)
            elif k == 1:
                dst[i] = dst[j] + shift
            elif k == 2:
                src[i] = dst[j] + shift
            else:
                dst[i] = src[j] + shift
        pairs, size = list(zip(src.tolist(), dst.tolist())), (6 * row).tolist()
        own = any(s and a != b and abs(a - b) < s for (a, b), s in zip(pairs, size))
        want = -2 if own or meet(pairs, size) else 0 if not any(size) else -1        # (-1: as far as the missing parents)
        t = (bd.BeamState * n)(*(bd.BeamState(a, b, s // 6, 8) for (a, b), s in zip(pairs, size)))
        assert L.lobra_beam_reorder(t, n, 2, 3, None, 3, None, None) == want, (trial, pairs[:4], size[:4])
        seen.add(want)
    assert n == 1 or {-1, -2} <= seen


def test_a_long_list_of_states_is_looked_at_quickly():
    """Keys and values of 80 layers, and of 640: eight times the tensors take less than 24 times as long on the host, where pair by pair it would be 64."""
    import time
    L, best = bd.lib(), {}
    for n in (160, 1280):
        t = (bd.BeamState * n)(*(bd.BeamState(*((1 << 20) + (i * 7919 % n) * 4096,) * 2, 64, 8) for i in range(n)))
        best[n] = math.inf
        for _ in range(30):
            a = time.perf_counter()
            assert L.lobra_beam_reorder(t, n, 2, 3, None, 3, None, None) == -1
            best[n] = min(best[n], time.perf_counter() - a)
    assert best[1280] < 24 * best[160], best


@pytest.mark.gpu
def test_reorder_that_would_write_its_own_parents():
    """The parents and the used lengths are read while states are written: a list that writes them is refused, one that has them next door is not; six rows of 64 bytes, 32
    bytes of parents (rows of three numbers, five apart), 8 of lengths, all in one allocation."""
    L, stream = bd.lib(), torch.cuda.current_stream().cuda_stream
    buf = torch.zeros(1 << 20, dtype=torch.uint8, device=DEV)
    p, away = buf.data_ptr() + 8192, buf.data_ptr() + (1 << 19)
    far = [(p + (i + 1) * 1024, p + (i + 1) * 1024 + 512) for i in range(300)]        # (more than what is sorted at a time)

    def R(pairs, parent, used=None):
        t = (bd.BeamState * len(pairs))(*(bd.BeamState(a, b, 64, 8) for a, b in pairs))
        return L.lobra_beam_reorder(t, len(pairs), 2, 3, parent, 5, used, stream)

    for pairs in ([(p, p)], [(p - 4096, p)], far + [(p, p)], [(p, p)] + far):
        for at in (p, p + 380, p - 28):
            assert R(pairs, at) == -2, at
        for at in (p, p + 380, p - 4):
            assert R(pairs, away, at) == -2, at
        assert R(pairs, p + 384, p - 8) == 0 and R(pairs, p - 32, p + 384) == 0
    assert R([(p, p + 4096)], p, p) == 0             # (what is only read may be both)
    torch.cuda.synchronize()
    row = torch.arange(6, dtype=torch.int32, device=DEV).repeat_interleave(16)
    state, par = buf[8192:8192 + 384].view(torch.int32), buf[8192 - 32:8192].view(torch.int32)
    state.copy_(row)
    par.copy_(torch.tensor([2, 0, 1, 9, 9, 1, 1, 0], dtype=torch.int32))
    assert R([(p, p)], p - 32) == 0
    assert state.view(6, 16)[:, 0].tolist() == [2, 0, 1, 4, 4, 3] and par.tolist() == [2, 0, 1, 9, 9, 1, 1, 0]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("T,V,k,temperature,teacher,pad", [(1, 6, 64, 1.0, "short", 8), (5, 1000, 20, 2.0, "full", 0), (12, 4099, 1, 4.0, "full", 3), (9, 32000, 65, 1.0, "short", 0),
                                                           (3, 70000, 128, 2.0, "full", 0)])
def test_distill_of_rows_of_the_lowest_value(dtype, tail, T, V, k, temperature, teacher, pad):
    """A row of nothing but a mask's lowest value, with a teacher: its tokens are equally likely, though ln of their number is lost next to the logits."""
    test_distill(dtype, tail, T, V, k, temperature, "lowest", teacher, pad)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("far", [1e6, -1e12, 3e38, -3e38])
def test_distill_far_from_0(dtype, tail, far):
    """Logits of one huge value with a few that are a little apart from it or far below it, and without a tail a teacher of huge values too."""
    T, V, k = 4, 300, 5
    g = torch.Generator().manual_seed(1)
    z = torch.full((T, V), far)
    z[0, ::7] += abs(far) * 2.0 ** -7                # (a step of bf16: far beyond what exp survives)
    z[1, 1::2] = -math.inf
    z[2, :200] = torch.finfo(torch.float32).min
    z = torch.nan_to_num(z.to(DT[dtype]).float(), posinf=3.3e38, neginf=-math.inf).to(DT[dtype])
    ids = torch.stack([torch.randperm(V, generator=g)[:k] for _ in range(T)]).int()
    ids[1] = ids[1] // 2 * 2
    ids[2] = 200 + ids[2] % 100
    ids[0] = ids[0] // 7 * 7                         # (elsewhere p is 0 and the loss beyond fp32)
    tl = torch.log_softmax(torch.randn(T, k + 2, generator=g), dim=1)[:, :k].contiguous()
    if not tail:
        tl[3] = far if abs(far) < 1e7 else -1e30
    desc = bd.make_distill_desc(dtype, T, V, k, tail=tail)
    loss, grad, _ = ref_distill(z, tl, ids, tail, 1.0)
    if tail:
        assert bool((loss[[1, 3]].abs() < 100).all())
    zd, td, idd = z.to(DEV), tl.to(DEV), ids.to(DEV)
    ld, st, dz = torch.empty(T, device=DEV), torch.empty(T, 4, device=DEV), torch.empty(T, V, dtype=DT[dtype], device=DEV)
    bd.lobra_token_distill_fwd(desc, zd, td, idd, ld, st)
    bd.lobra_token_distill_bwd(desc, zd, td, idd, st, torch.ones(T, device=DEV), dz)
    got = ld.double().cpu()
    fine = loss.abs() < 3.4e38
    assert bool((((got - loss).abs() <= 4e-6 + 2.0 ** -20 * loss.abs()) | ~fine).all()) and bool((got[~fine] > 3.3e38).all()), (got, loss)
    # (what a listed token stands for is rounded once, by 2^-24 of ln k or of the logit's distance, all else as in test_distill)
    off = (dz.double().cpu() - grad).abs()
    assert bool((off <= 2e-6 * 2 + (grad.abs() * 2.0 ** -8 if dtype == "bf16" else 0)).all()), (off.max(dim=1).values, got, loss)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("T,V,k,kind,teacher", [(4, 1, 2, "nan", "full"), (2, 1, 127, "nan", "short"), (10, 3, 63, "masked", "odd"), (10, 1, 128, "masked", "odd"), (3, 2, 3, "nan", "full")])
def test_distill_of_nothing_but_nan(dtype, tail, T, V, k, kind, teacher):
    """NaN that the tail leaves out of the sums, next to nothing; a teacher of NaN over logits of nothing."""
    test_distill(dtype, tail, T, V, k, 1.0, kind, teacher, 0)


def test_temperatures_whose_exponents_are_not_finite():
    """1 / temperature is finite from 2.94e-39 on, log2 e / temperature, which the exponentials take, from 4.24e-39."""
    L, p = bd.lib(), 4096
    for t, want in ((2e-39, -2), (3e-39, -2), (4.2e-39, -2), (4.3e-39, 0), (1e-38, 0), (3e38, 0)):
        d = bd.make_distill_desc("bf16", 3, 100, 5, temperature=t)
        assert L.lobra_token_distill_fwd(ctypes.byref(d), p, p, p, None, None, None) == want, t           # (without outputs: nothing is launched)
        if want:
            assert L.lobra_token_distill_bwd(ctypes.byref(d), p, p, p, p, p, p, 0, None) == want, t
