"""The layer on a base in 8-bit integers, against its definition in 64 bits.

Tolerances count roundings.  The whole numbers are compared as they are.  A rounding to bf16 is off by at most 2^-8 of its value: y and dx have one
at the end, the projected activations s_t A_t x and s_t B_t dy one before they are multiplied, and so has the weight in backward; each enters
with the sum of the magnitudes that it is multiplied with.  fp32 sums: 2e-6 of the largest.
"""
import ctypes
import math

import numpy as np
import pytest

from paper_2509_01193_amd import binding as bd

torch = pytest.importorskip("torch")
from test_step_ops import DEV, batch_of, guarded  # noqa: E402

HALF = 2.0 ** -8


def quantised(v):
    """(whole numbers, 32-bit scales) of the rows of v, in 64 bits."""
    v = v.double()
    top = v.abs().amax(dim=1, keepdim=True)
    bad = ~torch.isfinite(v).all(dim=1, keepdim=True)
    scale = torch.where(bad | (top < 127 * 2.0 ** -126), 0.0, top / 127).float().double()
    q = torch.where(scale > 0, v / torch.where(scale > 0, scale, 1.0), 0.0).round()
    return q, torch.where(bad, math.nan, scale)


def make(T, d_in, d_out, ranks, batch, n_proj=1, seed=0, std=1.0):
    off, task = batch_of(batch, T, len(ranks)) if T else ([0], [])
    if not ranks:
        task = [-1] * len(task)
    g = torch.Generator().manual_seed(seed + T + d_in + d_out)
    mk = lambda *s: torch.randn(*s, generator=g).bfloat16()
    stacked = [r * n_proj for r in ranks]
    R = sum(stacked)
    v = dict(x=mk(T, d_in) * std, W=mk(d_in, d_out) * 0.05, A=mk(R, d_in) * 0.1, B=mk(R, d_out // n_proj) * 0.1,
             s=torch.rand(max(len(ranks), 1), generator=g) + 0.5, dy=mk(T, d_out))
    return v, off, task, [0] + np.cumsum(stacked).tolist()


def reference(v, off, task, rank_off, n_proj):
    q, xs = quantised(v["x"])
    wq, ws = quantised(v["W"].t())
    What = (wq * ws).t()
    x, A, B, dy = (v[k].double() for k in ("x", "A", "B", "dy"))
    y, dx = (q * xs) @ What, dy @ What.t()
    y_off, dx_off = torch.zeros_like(y), HALF * (dy.abs() @ What.abs().t())
    dA, dB = torch.zeros_like(A), torch.zeros_like(B)
    dA_off, dB_off = torch.zeros_like(A), torch.zeros_like(B)
    dg = B.shape[1]
    of = np.repeat(np.asarray(task, dtype=int), np.diff(np.asarray(off)))
    for t in range(len(rank_off) - 1):
        rows = torch.from_numpy(np.nonzero(of == t)[0])
        if not len(rows):
            continue
        s, r = float(v["s"][t]), (rank_off[t + 1] - rank_off[t]) // n_proj
        for j in range(n_proj):
            w = slice(rank_off[t] + j * r, rank_off[t] + (j + 1) * r)
            cols = slice(j * dg, (j + 1) * dg)
            h, g = s * (x[rows] @ A[w].t()), s * (dy[rows][:, cols] @ B[w].t())
            y[rows, cols] += h @ B[w]
            y_off[rows, cols] += HALF * (h.abs() @ B[w].abs())
            dx[rows] += g @ A[w]
            dx_off[rows] += HALF * (g.abs() @ A[w].abs())
            dA[w], dA_off[w] = g.t() @ x[rows], HALF * (g.abs().t() @ x[rows].abs())
            dB[w], dB_off[w] = h.t() @ dy[rows][:, cols], HALF * (h.abs().t() @ dy[rows][:, cols].abs())
    return dict(y=y, dx=dx, dA=dA, dB=dB), dict(y=y_off, dx=dx_off, dA=dA_off, dB=dB_off), wq, ws


def within(got, ref, off, rounded, what):
    got, ref = got.detach().double().cpu(), ref
    top = ref[torch.isfinite(ref)].abs().max() if ref.numel() and bool(torch.isfinite(ref).any()) else 0.0
    bound = off + (HALF * (ref.abs() + off) if rounded else 0) + 2e-6 * top
    bad = ~(((got - ref).abs() <= bound) | (torch.isnan(got) & torch.isnan(ref)))
    assert not bool(bad.any()), "%s: %d of %d, e.g. %r for %r" % (what, int(bad.sum()), bad.numel(), got[bad][:3].tolist(), ref[bad][:3].tolist())


def on_device(v):
    return {k: t.to(DEV) for k, t in v.items()}


def weight(d, W, d_in, d_out):
    wq, wq_ok = guarded(d_out, bd.lobra_quant_pitch(d_in), dtype=torch.int8)
    ws, ws_ok = guarded(d_out, dtype=torch.float32)
    bd.lobra_quantise_weight(W, wq, ws)
    torch.cuda.synchronize()
    assert wq_ok() and ws_ok()
    return wq, ws


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("d_in,d_out,pad", [(1, 1, 0), (7, 5, 0), (256, 64, 0), (257, 65, 3), (300, 1000, 0), (1376, 130, 5)])
def test_weight_in_whole_numbers(dtype, d_in, d_out, pad):
    g = torch.Generator().manual_seed(d_in)
    W = torch.randn(d_in, d_out + pad, generator=g)
    W[:, 0] = 0                                      # a channel of zeros
    if d_out > 4:
        W[:, 1] = (torch.randint(-63, 63, (d_in,), generator=g) + 0.5)          # halves everywhere: a scale of 1
        W[0, 1] = 127.0
        W[:, 2] = W[:, 2] * 1e-37                    # next to the smallest numbers
        W[:, 3] = W[:, 3] * 1e-39                    # below them
        W[-1, 4] = math.inf if d_in % 2 else math.nan
    W = W.to(dtype)
    wide = W.to(DEV)
    wq, ws = weight(None, wide[:, :d_out], d_in, d_out)
    q, scale = quantised(W[:, :d_out].t())
    assert torch.equal(wq[:, :d_in].cpu().double(), q)
    assert not bool(wq[:, d_in:].any())
    got = ws.cpu().double()
    assert bool(((got == scale[:, 0]) | (torch.isnan(got) & torch.isnan(scale[:, 0]))).all())


SHAPES = [
    # T, d_in, d_out, ranks, batch, n_proj
    (1, 8, 8, [1], "one", 1), (1, 4096, 512, [16], "one", 1), (3, 264, 72, [3, 8], "tokens", 1), (40, 4096, 1024, [16] * 4, "tokens", 1),
    (64, 256, 256, [8, 128], "mixed", 1), (65, 1376, 136, [16, 64, 5], "mixed", 1), (200, 512, 2048, [16], "bare", 1), (255, 1000, 1000, [], "one", 1),
    (256, 256, 256, [16, 32], "mixed", 1), (257, 264, 264, [16, 33], "mixed", 1), (700, 1376, 1032, [8, 16, 32], "mixed", 1),
    (1030, 520, 4096, [64, 1, 16], "mixed", 1), (4500, 768, 1288, [16, 16, 8], "mixed", 1), (2600, 1032, 2056, [128], "one", 1),
    (33, 512, 384, [8, 16], "mixed", 3), (300, 640, 768, [16, 8], "mixed", 2), (2100, 520, 1536, [16, 32], "mixed", 3), (900, 264, 720, [8], "mixed", 3),
]


@pytest.mark.gpu
@pytest.mark.parametrize("T,d_in,d_out,ranks,batch,n_proj", SHAPES)
def test_layer(T, d_in, d_out, ranks, batch, n_proj):
    v, off, task, rank_off = make(T, d_in, d_out, ranks, batch, n_proj)
    v["x"][T // 2] = 0                               # a token of zeros
    if T > 3:
        v["x"][1] *= 1e-20
        v["x"][2] *= 1e20
        v["dy"][2] *= 1e-20
    ref, off_by, wq_ref, _ = reference(v, off, task, rank_off, n_proj)
    d = on_device(v)
    wq, ws = weight(d, d["W"], d_in, d_out)
    assert torch.equal(wq[:, :d_in].cpu().double(), wq_ref)
    plan = bd.Plan("bf16", T, d_in, d_out, rank_off if ranks else None, off, task, n_proj=n_proj)
    fwd, bwd = bd.lobra_mlora_quant_workspace_bytes(plan)
    G = {k: guarded(*t.shape, dtype=torch.bfloat16 if k in ("y", "dx") else torch.float32) for k, t in ref.items()}
    o = {k: t for k, (t, _) in G.items()}
    w = (d["x"], wq, ws) + ((d["A"], d["B"], d["s"]) if ranks else (None, None, None))
    rows = {k: (v["x"].double().abs().amax(dim=1) < 1e15) if k in ("y", "dx") else slice(None) for k in ref}
    for saved in (True, False):
        ws1, ok1 = guarded(max(fwd, 16), dtype=torch.uint8)
        ws2, ok2 = guarded(max(bwd, 16), dtype=torch.uint8)
        h, ok3 = guarded(max(plan.h_save_bytes, 16), dtype=torch.uint8)
        for t in o.values():
            t.fill_(7)
        bd.lobra_mlora_quant_fwd(plan, *w, o["y"], h if saved else None, ws1)
        bd.lobra_mlora_quant_bwd(plan, *w, d["dy"], h if saved else None, o["dx"], o["dA"] if ranks else None, o["dB"] if ranks else None, 0, ws2)
        torch.cuda.synchronize()
        assert ok1() and ok2() and ok3() and all(ok() for _, ok in G.values())
        for k in ref:
            if ranks or k in ("y", "dx"):
                within(o[k][rows[k]], ref[k][rows[k]], off_by[k][rows[k]], k in ("y", "dx"), "%s saved=%s" % (k, saved))
        if T > 3:                                    # the large row by itself, whose size would hide the others' errors
            within(o["y"][2:3], ref["y"][2:3], off_by["y"][2:3], True, "large row")
    if ranks:                                        # accumulated on what is there, without dx
        before = {k: o[k].clone() for k in ("dA", "dB")}
        o["dx"].fill_(7)
        bd.lobra_mlora_quant_bwd(plan, *w, d["dy"], None, o["dx"], o["dA"], o["dB"], bd.FLAG_ACCUMULATE_GRADS | bd.FLAG_NO_DX, ws2)
        torch.cuda.synchronize()
        assert bool((o["dx"] == 7).all())
        for k in ("dA", "dB"):
            assert torch.allclose(o[k], 2 * before[k], rtol=1e-5, atol=2e-6 * float(ref[k].abs().max()))


@pytest.mark.gpu
def test_tokens_in_whole_numbers():
    """Rows of halves, of one value, of nothing, and of numbers that are none, seen through a base that passes a channel each on."""
    T, d = 130, 256
    g = torch.Generator().manual_seed(5)
    x = torch.randint(-63, 63, (T, d), generator=g) + 0.5
    x[:, 0] = 127.0
    x[1], x[2], x[3, 17], x[4, 250], x[5] = 0, -3.0, math.nan, -math.inf, 1e-38
    x[6:40] = torch.randn(34, d, generator=g)
    x = x.bfloat16()
    W = torch.eye(d).bfloat16().to(DEV) * 127        # a scale of 1 per channel
    wq, ws = weight(None, W, d, d)
    plan = bd.Plan("bf16", T, d, d, None, [0, T], [-1])
    y = torch.empty(T, d, dtype=torch.bfloat16, device=DEV)
    wsb = torch.empty(bd.lobra_mlora_quant_workspace_bytes(plan)[0], dtype=torch.uint8, device=DEV)
    bd.lobra_mlora_quant_fwd(plan, x.to(DEV), wq, ws, None, None, None, y, None, wsb)
    q, scale = quantised(x)
    # (fp32 in between: whole numbers times two scales, two roundings, then one to bf16, which may fall on the other side of a half)
    ref = (q * 127).float() * scale.float()
    got, want = y.cpu().double(), ref.bfloat16().double()
    same = (got == want) | (torch.isnan(got) & torch.isnan(want)) | ((got - ref.double()).abs() <= HALF * (1 + 2.0 ** -14) * ref.double().abs())
    assert bool(same.all())
    assert bool(torch.isnan(got[3]).all()) and bool(torch.isnan(got[4]).all()) and not bool(torch.isnan(got[5:]).any())
    # the whole numbers themselves: what is printed is nearer to them than to their neighbours
    back = torch.round(got[6:] / (127 * scale[6:]))
    assert float((back - q[6:]).abs().max()) <= 0.5 * 127 * HALF + 0.5


@pytest.mark.gpu
def test_sums_of_the_longest_rows():
    """127 x 127 over the longest row that is taken: sums next to the end of 32 bits."""
    T, d, f = 3, bd.MAX_QUANT_IN, 64
    x, W = torch.ones(T, d, dtype=torch.bfloat16), torch.ones(d, f, dtype=torch.bfloat16)
    x[1] = -1
    W[:, 1] = -1
    x[2, ::2] = -1
    wq, ws = weight(None, W.to(DEV), d, f)
    plan = bd.Plan("bf16", T, d, f, None, [0, T], [-1])
    y = torch.empty(T, f, dtype=torch.bfloat16, device=DEV)
    wsb = torch.empty(bd.lobra_mlora_quant_workspace_bytes(plan)[0], dtype=torch.uint8, device=DEV)
    bd.lobra_mlora_quant_fwd(plan, x.to(DEV), wq, ws, None, None, None, y, None, wsb)
    ref = x.double() @ W.double()
    assert bool(((y.cpu().double() - ref).abs() <= HALF * ref.abs()).all())


@pytest.mark.gpu
@pytest.mark.parametrize("T", [40, 300, 4500])
def test_what_is_not_finite_stays_where_it_is(T):
    d, f = 512, 1024
    v, off, task, rank_off = make(T, d, f, [8, 16, 8], "mixed" if T > 40 else "tokens")
    of = torch.from_numpy(np.repeat(np.asarray(task), np.diff(np.asarray(off))))
    v["A"][rank_off[1]:rank_off[2]] = math.nan       # another task's adapter
    v["x"][T // 3, 100] = math.inf
    v["W"][5, 9] = math.nan
    plan = bd.Plan("bf16", T, d, f, rank_off, off, task)
    dv = on_device(v)
    wq, ws = weight(None, dv["W"], d, f)
    y = torch.empty(T, f, dtype=torch.bfloat16, device=DEV)
    wsb = torch.empty(bd.lobra_mlora_quant_workspace_bytes(plan)[0], dtype=torch.uint8, device=DEV)
    bd.lobra_mlora_quant_fwd(plan, dv["x"], wq, ws, dv["A"], dv["B"], dv["s"], y, None, wsb)
    nan = torch.isnan(y.cpu())
    want = (of == 1)[:, None].expand(T, f).clone()
    want[T // 3] = True
    want[:, 9] = True
    assert torch.equal(nan, want)


@pytest.mark.gpu
def test_gradients_against_differences():
    """Of the adapters; x enters the base rounded, so its gradient is that of the layer on Ŵ with x as it is."""
    T, d, f = 37, 64, 72
    v, off, task, rank_off = make(T, d, f, [8, 16], "mixed", seed=3)
    plan = bd.Plan("bf16", T, d, f, rank_off, off, task)
    dv = on_device(v)
    wq, ws = weight(None, dv["W"], d, f)
    wsb = torch.empty(max(bd.lobra_mlora_quant_workspace_bytes(plan)), dtype=torch.uint8, device=DEV)
    y, dx = torch.empty(T, f, dtype=torch.bfloat16, device=DEV), torch.empty(T, d, dtype=torch.bfloat16, device=DEV)
    dA, dB = torch.empty(24, d, device=DEV), torch.empty(24, f, device=DEV)
    bd.lobra_mlora_quant_bwd(plan, dv["x"], wq, ws, dv["A"], dv["B"], dv["s"], dv["dy"], None, dx, dA, dB, 0, wsb)

    def loss(A, B):
        bd.lobra_mlora_quant_fwd(plan, dv["x"], wq, ws, A, B, dv["s"], y, None, wsb)
        return (y.double() * dv["dy"].double()).cpu()

    g = torch.Generator().manual_seed(1)
    for name, grad in (("A", dA), ("B", dB)):
        step = torch.randn(dv[name].shape, generator=g).to(DEV) * 0.5
        up, down = (dict(A=dv["A"], B=dv["B"], **{}) for _ in range(2))
        up[name], down[name] = (dv[name] + step).bfloat16(), (dv[name] - step).bfloat16()
        moved = (up[name].double() - down[name].double())
        a, b = loss(up["A"], up["B"]), loss(down["A"], down["B"])
        # bilinear: the difference is exact but for roundings: both y, and the projections inside (random in sign: four times their root mean square)
        noise = 4 * HALF * math.sqrt(float((a ** 2).sum() + (b ** 2).sum()))
        assert abs(float((a - b).sum()) - float((grad.double() * moved).sum())) <= 2 * noise
    x = dv["x"].double().cpu()
    ref = reference(v, off, task, rank_off, 1)
    assert float((dx.double().cpu() - ref[0]["dx"]).norm() / ref[0]["dx"].norm()) < HALF


@pytest.mark.gpu
@pytest.mark.parametrize("T,d_in,d_out", [(40, 1024, 520), (300, 512, 264), (2304, 512, 1024)])
def test_on_another_stream_and_in_a_graph(T, d_in, d_out):
    v, off, task, rank_off = make(T, d_in, d_out, [16, 8], "mixed")
    d = on_device(v)
    wq, ws = weight(None, d["W"], d_in, d_out)
    plan = bd.Plan("bf16", T, d_in, d_out, rank_off, off, task)
    wsb = torch.empty(max(bd.lobra_mlora_quant_workspace_bytes(plan)), dtype=torch.uint8, device=DEV)
    h = torch.empty(plan.h_save_bytes, dtype=torch.uint8, device=DEV)

    def outputs():
        return dict(y=torch.zeros(T, d_out, dtype=torch.bfloat16, device=DEV), dx=torch.zeros(T, d_in, dtype=torch.bfloat16, device=DEV),
                    dA=torch.zeros(24, d_in, device=DEV), dB=torch.zeros(24, d_out, device=DEV))

    def go(o):
        w = (d["x"], wq, ws, d["A"], d["B"], d["s"])
        bd.lobra_mlora_quant_fwd(plan, *w, o["y"], h, wsb)
        bd.lobra_mlora_quant_bwd(plan, *w, d["dy"], h, o["dx"], o["dA"], o["dB"], 0, wsb)

    eager, other, graphed = outputs(), outputs(), outputs()
    go(eager)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        go(other)
    torch.cuda.synchronize()
    assert all(torch.equal(eager[k], other[k]) for k in eager)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        go(graphed)
    for r in range(3):
        d["x"].mul_(0.5 if r else 1.0)
        graph.replay()
        torch.cuda.synchronize()
        go(eager)
        torch.cuda.synchronize()
        assert all(torch.equal(eager[k], graphed[k]) for k in eager), r


@pytest.mark.gpu
def test_of_no_tokens():
    plan = bd.Plan("bf16", 0, 64, 72, [0, 8], [0], [])
    dA, dB = torch.ones(8, 64, device=DEV), torch.ones(8, 72, device=DEV)
    assert bd.lobra_mlora_quant_workspace_bytes(plan)[0] == 0
    bd.lobra_mlora_quant_fwd(plan, None, None, None, None, None, None, None)
    ws = torch.empty(max(bd.lobra_mlora_quant_workspace_bytes(plan)[1], 16), dtype=torch.uint8, device=DEV)
    bd.lobra_mlora_quant_bwd(plan, None, None, None, None, None, None, None, None, None, dA, dB, bd.FLAG_ACCUMULATE_GRADS, ws)
    assert bool((dA == 1).all()) and bool((dB == 1).all())
    bd.lobra_mlora_quant_bwd(plan, None, None, None, None, None, None, None, None, None, dA, dB, 0, ws)
    assert not bool(dA.any()) and not bool(dB.any())


def test_weight_refusals():
    L, p = bd.lib(), 4096
    call = lambda dt=bd.BF16, k=64, n=64, ld=0, W=p, q=p, s=p: L.lobra_quantise_weight(dt, k, n, ld, W, q, s, None)
    assert call(dt=2) == -3 and call(k=0) == -2 and call(k=bd.MAX_QUANT_IN + 1) == -2 and call(n=0) == -2 and call(n=(1 << 20) + 1) == -2 and call(ld=63) == -2
    assert call(ld=1 << 40) == -2
    assert call(W=None) == -1 and call(q=None) == -1 and call(s=None) == -1
    assert call(W=p + 2) == -8 and call(q=p + 8) == -8 and call(s=p + 4) == -8
    assert [bd.lobra_quant_pitch(k) for k in (-1, 0, 1, 256, 257, 1 << 17)] == [0, 0, 256, 256, 512, 1 << 17]
    W, q, s = torch.zeros(8, 16), torch.zeros(16, 256, dtype=torch.int8), torch.zeros(16)
    for bad in (dict(W=W.double()), dict(W=W.half()), dict(W=W.t()), dict(Wq=q.float()), dict(Wq=q[:15]), dict(Wq=q[:, :128]), dict(w_scale=s[:15]), dict(w_scale=s.double())):
        with pytest.raises(AssertionError):
            bd.lobra_quantise_weight(**{**dict(W=W, Wq=q, w_scale=s), **bad}, stream=0)


def test_plans_that_do_not_run_it():
    L, n = bd.lib(), ctypes.c_size_t()
    for args, flags, want in ((("f32", 8, 64, 64), 0, -3), (("bf16", 8, 64, 64), bd.PLAN_PLAIN_KERNELS, -3), (("bf16", 8, bd.MAX_QUANT_IN + 8, 64), 0, -2), (("bf16", 8, 64, 64), 0, 0)):
        plan = bd.Plan(*args, [0, 8], [0, 8], [0], flags=flags | bd.PLAN_HOST_ONLY)
        assert L.lobra_mlora_quant_workspace_bytes(plan.handle, ctypes.byref(n), None) == want
        assert L.lobra_mlora_quant_workspace_bytes(plan.handle, None, ctypes.byref(n)) == want
    p = 4096
    assert L.lobra_mlora_quant_fwd(plan.handle, *[p] * 7, None, p, 1 << 20, None) == -10         # (host only)
    assert L.lobra_mlora_quant_workspace_bytes(None, ctypes.byref(n), None) == -10
    assert L.lobra_mlora_quant_fwd(None, *[p] * 7, None, p, 1 << 20, None) == -10
    assert L.lobra_mlora_quant_bwd(None, *[p] * 11, 0, p, 1 << 20, None) == -10
    x = torch.zeros(8, 64).bfloat16()
    q, s, f = torch.zeros(64, 256, dtype=torch.int8), torch.zeros(64), torch.zeros(8, 64)
    ok = dict(x=x, Wq=q, w_scale=s, A=x, B=x, s=s, y=x, ws=None, stream=0, check=False)
    assert bd.lobra_mlora_quant_fwd(plan, **ok) == -10
    for bad in (dict(x=f), dict(x=x[:7]), dict(Wq=q.view(torch.uint8)), dict(Wq=q[:63]), dict(w_scale=s[:63]), dict(A=f), dict(B=f), dict(y=f), dict(y=x[:7]), dict(s=s.double())):
        with pytest.raises(AssertionError):
            bd.lobra_mlora_quant_fwd(plan, **{**ok, **bad})
    okb = dict(x=x, Wq=q, w_scale=s, A=x, B=x, s=s, dy=x, h_saved=None, dx=x, dA=f, dB=f, stream=0, check=False)
    assert bd.lobra_mlora_quant_bwd(plan, **okb) == -10
    for bad in (dict(dy=f), dict(dy=x[:7]), dict(dx=f), dict(dx=x[:7]), dict(dA=x), dict(dB=x), dict(Wq=q[:63])):
        with pytest.raises(AssertionError):
            bd.lobra_mlora_quant_bwd(plan, **{**okb, **bad})


@pytest.mark.gpu
def test_refusals():
    T, d, f = 40, 64, 72
    v, off, task, rank_off = make(T, d, f, [8], "one")
    dv = on_device(v)
    wq, ws = weight(None, dv["W"], d, f)
    plan = bd.Plan("bf16", T, d, f, rank_off, off, task)
    fwd, bwd = bd.lobra_mlora_quant_workspace_bytes(plan)
    y, dx = torch.empty(T, f, dtype=torch.bfloat16, device=DEV), torch.empty(T, d, dtype=torch.bfloat16, device=DEV)
    wsf, wsb = torch.empty(fwd, dtype=torch.uint8, device=DEV), torch.empty(bwd, dtype=torch.uint8, device=DEV)
    dA, dB = torch.empty(8, d, device=DEV), torch.empty(8, f, device=DEV)
    base = dict(x=dv["x"], Wq=wq, w_scale=ws, A=dv["A"], B=dv["B"], s=dv["s"])
    F = lambda **kw: bd.lobra_mlora_quant_fwd(plan, **{**base, **dict(y=y, ws=wsf), **kw}, check=False)
    B = lambda **kw: bd.lobra_mlora_quant_bwd(plan, **{**base, **dict(dy=dv["dy"], h_saved=None, dx=dx, dA=dA, dB=dB, ws=wsb), **kw}, check=False)
    assert F() == 0 and B() == 0
    for k in base:
        assert F(**{k: None}) == -1 and B(**{k: None}) == -1
    assert F(y=None) == -1 and B(dy=None) == -1 and B(dx=None) == -1 and B(dA=None) == -1
    assert F(ws=None) == -7 and F(ws=wsf[:fwd - 1]) == -7 and B(ws=None) == -7 and B(ws=wsb[:bwd - 1]) == -7
    off16 = torch.empty(max(fwd, bwd) + 16, dtype=torch.uint8, device=DEV)[8:]
    assert F(ws=off16) == -8 and B(ws=off16) == -8
    torch.cuda.synchronize()


@pytest.mark.gpu
def test_more_rows_than_a_launch_holds():
    """Rows behind the first 2^22, which is where a second launch quantises them."""
    T, d, f = (1 << 22) + 5, 8, 8
    g = torch.Generator(device=DEV).manual_seed(1)
    x = torch.randn(T, d, device=DEV, generator=g).bfloat16()
    W = torch.randn(d, f, device=DEV, generator=g).bfloat16()
    wq, ws = weight(None, W, d, f)
    plan = bd.Plan("bf16", T, d, f, None, [0, T], [-1])
    y = torch.empty(T, f, dtype=torch.bfloat16, device=DEV)
    wsb = torch.empty(bd.lobra_mlora_quant_workspace_bytes(plan)[0], dtype=torch.uint8, device=DEV)
    bd.lobra_mlora_quant_fwd(plan, x, wq, ws, None, None, None, y, None, wsb)
    rows = torch.cat([torch.arange(100), torch.arange((1 << 22) - 50, T)])
    v = dict(x=x.cpu()[rows], W=W.cpu(), A=torch.zeros(0, d), B=torch.zeros(0, f), s=torch.ones(1), dy=torch.zeros(len(rows), f))
    ref, off, _, _ = reference(v, [0, len(rows)], [-1], [0], 1)
    within(y.cpu()[rows], ref["y"], off["y"], True, "y")


@pytest.mark.gpu
@pytest.mark.parametrize("T,std_x,std_w", [(40, 1e30, 1e-30), (700, 1e33, 1e-30), (700, 1e-30, 1e4)])
def test_scales_far_apart(T, std_x, std_w):
    """Tokens and channels whose scales only together are of ordinary size."""
    d, f = 512, 264
    v, off, task, rank_off = make(T, d, f, [], "one")
    v["x"], v["W"] = (v["x"].double() * std_x).bfloat16(), (v["W"].double() * std_w).bfloat16()
    ref, off_by, _, _ = reference(v, off, task, rank_off, 1)
    dv = on_device(v)
    wq, ws = weight(None, dv["W"], d, f)
    plan = bd.Plan("bf16", T, d, f, None, off, task)
    y = torch.empty(T, f, dtype=torch.bfloat16, device=DEV)
    wsb = torch.empty(bd.lobra_mlora_quant_workspace_bytes(plan)[0], dtype=torch.uint8, device=DEV)
    bd.lobra_mlora_quant_fwd(plan, dv["x"], wq, ws, None, None, None, y, None, wsb)
    within(y, ref["y"], off_by["y"], True, "y")


@pytest.mark.gpu
@pytest.mark.parametrize("T,d_in,d_out,ranks,batch,n_proj", [
    (1, 264, 8, [4], "one", 1), (16, 520, 1032, [16, 8, 3], "tokens", 1), (17, 9000, 264, [16, 8], "tokens", 1), (31, 1376, 4096, [32, 5], "mixed", 1),
    (48, 4096, 72, [8, 16, 1, 32], "tokens", 1), (48, 256, 4096, [16], "bare", 1), (33, 768, 1536, [8], "tokens", 3), (48, 512, 2064, [16, 8], "mixed", 2),
    (64, 512, 264, [16, 8], "tokens", 1), (65, 512, 264, [16, 8], "tokens", 1), (64, 1024, 4096, [16], "bare", 1), (16, 512, 8192, [16, 8], "tokens", 1),
    (17, 512, 4104, [16, 8], "tokens", 1), (16, 264, 8200, [16, 8], "tokens", 1), (15, 2304, 6144, [8], "tokens", 3), (50, 264, 1032, [32, 8], "tokens", 1),
    (49, 512, 264, [16, 8], "tokens", 1), (48, 512, 4104, [16, 8], "tokens", 1), (48, 512, 264, [33, 8], "tokens", 1), (40, 512, 520, [], "tokens", 1),
])
def test_few_tokens(T, d_in, d_out, ranks, batch, n_proj):
    """On both sides of what the kernels for few tokens take; forward with and without what backward starts from."""
    test_layer(T, d_in, d_out, ranks, batch, n_proj)


def test_host_tensors_and_short_ones():
    with pytest.raises(AssertionError, match="host tensor"):
        bd.lobra_quantise_weight(torch.zeros(8, 16), torch.zeros(16, 256, dtype=torch.int8), torch.zeros(16), stream=0)
    plan = bd.Plan("bf16", 8, 64, 64, [0, 8, 24], [0, 4, 8], [0, 1], flags=bd.PLAN_HOST_ONLY)
    x, a, q, s, f = torch.zeros(8, 64).bfloat16(), torch.zeros(24, 64).bfloat16(), torch.zeros(64, 256, dtype=torch.int8), torch.zeros(64), torch.zeros(24, 64)
    fwd = dict(x=x, Wq=q, w_scale=s, A=a, B=a, s=s[:2], y=x, stream=0, check=False)
    bwd = dict(x=x, Wq=q, w_scale=s, A=a, B=a, s=s[:2], dy=x, h_saved=None, dx=x, dA=f, dB=f, stream=0, check=False)
    assert bd.lobra_mlora_quant_fwd(plan, **fwd) == -10 and bd.lobra_mlora_quant_bwd(plan, **bwd) == -10
    short = torch.zeros(plan.h_save_bytes - 1, dtype=torch.uint8)
    for bad in (dict(A=a[:23]), dict(B=a[:23]), dict(s=s[:1]), dict(h_save=short)):
        with pytest.raises(AssertionError):
            bd.lobra_mlora_quant_fwd(plan, **{**fwd, **bad})
    for bad in (dict(dA=f[:23]), dict(dB=f[:23]), dict(A=a[:23]), dict(s=s[:1]), dict(h_saved=short)):
        with pytest.raises(AssertionError):
            bd.lobra_mlora_quant_bwd(plan, **{**bwd, **bad})


@pytest.mark.gpu
def test_no_tokens():
    """Nothing is read; the gradients are those of nothing."""
    plan = bd.Plan("bf16", 0, 64, 72, [0, 8], [0], [])
    fwd, bwd = bd.lobra_mlora_quant_workspace_bytes(plan)
    assert fwd == 0
    dA, dB = torch.full((8, 64), 7.0, device=DEV), torch.full((8, 72), 7.0, device=DEV)
    W = torch.randn(64, 72, device=DEV).bfloat16()
    wq, ws = weight(None, W, 64, 72)
    A, B, s = torch.ones(8, 64, device=DEV).bfloat16(), torch.ones(8, 72, device=DEV).bfloat16(), torch.ones(1, device=DEV)
    e = torch.empty(0, 64, device=DEV).bfloat16()
    bd.lobra_mlora_quant_fwd(plan, e, wq, ws, A, B, s, torch.empty(0, 72, device=DEV).bfloat16())
    bd.lobra_mlora_quant_bwd(plan, e, wq, ws, A, B, s, torch.empty(0, 72, device=DEV).bfloat16(), None, e, dA, dB, 0, torch.empty(max(bwd, 16), dtype=torch.uint8, device=DEV))
    torch.cuda.synchronize()
    assert bool((dA == 0).all()) and bool((dB == 0).all())


def test_weights_whose_rows_overlap_are_refused():
    """A row pitch below a row's length (a broadcast row has 0, which the library takes for rows back to back) would be read as d_in rows that are not there."""
    q, s = torch.zeros(16, 256, dtype=torch.int8), torch.zeros(16)
    for W in (torch.zeros(16).expand(8, 16), torch.zeros(1, 16).bfloat16().expand(8, 16), torch.zeros(64).as_strided((8, 16), (4, 1)), torch.zeros(1).expand(8, 16)):
        with pytest.raises(AssertionError, match="rows of a weight"):
            bd.lobra_quantise_weight(W, q, s, stream=0)
    with pytest.raises(AssertionError, match="host tensor"):          # (a single row has no pitch)
        bd.lobra_quantise_weight(torch.zeros(16).expand(1, 16), q, s, stream=0)


@pytest.mark.gpu
@pytest.mark.parametrize("T,d,f,ranks,n_proj", [
    (40, 512, 264, [], 1), (40, 512, 264, [8], 1), (100, 1024, 264, [8], 1), (200, 512, 512, [8], 2), (300, 512, 128, [], 1), (700, 512, 264, [8], 1), (1500, 768, 1032, [], 1),
    (4500, 512, 1024, [8], 1),
])
def test_scales_of_every_size(T, d, f, ranks, n_proj):
    """Channels and tokens between 1e-34 and 1e37 side by side: where a product of both is an ordinary number it is that number, whatever lies on the way to it."""
    v, off, task, rank_off = make(T, d, f, ranks, "one", n_proj)
    tokens, channels = (1e-34, 1.0, 1e30, 1e-20), (1e37, 1.0, 1e-30, 1e33, 1e20)
    v["x"] = (v["x"].double() * torch.tensor(tokens)[torch.arange(T) % len(tokens)][:, None].double()).bfloat16()
    v["W"] = (v["W"].double() * torch.tensor(channels)[torch.arange(f) % len(channels)].double()).bfloat16()
    v["A"].zero_()
    q, xs = quantised(v["x"])
    wq, wsc = quantised(v["W"].t())
    ref = (q @ wq.t()) * xs * wsc[:, 0]
    dv = on_device(v)
    Wq, ws = weight(None, dv["W"], d, f)
    plan = bd.Plan("bf16", T, d, f, rank_off if ranks else None, off, task, n_proj=n_proj)
    fwd, _ = bd.lobra_mlora_quant_workspace_bytes(plan)
    wsb, h = torch.empty(fwd, dtype=torch.uint8, device=DEV), torch.empty(max(plan.h_save_bytes, 16), dtype=torch.uint8, device=DEV)
    top = torch.finfo(torch.bfloat16).max
    for kept in (None, h):
        y = torch.empty(T, f, dtype=torch.bfloat16, device=DEV)
        bd.lobra_mlora_quant_fwd(plan, dv["x"], Wq, ws, *((dv["A"], dv["B"], dv["s"]) if ranks else (None,) * 3), y, kept, wsb)
        got = y.double().cpu()
        # whole sums, three roundings of 2^-24 (six where splits of a sum are added), one to bf16; below the normal numbers nothing is promised
        good = (got - ref).abs() <= HALF * (1 + 2.0 ** -12) * ref.abs() + 2.0 ** -126
        split = (got - ref).abs() <= HALF * ref.abs() + 2e-6 * ((q.abs() @ wq.abs().t()) * xs * wsc[:, 0]) + 2.0 ** -126
        large = ref.abs() > top * (1 - HALF)
        good = torch.where(large, (got * ref.sign() >= top * (1 - HALF)), good | split)
        assert bool(good.all()), (int((~good).sum()), good.numel(), got[~good][:4].tolist(), ref[~good][:4].tolist())
        assert int(large.sum()) > 0 and int(((ref.abs() > 1) & ~large).sum()) > T * f // 10


@pytest.mark.gpu
@pytest.mark.parametrize("T,d,f,ranks,n_proj", [(40, 512, 264, [8], 1), (300, 640, 768, [16, 8], 2), (2600, 1032, 520, [16, 8], 1), (64, 256, 264, [], 1)])
def test_backward_without_dx_needs_no_room_for_the_weight(T, d, f, ranks, n_proj):
    v, off, task, rank_off = make(T, d, f, ranks, "mixed" if ranks else "one", n_proj)
    dv = on_device(v)
    wq, ws = weight(None, dv["W"], d, f)
    plan = bd.Plan("bf16", T, d, f, rank_off if ranks else None, off, task, n_proj=n_proj)
    ad = (dv["A"], dv["B"], dv["s"]) if ranks else (None,) * 3
    full = torch.empty(bd.lobra_mlora_quant_workspace_bytes(plan)[1], dtype=torch.uint8, device=DEV)
    own, ok = guarded(max(plan.bwd_ws_bytes, 16), dtype=torch.uint8)
    R = sum(ranks) * n_proj
    G = [[torch.full(s, 5.0, device=DEV) for s in ((R, d), (R, f // n_proj))] if ranks else [None, None] for _ in range(2)]
    bd.lobra_mlora_quant_bwd(plan, dv["x"], wq, ws, *ad, dv["dy"], None, torch.empty(T, d, device=DEV, dtype=torch.bfloat16), *G[0], 0, full)
    bd.lobra_mlora_quant_bwd(plan, dv["x"], wq, ws, *ad, dv["dy"], None, None, *G[1], bd.FLAG_NO_DX, own if ranks else None)
    torch.cuda.synchronize()
    assert ok()
    if ranks:
        for a, b in zip(*G):                         # (with dx the projection of dy may run in the product's launch: another order of sums)
            assert torch.allclose(a, b, rtol=2 * HALF, atol=2 * HALF * float(a.abs().max()))
        call = lambda n: bd.lobra_mlora_quant_bwd(plan, dv["x"], wq, ws, *ad, dv["dy"], None, None, *G[1], bd.FLAG_NO_DX, own[:n], check=False)
        assert call(0) == -7 and bd.lobra_mlora_quant_bwd(plan, dv["x"], None, ws, *ad, dv["dy"], None, None, *G[1], bd.FLAG_NO_DX, own, check=False) == -1
