"""The steps of joint fine-tuning around the LoRA linears, as measurable cases: plain, through the library, and in 64 bits.

A case is a plain dict.  Its `kind` says which operator one pass goes through:

  score     log probability of a given token per row of logits, entropy and the likeliest alternatives (serving, evaluation):
            lobra_token_logprob_fwd
  loss      the same without alternatives, then the gradient of the logits (training): lobra_token_logprob_fwd, _bwd
  clip      the norm of every task's gradient over all layers' dA and dB, the factor that clips it, and, with `out`, the
            clipped gradients: lobra_grad_clip
  norm      the end of one residual block and the start of the next: the block's output normed, gated by its token's task,
            scaled and added to the residual, the sum normed: lobra_mlora_block_norm_fwd, with `back` also _bwd
  gated     the gated feed-forward block's up side: gate and up projection with their adapters, activation, product:
            lobra_mlora_gated_fwd, with `back` also _bwd

`own` says who computes: False - elementary torch operations in 32 bits; True - the library.  Widths are those of the layers
that the library's other cases have (4096 and 11008, 8192 and 28672, 11008 / 8 = 1376) or generic.
"""
import math
import random

import numpy as np
import torch

own = False

DEV = "cuda:0"


def listed():
    return [
        # one new token for each of 40 requests: its log probability and 20 alternatives, as a serving interface reports them
        dict(name="score_decode", kind="score", dtype="bf16", T=40, V=32000, top_k=20, masked=0.0),
        # an evaluation batch over a large vocabulary, a tenth of it barred (padding, tokens that may not be sampled)
        dict(name="score_eval", kind="score", dtype="bf16", T=4096, V=128000, top_k=8, masked=0.1),
        # the loss of a packed training batch, prompts and pads without a target (a third of the tokens)
        dict(name="loss_8k", kind="loss", dtype="bf16", T=8190, V=32000, bare=0.33, entropy=False),
        # fp32 logits of an odd vocabulary, rows aligned to nothing, with an entropy bonus in the loss
        dict(name="loss_f32_odd", kind="loss", dtype="f32", T=1000, V=50257, bare=0.1, entropy=True),
        # the optimizer's view of one fused layer of a 7B model, clipped gradients written out
        dict(name="clip_layer", kind="clip", layers="4096:4096", repeat=1, tasks=4, ranks="16", out=True),
        # all seven linears of the 32 layers of a 7B model, four tasks of rank 16: the factors go to the Adam step
        dict(name="clip_7b", kind="clip", layers="4096:4096,4096:4096,4096:4096,4096:4096,4096:11008,4096:11008,11008:4096",
             repeat=32, tasks=4, ranks="16", out=False),
        # decoding: 40 one-token requests to eight tasks between two blocks
        dict(name="norm_decode", kind="norm", dtype="bf16", T=40, d=4096, tasks=8, mean_len=1, bare=0.1, post=True, gate=True,
             back=False),
        # a packed training batch between two blocks of a 7B model
        dict(name="norm_16k", kind="norm", dtype="bf16", T=16384, d=4096, tasks=4, mean_len=400, bare=0.0, post=True, gate=True,
             back=True),
        # an fp32 model of odd width
        dict(name="norm_f32_odd", kind="norm", dtype="f32", T=2999, d=1025, tasks=3, mean_len=70, bare=0.1, post=True, gate=True,
             back=True),
        # decoding through the gated block of a 7B model
        dict(name="gated_decode", kind="gated", dtype="bf16", act="silu", T=40, d_in=4096, f=11008, tasks=8, ranks="16", mean_len=1,
             bare=0.1, back=False),
        # training: the gated block of a 7B model on 16384 packed tokens, the largest here
        dict(name="gated_16k", kind="gated", dtype="bf16", act="silu", T=16384, d_in=4096, f=11008, tasks=4, ranks="16", mean_len=400,
             bare=0.0, back=True),
        # one of eight tensor-parallel shards of it, an odd number of tokens, some of no task, mixed ranks
        dict(name="gated_shard", kind="gated", dtype="bf16", act="gelu", T=8190, d_in=4096, f=1376, tasks=6, ranks="8,16,32", mean_len=300,
             bare=0.1, back=True),
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm."""
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return n + int(n == 24 * 128)            # (a size of no layer here)


def _width(rng, lo, hi):
    """A bf16 layer width: mostly whole multiples of 128 as models have them, else any multiple of 8."""
    w = _spread(rng, lo, hi)
    m = rng.choice([128, 128, 256, 32, 8])
    w = max(m, w // m * m)
    return w + m * int(w == 24 * 128)


def draw(rng):
    kind = rng.choice(["score", "score", "loss", "loss", "clip", "norm", "norm", "gated", "gated", "gated"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    tasks = rng.choice([1, 2, 4, 8, 16])
    if kind in ("score", "loss"):
        V = _spread(rng, 1000, 131072)
        if rng.random() < 0.6:
            V = V // 64 * 64 + 64
            V += 64 * int(V == 24 * 128)
        most = (250 if dtype == "f32" else 500) * 10**6 // V
        T = min(_spread(rng, 1, 16384), most)
        if kind == "score":
            return dict(kind=kind, dtype=dtype, T=T, V=V, top_k=rng.choice([0, 1, 5, 20, 32]), masked=rng.choice([0.0, 0.1, 0.9]))
        return dict(kind=kind, dtype=dtype, T=T, V=V, bare=rng.choice([0.0, 0.33, 0.8]), entropy=rng.random() < 0.4)
    if kind == "clip":
        d, f = _width(rng, 256, 4096), _width(rng, 512, 11008)
        layers = rng.choice(["%d:%d" % (d, d), "%d:%d,%d:%d" % (d, f, f, d), "%d:%d,%d:%d,%d:%d" % (d, d, d, f, f, d)])
        return dict(kind=kind, layers=layers, repeat=_spread(rng, 1, 32), tasks=min(tasks, 8), ranks=rng.choice(["8", "16", "4,8,16", "3,7"]),
                    out=rng.random() < 0.5)
    if kind == "norm":
        d = _spread(rng, 64, 8192)
        if dtype == "bf16":
            d = max(64, d // 8 * 8) if rng.random() < 0.3 else _width(rng, 128, 8192)
        T = min(_spread(rng, 1, 16384), 1000 * 66000 // d)
        return dict(kind=kind, dtype=dtype, T=T, d=d, tasks=tasks, mean_len=1 if T < 100 else _spread(rng, 30, 1500),
                    bare=rng.choice([0.0, 0.1]), post=rng.random() < 0.6, gate=rng.random() < 0.6, back=T >= 100 and rng.random() < 0.7)
    if dtype == "f32":
        T, d, f = _spread(rng, 1, 3000), _spread(rng, 96, 1024), _width(rng, 96, 2048)
    else:
        T, d, f = _spread(rng, 1, 16384), _width(rng, 256, 4096), _width(rng, 512, 8192)
    return dict(kind=kind, dtype=dtype, act=rng.choice(["silu", "silu", "gelu"]), T=T, d_in=d, f=f, tasks=tasks,
                ranks=rng.choice(["8", "16", "16", "32", "8,16,64"]), mean_len=1 if T < 100 else _spread(rng, 30, 1500),
                bare=rng.choice([0.0, 0.1]), back=T >= 100 and rng.random() < 0.7)


# ------------------------------------------------------------------------------------------------------------------
# inputs
# ------------------------------------------------------------------------------------------------------------------
def _ranks(case):
    r = [int(v) for v in str(case["ranks"]).split(",")]
    return [r[t % len(r)] for t in range(case["tasks"])]


def _table(case):
    """The packed batch: sequences with right-skewed lengths in random order, each of some task (-1: none)."""
    rng = random.Random("%(T)d %(tasks)d %(mean_len)d %(bare)s" % case)
    off, task = [0], []
    while off[-1] < case["T"]:
        n = int(round(case["mean_len"] * math.exp(rng.gauss(-0.5, 1.0)))) if case["mean_len"] > 1 else 1
        off.append(off[-1] + min(max(n, 1), case["T"] - off[-1]))
        task.append(-1 if rng.random() < case["bare"] else rng.randrange(case["tasks"]))
    return off, task


def _dtype(case):
    return torch.float32 if case.get("dtype") == "f32" else torch.bfloat16


def _shapes(case):
    """clip: (rows, width) of every gradient, A then B of each layer."""
    R = sum(_ranks(case))
    per = [tuple(int(v) for v in pair.split(":")) for pair in case["layers"].split(",")]
    return [(R, w) for _ in range(case["repeat"]) for pair in per for w in pair]


def _inputs(case, seed):
    g = torch.Generator(device=DEV).manual_seed(int(seed))
    dt = _dtype(case)

    def normal(std, *shape, dtype=dt):
        return torch.randn(*shape, device=DEV, dtype=dtype, generator=g).mul_(std)

    def uniform(*shape):
        return torch.rand(*shape, device=DEV, generator=g)

    kind = case["kind"]
    if kind in ("score", "loss"):
        T, V = case["T"], case["V"]
        # logits as a trained head gives them: a spread of a few units, the target usually among the likely ones
        v = dict(logits=normal(2.5, T, V))
        target = torch.randint(0, V, (T,), device=DEV, generator=g)
        rows = torch.arange(T, device=DEV)
        v["logits"][rows, target] += (uniform(T) * 16).to(dt)
        if kind == "score":
            if case["masked"]:
                # the same columns in every row; the tokens whose probability is asked for are none of them
                barred = uniform(V) < case["masked"]
                barred[0] = False
                v["logits"][:, barred] = float("-inf")
                allowed = (~barred).nonzero().flatten()
                target = allowed[target % len(allowed)]
            v["target"] = target.to(torch.int32)
            return v
        bare = uniform(T) < case["bare"]
        v["target"] = torch.where(bare, torch.full_like(target, -1), target).to(torch.int32)
        # the loss is a mean over the tokens that have a target
        v["dlogp"] = torch.where(bare, torch.zeros(T, device=DEV), -(uniform(T) + 0.5) / T)
        v["dentropy"] = torch.where(bare, torch.zeros(T, device=DEV), -0.01 * (uniform(T) + 0.5) / T) if case["entropy"] else None
        return v
    if kind == "clip":
        n = case["tasks"]
        v = dict(grads=[normal(1e-3, r, d, dtype=torch.float32) for r, d in _shapes(case)], grad_scale=uniform(n) + 0.5)
        elements = sum(r * d for r, d in _shapes(case)) / n
        # about half the tasks are clipped
        v["max_norm"] = 1e-3 * math.sqrt(elements) * (uniform(n) + 0.5)
        v["step"] = torch.randint(1, 500, (n,), device=DEV, generator=g, dtype=torch.int32)
        return v
    if kind == "norm":
        T, d = case["T"], case["d"]
        v = dict(r=normal(2.0, T, d), b=normal(0.7, T, d), w_pre=normal(0.2, d) + 1)
        v["w_post"] = normal(0.2, d) + 1 if case["post"] else None
        v["gate"] = normal(0.3, case["tasks"], d) + 1 if case["gate"] else None
        if case["back"]:
            v["dr_out"], v["dx"] = normal(1.0, T, d), normal(1.0, T, d)
        return v
    T, d, f, R = case["T"], case["d_in"], case["f"], sum(_ranks(case))
    # adapters of both projections, stacked per task; a scale per task
    v = dict(x=normal(1.0, T, d), W=normal(0.02, d, 2 * f), A=normal(0.02, 2 * R, d), B=normal(0.02, 2 * R, f), s=uniform(case["tasks"]) + 0.5)
    if case["back"]:
        v["dh"] = normal(1.0, T, f)
    return v


EPS, ALPHA = 1e-6, 0.5


def prepare(case, seed):
    st = dict(case=dict(case))
    st.update(_inputs(case, seed))
    kind, dt = case["kind"], _dtype(case)

    def empty(*shape, dtype=torch.float32):
        return torch.empty(*shape, dtype=dtype, device=DEV)

    if kind in ("norm", "gated"):
        st["off"], st["task"] = _table(case)
    if kind == "gated":
        st["rank_off"] = np.concatenate([[0], np.cumsum([2 * r for r in _ranks(case)])])
    if kind == "clip":
        st["rank_off"] = np.concatenate([[0], np.cumsum(_ranks(case))])
    if not own:
        # which rows belong to which task, as a program without the library would keep it
        if kind in ("norm", "gated"):
            of = torch.tensor(np.repeat(np.asarray(st["task"]), np.diff(np.asarray(st["off"]))), device=DEV)
            st["of"] = of
            st["rows"] = [(of == t).nonzero().flatten() for t in range(case["tasks"])]
        if kind == "clip":
            st["of"] = torch.tensor(np.repeat(np.arange(case["tasks"]), _ranks(case)), device=DEV)
        return st
    from paper_2509_01193_amd import binding as lobra
    if kind in ("score", "loss"):
        T, V = case["T"], case["V"]
        st["desc"] = lobra.make_logprob_desc(case["dtype"], T, V, top_k=case.get("top_k", 0))
        st.update(logp=empty(T), lse=empty(T), ent=empty(T) if kind == "score" or case["entropy"] else None)
        if kind == "score":
            k = case["top_k"]
            st.update(top_logp=empty(T, k) if k else None, top_id=empty(T, k, dtype=torch.int32) if k else None)
        else:
            st.update(rest=empty(T), dlogits=empty(T, V, dtype=dt))
    elif kind == "clip":
        st["outs"] = [torch.empty_like(g) if case["out"] else None for g in st["grads"]]
        st["set"] = lobra.GradSet([(g, o, st["rank_off"]) for g, o in zip(st["grads"], st["outs"])], case["tasks"])
        st["ws"] = empty(max(st["set"].ws_bytes, 16), dtype=torch.uint8)
        n = case["tasks"]
        st.update(norm=empty(n), scale=empty(n), step_out=empty(n, dtype=torch.int32))
    elif kind == "norm":
        T, d, n = case["T"], case["d"], case["tasks"]
        # the plan of the layer that reads x, which the program has anyway
        st["plan"] = lobra.Plan(case["dtype"], T, d, max(d // 8 * 8, 8), np.arange(n + 1) * 8, st["off"], st["task"])
        st["cfg"] = lobra.BlockNormConfig(EPS, ALPHA)
        st.update(r_out=empty(T, d, dtype=dt), x=empty(T, d, dtype=dt), rstd_post=empty(T) if case["post"] else None, rstd_pre=empty(T))
        if case["back"]:
            st.update(dr=empty(T, d, dtype=dt), db=empty(T, d, dtype=dt), dw_pre=empty(d))
            st.update(dgate=empty(n, d) if case["gate"] else None, dw_post=empty(d) if case["post"] else None)
            st["ws"] = empty(max(lobra.lobra_mlora_block_norm_workspace_bytes(st["plan"]), 16), dtype=torch.uint8)
    else:
        T, d, f = case["T"], case["d_in"], case["f"]
        st["plan"] = lobra.Plan(case["dtype"], T, d, 2 * f, st["rank_off"], st["off"], st["task"], n_proj=2)
        st["code"] = {"silu": lobra.ACT_SILU, "gelu": lobra.ACT_GELU_TANH}[case["act"]]
        st["h"] = empty(T, f, dtype=dt)
        ws = lobra.lobra_mlora_gated_workspace_bytes(st["plan"], save=case["back"])
        if case["back"]:
            st.update(gu=empty(T, 2 * f, dtype=dt), dgu=empty(T, 2 * f, dtype=dt), dx_out=empty(T, d, dtype=dt))
            st.update(dA=torch.empty_like(st["A"], dtype=torch.float32), dB=torch.empty_like(st["B"], dtype=torch.float32))
            st["h_save"] = empty(max(st["plan"].h_save_bytes, 16), dtype=torch.uint8)
            ws = max(ws, st["plan"].bwd_ws_bytes)
        st["ws"] = empty(max(ws, 16), dtype=torch.uint8)
    return st


# ------------------------------------------------------------------------------------------------------------------
# one pass
# ------------------------------------------------------------------------------------------------------------------
def run(st):
    kind = st["case"]["kind"]
    if own:
        return {"score": _own_logprob, "loss": _own_logprob, "clip": _own_clip, "norm": _own_norm, "gated": _own_gated}[kind](st)
    return {"score": _plain_score, "loss": _plain_loss, "clip": _plain_clip, "norm": _plain_norm, "gated": _plain_gated}[kind](st)


def _own_logprob(st):
    from paper_2509_01193_amd import binding as lobra
    if st["case"]["kind"] == "score":
        lobra.lobra_token_logprob_fwd(st["desc"], st["logits"], st["target"], st["logp"], st["lse"], None, st["ent"], st["top_logp"],
                                      st["top_id"])
        out = dict(logp=st["logp"], lse=st["lse"], entropy=st["ent"])
        if st["case"]["top_k"]:
            out.update(top_logp=st["top_logp"], top_id=st["top_id"])
        return out
    lobra.lobra_token_logprob_fwd(st["desc"], st["logits"], st["target"], st["logp"], st["lse"], st["rest"], st["ent"])
    lobra.lobra_token_logprob_bwd(st["desc"], st["logits"], st["target"], st["lse"], st["rest"], st["ent"], st["dlogp"], st["dentropy"],
                                  st["dlogits"])
    out = dict(logp=st["logp"], lse=st["lse"], dlogits=st["dlogits"])
    if st["ent"] is not None:
        out["entropy"] = st["ent"]
    return out


def _own_clip(st):
    from paper_2509_01193_amd import binding as lobra
    lobra.lobra_grad_clip(st["set"], st["max_norm"], st["grad_scale"], st["step"], st["norm"], st["scale"], st["step_out"], ws=st["ws"])
    out = dict(norm=st["norm"], scale=st["scale"], step=st["step_out"])
    if st["case"]["out"]:
        out["clipped"] = st["outs"]
    return out


def _own_norm(st):
    from paper_2509_01193_amd import binding as lobra
    lobra.lobra_mlora_block_norm_fwd(st["plan"], st["cfg"], st["r"], st["b"], st["w_post"], st["gate"], st["w_pre"], st["r_out"], st["x"],
                                     st["rstd_post"], st["rstd_pre"])
    out = dict(r_out=st["r_out"], x=st["x"])
    if st["case"]["back"]:
        lobra.lobra_mlora_block_norm_bwd(st["plan"], st["cfg"], st["r_out"], st["b"], st["w_post"], st["gate"], st["w_pre"], st["rstd_post"],
                                         st["rstd_pre"], st["dr_out"], st["dx"], st["dr"], st["db"], st["dgate"], st["dw_post"], st["dw_pre"],
                                         ws=st["ws"])
        out.update(dr=st["dr"], db=st["db"])
        # summed in 32 bits over a step's chunks; handed on in the parameters' type, as an exchange between replicas takes them
        out.update({k: st[k].to(st["r"].dtype) for k in ("dgate", "dw_post", "dw_pre") if st[k] is not None})
    return out


def _own_gated(st):
    from paper_2509_01193_amd import binding as lobra
    w = (st["x"], st["W"], st["A"], st["B"], st["s"])
    if not st["case"]["back"]:
        lobra.lobra_mlora_gated_fwd(st["plan"], st["code"], *w, None, st["h"], None, st["ws"])
        return dict(h=st["h"])
    lobra.lobra_mlora_gated_fwd(st["plan"], st["code"], *w, st["gu"], st["h"], st["h_save"], st["ws"])
    lobra.lobra_mlora_gated_bwd(st["plan"], st["code"], *w, st["gu"], st["dh"], st["h_save"], st["dgu"], st["dx_out"], st["dA"], st["dB"], 0,
                                st["ws"])
    # the adapters' gradients likewise: summed in 32 bits, handed on in the adapters' type
    return {"h": st["h"], "gu": st["gu"], "dgu": st["dgu"], "dx": st["dx_out"], "dA": st["dA"].to(st["A"].dtype), "dB": st["dB"].to(st["B"].dtype)}


# ---- plain forms: 32 bits throughout, rounded once at the end; a tensor that forward hands to backward (the new residual, the
#      saved projections) is in backward what forward gave out -----------------------------------------------------------
def _plain_statistics(z):
    m = z.max(dim=1, keepdim=True).values
    e = (z - m).exp()
    s = e.sum(dim=1, keepdim=True)
    return m, e, s, (m + s.log())


def _target_logp(z, target, lse):
    """z_target - lse, 0 for a row without a target."""
    has = target >= 0
    at = z.gather(1, target.clamp(min=0).long()[:, None])
    return torch.where(has, (at - lse)[:, 0], torch.zeros_like(lse[:, 0]))


def _plain_entropy(z, m, e, s):
    shifted = torch.where(e > 0, (z - m) * e, torch.zeros_like(e))
    return (s.log() - shifted.sum(dim=1, keepdim=True) / s)[:, 0]


def _plain_score(st):
    z, k = st["logits"].float(), st["case"]["top_k"]
    m, e, s, lse = _plain_statistics(z)
    out = dict(logp=_target_logp(z, st["target"], lse), lse=lse[:, 0], entropy=_plain_entropy(z, m, e, s))
    del e
    if k:
        # by value, the lowest index first among equals: one whole number that orders like that
        V = z.shape[1]
        bits = (z + 0.0).view(torch.int32).long()
        order = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits) * (1 << 20) + (V - 1 - torch.arange(V, device=DEV))
        at = V - 1 - (order.topk(k, dim=1).values & ((1 << 20) - 1))
        out.update(top_logp=z.gather(1, at) - lse, top_id=at.int())
    return out


def _plain_loss(st):
    z = st["logits"].float()
    m, e, s, lse = _plain_statistics(z)
    out = dict(logp=_target_logp(z, st["target"], lse), lse=lse[:, 0])
    p = e / s
    w = st["dlogp"][:, None]
    grad = -w * p
    if st["case"]["entropy"]:
        ent = _plain_entropy(z, m, e, s)
        out["entropy"] = ent
        grad -= st["dentropy"][:, None] * p * ((z - lse) + ent[:, None])
    target = st["target"].long()
    grad.scatter_add_(1, target.clamp(min=0)[:, None], torch.where(target[:, None] >= 0, w, torch.zeros_like(w)))
    out["dlogits"] = grad.to(st["logits"].dtype)
    return out


def _plain_clip(st):
    of, n = st["of"], st["case"]["tasks"]
    total = torch.zeros(n, device=DEV)
    for g in st["grads"]:
        total.index_add_(0, of, (g * g).sum(dim=1))
    norm = st["grad_scale"].abs() * total.sqrt()
    fine = torch.isfinite(norm)
    factor = torch.where(norm > st["max_norm"], st["max_norm"] / norm, torch.ones_like(norm))
    scale = torch.where(fine, st["grad_scale"] * factor, torch.zeros_like(norm))
    out = dict(norm=norm, scale=scale, step=torch.where(fine, st["step"], torch.zeros_like(st["step"])))
    if st["case"]["out"]:
        out["clipped"] = [g * scale[of][:, None] for g in st["grads"]]
    return out


def _plain_norm(st):
    case, dt = st["case"], st["r"].dtype
    r, b, w_pre = st["r"].float(), st["b"].float(), st["w_pre"].float()
    n = torch.rsqrt((b * b).mean(dim=1, keepdim=True) + EPS) if case["post"] else None
    bn = b * n if case["post"] else b
    w_post = st["w_post"].float() if case["post"] else torch.ones_like(w_pre)
    of, known = st["of"].clamp(min=0), (st["of"] >= 0)[:, None]
    gate = torch.where(known, st["gate"].float()[of], torch.ones_like(b)) if case["gate"] else torch.ones_like(b)
    rp = r + ALPHA * gate * (w_post * bn)
    r_out = rp.to(dt)
    rs = r_out.float()                       # the residual that is kept is the one that is normed, in forward too
    m = torch.rsqrt((rs * rs).mean(dim=1, keepdim=True) + EPS)
    out = dict(r_out=r_out, x=(rs * m * w_pre).to(dt))
    if not case["back"]:
        return out
    dx = st["dx"].float()
    rn, u = rs * m, w_pre * dx
    g = st["dr_out"].float() + m * (u - rn * (u * rn).mean(dim=1, keepdim=True))
    out["dr"] = g.to(dt)
    out["dw_pre"] = (dx * rn).sum(dim=0).to(dt)
    v = ALPHA * gate * g
    if case["gate"]:
        dgate = torch.zeros(case["tasks"], case["d"], device=DEV)
        contribution = ALPHA * g * w_post * bn
        for t, rows in enumerate(st["rows"]):
            dgate[t] = contribution[rows].sum(dim=0)
        out["dgate"] = dgate.to(dt)
    if case["post"]:
        out["dw_post"] = (v * bn).sum(dim=0).to(dt)
        v = v * w_post
        v = n * (v - bn * (v * bn).mean(dim=1, keepdim=True))
    out["db"] = v.to(dt)
    return out


def _plain_activation(act, g):
    """The activation and its derivative."""
    if act == "silu":
        q = 1 / (1 + (-g).exp())
        return g * q, q * (1 + g * (1 - q))
    c = math.sqrt(2 / math.pi)
    t = torch.tanh(c * (g + 0.044715 * g * g * g))
    return 0.5 * g * (1 + t), 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * c * (1 + 3 * 0.044715 * g * g)


def _plain_gated(st):
    case, dt = st["case"], st["x"].dtype
    f = case["f"]
    x, W, A, B = (st[k].float() for k in ("x", "W", "A", "B"))
    y = x @ W
    kept = []
    for t, rows in enumerate(st["rows"]):
        r0, r = int(st["rank_off"][t]), _ranks(case)[t]
        for j in (0, 1):
            w = slice(r0 + j * r, r0 + (j + 1) * r)
            low = st["s"][t] * (x[rows] @ A[w].t())
            y[rows, j * f:(j + 1) * f] += low @ B[w]
            kept.append((t, j, w, low))
    a, da = _plain_activation(case["act"], y[:, :f])
    out = dict(h=(a * y[:, f:]).to(dt))
    if not case["back"]:
        return out
    out["gu"] = y.to(dt)
    y = out["gu"].float()
    a, da = _plain_activation(case["act"], y[:, :f])
    dh = st["dh"].float()
    dy = torch.cat([dh * y[:, f:] * da, dh * a], dim=1)
    dx = dy @ W.t()
    dA, dB = torch.zeros_like(A), torch.zeros_like(B)
    for t, j, w, low in kept:
        rows = st["rows"][t]
        part = dy[rows, j * f:(j + 1) * f]
        back = st["s"][t] * (part @ B[w].t())
        dx[rows] += back @ A[w]
        dA[w] = back.t() @ x[rows]
        dB[w] = low.t() @ part
    out.update(dgu=dy.to(dt), dx=dx.to(dt), dA=dA.to(dt), dB=dB.to(dt))
    return out


# ------------------------------------------------------------------------------------------------------------------
# what a pass cannot do without
# ------------------------------------------------------------------------------------------------------------------
def work(case):
    kind, e = case["kind"], 4 if case.get("dtype") == "f32" else 2
    if kind == "score":
        n = case["T"] * case["V"]
        return dict(bytes=n * e + case["T"] * (16 + 8 * case["top_k"]), flops=5 * n)
    if kind == "loss":
        n = case["T"] * case["V"]
        return dict(bytes=2 * n * e + case["T"] * 24, flops=(12 if case["entropy"] else 8) * n)
    if kind == "clip":
        n = sum(r * d for r, d in _shapes(case))
        return dict(bytes=n * 4 * (2 if case["out"] else 1) + case["tasks"] * 24, flops=(3 if case["out"] else 2) * n)
    if kind == "norm":
        n, d = case["T"] * case["d"], case["d"]
        small = d * (1 + int(case["post"]) + (case["tasks"] if case["gate"] else 0))
        if not case["back"]:
            return dict(bytes=4 * n * e + small * e, flops=9 * n)
        # r, b -> r_out, x; then dr_out, dx -> dr, db
        return dict(bytes=8 * n * e + small * 2 * e, flops=30 * n)
    T, d, f, ranks = case["T"], case["d_in"], case["f"], _ranks(case)
    off, tk = _table(case)
    weighted = sum((off[k + 1] - off[k]) * ranks[t] for k, t in enumerate(tk) if t >= 0)
    adapters = 2 * sum(ranks) * (d + f)
    nbytes = (T * (d + f) + 2 * d * f + adapters) * e
    flops = 4 * T * d * f + 4 * weighted * (d + f) + 8 * T * f
    if case["back"]:
        # gate and up are kept for backward; dh, -> their gradients, dx, dA, dB
        nbytes += (2 * T * f + T * (3 * f + d)) * e + adapters * e
        flops += 4 * T * d * f + 8 * weighted * (d + f) + 16 * T * f
    return dict(bytes=nbytes, flops=flops)


# ------------------------------------------------------------------------------------------------------------------
# the operators' definition in 64 bits
# ------------------------------------------------------------------------------------------------------------------
def exact(case, seed):
    v = _inputs(case, seed)
    return {"score": _exact_logprob, "loss": _exact_logprob, "clip": _exact_clip, "norm": _exact_norm, "gated": _exact_gated}[case["kind"]](case, v)


def _exact_logprob(case, v):
    parts = {}
    for r0 in range(0, case["T"], 512):
        z = v["logits"][r0:r0 + 512].double()
        tgt = v["target"][r0:r0 + 512].tolist()
        lse = torch.logsumexp(z, dim=1)
        lp = z - lse[:, None]                                       # log probabilities
        p = lp.exp()
        ent = -torch.where(p > 0, p * lp, 0.0).sum(dim=1)
        piece = dict(logp=torch.stack([lp[i, t] if t >= 0 else lp.new_zeros(()) for i, t in enumerate(tgt)]), lse=lse)
        if case["kind"] == "score":
            piece["entropy"] = ent
            if case["top_k"]:
                vals, at = torch.sort(z, dim=1, descending=True, stable=True)
                piece.update(top_logp=vals[:, :case["top_k"]] - lse[:, None], top_id=at[:, :case["top_k"]].int())
        else:
            w = v["dlogp"][r0:r0 + 512].double()
            onehot = torch.zeros_like(z)
            live = [i for i, t in enumerate(tgt) if t >= 0]
            onehot[live, [tgt[i] for i in live]] = 1.0
            d = w[:, None] * torch.where((v["target"][r0:r0 + 512] >= 0)[:, None], onehot - p, -p)
            if case["entropy"]:
                piece["entropy"] = ent
                d += v["dentropy"][r0:r0 + 512].double()[:, None] * (-p * (lp + ent[:, None]))
            piece["dlogits"] = d
        for k, t in piece.items():
            parts.setdefault(k, []).append(t)
    return {k: torch.cat(ts) for k, ts in parts.items()}


def _exact_clip(case, v):
    ranks = _ranks(case)
    squares = [0.0] * case["tasks"]
    for g in v["grads"]:
        for t, part in enumerate(g.split(ranks)):
            squares[t] = squares[t] + part.double().square().sum()
    gs, most = v["grad_scale"].double(), v["max_norm"].double()
    norm = gs.abs() * torch.stack(squares).sqrt()
    scale = gs * torch.clamp(most / norm, max=1.0)
    out = dict(norm=norm, scale=scale, step=v["step"])
    if case["out"]:
        out["clipped"] = [torch.cat([part.double() * scale[t] for t, part in enumerate(g.split(ranks))]) for g in v["grads"]]
    return out


def _exact_norm(case, v):
    off, tk = _table(case)
    T, d, n = case["T"], case["d"], case["tasks"]
    rows_of = {t: [] for t in range(-1, n)}
    for k, t in enumerate(tk):
        rows_of[t] += range(off[k], off[k + 1])
    gate = torch.ones(T, d, dtype=torch.float64, device=DEV)
    if case["gate"]:
        for t in range(n):
            gate[rows_of[t]] = v["gate"][t].double()
    b = v["b"].double()
    post = case["post"]
    rms_b = (b.square().mean(dim=1, keepdim=True) + EPS).sqrt() if post else 1.0
    hat = b / rms_b
    wp = v["w_post"].double() if post else 1.0
    # the definition rounds the residual to the type in which it is kept before it is normed
    r_new = v["r"].double() + ALPHA * gate * wp * hat
    kept = r_new.to(v["r"].dtype).double()
    rms_r = (kept.square().mean(dim=1, keepdim=True) + EPS).sqrt()
    w = v["w_pre"].double()
    out = dict(r_out=r_new, x=w * kept / rms_r)
    if case["back"]:
        dx, y = v["dx"].double(), kept / rms_r
        inner = (dx * w * y).sum(dim=1, keepdim=True) / d
        g = v["dr_out"].double() + (dx * w - y * inner) / rms_r
        out["dr"], out["dw_pre"] = g, (dx * y).sum(dim=0)
        if case["gate"]:
            out["dgate"] = torch.stack([(ALPHA * wp * hat[rows_of[t]] * g[rows_of[t]]).sum(dim=0) for t in range(n)])
        if post:
            q = ALPHA * gate * g
            out["dw_post"] = (q * hat).sum(dim=0)
            q = q * wp
            out["db"] = (q - hat * ((q * hat).sum(dim=1, keepdim=True) / d)) / rms_b
        else:
            out["db"] = ALPHA * gate * g
    return out


def _exact_gated(case, v):
    off, tk = _table(case)
    f, ranks = case["f"], _ranks(case)
    x, W, A, B, s = (v[k].double() for k in ("x", "W", "A", "B", "s"))
    of = torch.tensor(np.repeat(np.asarray(tk), np.diff(np.asarray(off))), device=DEV)
    # per projection: the shared product, then every task's low-rank term on the rows of its tokens
    halves = []
    for j in (0, 1):
        y = x @ W[:, j * f:(j + 1) * f]
        row = 0
        for t, r in enumerate(ranks):
            idx = (of == t).nonzero().flatten()
            w = slice(row + j * r, row + (j + 1) * r)
            if len(idx):
                y[idx] += s[t] * ((x[idx] @ A[w].T) @ B[w])
            row += 2 * r
        halves.append(y)
    g, u = halves

    def act(g):
        if case["act"] == "silu":
            q = torch.sigmoid(g)
            return g * q, q + g * q * (1 - q)
        k = math.sqrt(2 / math.pi)
        th = torch.tanh(k * (g + 0.044715 * g ** 3))
        return g * (1 + th) / 2, (1 + th) / 2 + g * (1 - th ** 2) / 2 * k * (1 + 0.134145 * g ** 2)

    out = dict(h=act(g)[0] * u)
    if not case["back"]:
        return out
    out["gu"] = torch.cat([g, u], dim=1)
    # backward is defined on the projections as they were kept
    g, u = (t.to(v["x"].dtype).double() for t in (g, u))
    a, da = act(g)
    dh = v["dh"].double()
    dhalves = [dh * u * da, dh * a]
    dx = torch.zeros_like(x)
    dA, dB = torch.zeros_like(A), torch.zeros_like(B)
    for j, dy in enumerate(dhalves):
        dx += dy @ W[:, j * f:(j + 1) * f].T
        row = 0
        for t, r in enumerate(ranks):
            idx = (of == t).nonzero().flatten()
            w = slice(row + j * r, row + (j + 1) * r)
            if len(idx):
                low = dy[idx] @ B[w].T
                dx[idx] += s[t] * (low @ A[w])
                dA[w] = s[t] * (low.T @ x[idx])
                dB[w] = s[t] * ((x[idx] @ A[w].T).T @ dy[idx])
            row += 2 * r
    out.update(dgu=torch.cat(dhalves, dim=1), dx=dx, dA=dA, dB=dB)
    return out
