"""An 8-bit base, adapters trained on a teacher's likeliest tokens, and beam search, as measurable cases: plain, through the library,
and in 64 bits.

A case is a plain dict.  Its `kind` says which operator one pass goes through:

  q8        the LoRA linear on a frozen base held in 8-bit integers with a scale per channel, the tokens quantised with a scale each as
            they come: lobra_mlora_quant_fwd, with `back` also lobra_mlora_quant_bwd
  distill   the loss of rows of logits against the likeliest tokens of a teacher, and the gradient of the logits:
            lobra_token_distill_fwd, _bwd
  beam      a step of beam search: the best continuations over the beams and the vocabulary of every request, then what is kept per
            sequence put in the order of the beams that go on: lobra_beam_select, lobra_beam_reorder

`own` says who computes: False - elementary torch operations in 32 bits (64 where values next to a border decide); True - the library.
Widths are those of the layers that the library's other cases have (4096 and 11008, 1376 = 11008 / 8) or generic.
"""
import math
import random

import numpy as np
import torch

own = False

DEV = "cuda:0"


def listed():
    return [
        # one new token for each of 40 requests through a linear of a 7B model
        dict(name="q8_decode", kind="q8", T=40, d_in=4096, d_out=4096, tasks=8, ranks="16", mean_len=1, bare=0.1, back=False),
        # a few prompts at once through the gate projection of such a model, mixed ranks, an odd number of tokens
        dict(name="q8_prompts", kind="q8", T=777, d_in=4096, d_out=11008, tasks=6, ranks="8,16,32", mean_len=120, bare=0.1, back=False),
        # an evaluation batch through the same projection, the largest product here
        dict(name="q8_16k", kind="q8", T=16384, d_in=4096, d_out=11008, tasks=4, ranks="16", mean_len=400, bare=0.0, back=False),
        # training the adapters of one linear of a 7B model on a packed batch
        dict(name="q8_train", kind="q8", T=8190, d_in=4096, d_out=4096, tasks=4, ranks="16", mean_len=400, bare=0.0, back=True),
        # one of eight tensor-parallel shards of its down projection: a width that is no power of two
        dict(name="q8_shard", kind="q8", T=2999, d_in=1376, d_out=4096, tasks=3, ranks="16,64", mean_len=300, bare=0.1, back=True),
        # the loss of one short sequence
        dict(name="distill_short", kind="distill", dtype="bf16", T=48, V=32000, top_k=8, tail=False, temperature=1.0, bare=0.2),
        # a packed training batch against the 20 likeliest tokens of a softened teacher, prompts without one (a third of the tokens)
        dict(name="distill_8k", kind="distill", dtype="bf16", T=8190, V=32000, top_k=20, tail=False, temperature=2.0, bare=0.33),
        # a large vocabulary; what the teacher's list leaves out counts as one more token
        dict(name="distill_vocab", kind="distill", dtype="bf16", T=4096, V=128000, top_k=64, tail=True, temperature=1.0, bare=0.1),
        # fp32 logits of an odd vocabulary, rows aligned to nothing
        dict(name="distill_f32_odd", kind="distill", dtype="f32", T=1000, V=50257, top_k=32, tail=True, temperature=1.0, bare=0.1),
        # one request with four beams
        dict(name="beam_one", kind="beam", dtype="bf16", n_req=1, beams=4, n_out=4, V=32000, states=2, length=128, width=512, done=0.0, first=False),
        # a serving batch over a large vocabulary
        dict(name="beam_batch", kind="beam", dtype="bf16", n_req=64, beams=8, n_out=8, V=128000, states=4, length=256, width=512, done=0.1,
             first=False),
        # fp32 logits of an odd vocabulary, twice as many candidates as beams, odd rows of state
        dict(name="beam_f32_odd", kind="beam", dtype="f32", n_req=5, beams=5, n_out=10, V=50257, states=3, length=77, width=33, done=0.2, first=False),
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A layer width: mostly whole multiples of 128 as models have them, else any multiple of 8."""
    m = rng.choice([128, 128, 256, 32, 8])
    return max(m, _spread(rng, lo, hi) // m * m)


def draw(rng):
    kind = rng.choice(["q8", "q8", "q8", "distill", "distill", "beam", "beam"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if kind == "q8":
        T, d, f = _spread(rng, 1, 16384), _width(rng, 256, 4096), _width(rng, 256, 11008)
        return dict(kind=kind, T=T, d_in=d, d_out=f, tasks=rng.choice([1, 2, 4, 8, 16]), ranks=rng.choice(["8", "16", "16", "32", "8,16,64"]),
                    mean_len=1 if T < 100 else _spread(rng, 30, 1500), bare=rng.choice([0.0, 0.1]),
                    back=T >= 100 and T * d * f < 3 * 10**11 and rng.random() < 0.5)
    V = _spread(rng, 1000, 131072)
    if rng.random() < 0.6:
        V = V // 64 * 64 + 64
    if kind == "distill":
        T = min(_spread(rng, 1, 16384), (250 if dtype == "f32" else 500) * 10**6 // V)
        return dict(kind=kind, dtype=dtype, T=T, V=V, top_k=rng.choice([1, 4, 10, 32, 64, 128]), tail=rng.random() < 0.5,
                    temperature=rng.choice([1.0, 1.0, 2.0, 0.7]), bare=rng.choice([0.0, 0.33, 0.8]))
    beams = rng.choice([1, 2, 4, 5, 8, 16])
    n_req = max(1, min(_spread(rng, 1, 256), (30 if dtype == "f32" else 60) * 10**6 // (V * beams)))
    length, width = _spread(rng, 1, 512), rng.choice([1, 33, 128, 512, 576])
    states = max(1, min(rng.choice([1, 2, 8, 40]), 400 * 10**6 // (n_req * beams * length * width * 4)))
    return dict(kind=kind, dtype=dtype, n_req=n_req, beams=beams, n_out=beams * rng.choice([1, 2]), V=V, states=states, length=length, width=width,
                done=rng.choice([0.0, 0.2]), first=rng.random() < 0.2)


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


DONE_TOKEN = 2


def _inputs(case, seed):
    g = torch.Generator(device=DEV).manual_seed(int(seed))
    dt = _dtype(case)

    def normal(std, *shape, dtype=dt):
        return torch.randn(*shape, device=DEV, dtype=dtype, generator=g).mul_(std)

    def uniform(*shape):
        return torch.rand(*shape, device=DEV, generator=g)

    kind = case["kind"]
    if kind == "q8":
        T, d, f, R = case["T"], case["d_in"], case["d_out"], sum(_ranks(case))
        # some channels of the activations are larger than the rest, as they are behind a norm
        x = normal(1.0, T, d) * (1 + 7 * (uniform(d) < 0.01)).to(dt)
        v = dict(x=x, W=normal(0.02, d, f), A=normal(0.02, R, d), B=normal(0.02, R, f), s=uniform(case["tasks"]) + 0.5)
        if case["back"]:
            v["dy"] = normal(1.0, T, f)
        return v
    if kind == "distill":
        T, V, k = case["T"], case["V"], case["top_k"]
        teacher = normal(2.5, T, V)
        teacher[torch.arange(T, device=DEV), torch.randint(0, V, (T,), device=DEV, generator=g)] += (uniform(T) * 16).to(dt)
        top, ids = teacher.topk(k, dim=1)
        # the teacher's log probabilities; where what the list leaves out counts, they are those at the temperature
        t = case["temperature"] if case["tail"] else 1.0
        lse = torch.cat([torch.logsumexp(teacher[r:r + 512].float() / t, dim=1) for r in range(0, T, 512)])
        v = dict(logits=teacher.add_(normal(0.7, T, V)), teacher_logp=top.float() / t - lse[:, None], teacher_id=ids.to(torch.int32))
        # rows without a teacher, and lists that are shorter than the others
        bare = uniform(T) < case["bare"]
        kept = torch.where(bare, torch.zeros(T, device=DEV), torch.where(uniform(T) < 0.8, float(k), (uniform(T) * k).ceil()))
        none = torch.arange(k, device=DEV)[None, :] >= kept[:, None]
        v["teacher_logp"][none] = float("-inf")
        v["teacher_id"][none] = -1
        v["dloss"] = torch.where(bare, torch.zeros(T, device=DEV), (uniform(T) + 0.5) / T)
        return v
    n, b, V = case["n_req"], case["beams"], case["V"]
    logits = normal(2.0, n * b, V)
    logits[torch.arange(n * b, device=DEV), torch.randint(0, V, (n * b,), device=DEV, generator=g)] += (uniform(n * b) * 10).to(dt)
    score = -20 * uniform(n, b)
    if case["first"]:
        score[:, 1:] = float("-inf")                 # the first step of a request: one beam
    return dict(logits=logits, score=score, done=(uniform(n, b) < case["done"]).to(torch.int32),
                states=[normal(1.0, n * b, case["length"], case["width"]) for _ in range(case["states"])],
                used=torch.randint(1, case["length"] + 1, (n,), device=DEV, generator=g, dtype=torch.int32))


def prepare(case, seed):
    st = dict(case=dict(case))
    st.update(_inputs(case, seed))
    kind, dt = case["kind"], _dtype(case)

    def empty(*shape, dtype=torch.float32):
        return torch.empty(*shape, dtype=dtype, device=DEV)

    if kind == "beam":
        # where the kept states go: the caller's second set of buffers
        st["next"] = [torch.zeros_like(t) for t in st["states"]]
    if kind == "q8":
        st["off"], st["task"] = _table(case)
        st["rank_off"] = np.concatenate([[0], np.cumsum(_ranks(case))])
    if not own:
        if kind == "q8":
            # which rows belong to which task, as a program without the library would keep it; the weight in 8 bits, made once
            of = torch.tensor(np.repeat(np.asarray(st["task"]), np.diff(np.asarray(st["off"]))), device=DEV)
            st["rows"] = [(of == t).nonzero().flatten() for t in range(case["tasks"])]
            q, scale = _plain_quantise(st["W"].t())
            st["Wq"], st["w_scale"] = q.t().contiguous().to(torch.int8), scale[:, 0]
            del st["W"]
        return st
    from paper_2509_01193_amd import binding as lobra
    if kind == "q8":
        T, d, f = case["T"], case["d_in"], case["d_out"]
        st["plan"] = lobra.Plan("bf16", T, d, f, st["rank_off"], st["off"], st["task"])
        st["Wq"], st["w_scale"] = empty(f, lobra.lobra_quant_pitch(d), dtype=torch.int8), empty(f)
        lobra.lobra_quantise_weight(st["W"], st["Wq"], st["w_scale"])
        del st["W"]
        st["y"] = empty(T, f, dtype=dt)
        fwd, bwd = lobra.lobra_mlora_quant_workspace_bytes(st["plan"])
        st["ws"] = empty(max(fwd, bwd if case["back"] else 0, 16), dtype=torch.uint8)
        if case["back"]:
            st.update(dx=empty(T, d, dtype=dt), dA=torch.empty_like(st["A"], dtype=torch.float32), dB=torch.empty_like(st["B"], dtype=torch.float32))
            st["h_save"] = empty(max(st["plan"].h_save_bytes, 16), dtype=torch.uint8)
    elif kind == "distill":
        T = case["T"]
        st["desc"] = lobra.make_distill_desc(case["dtype"], T, case["V"], case["top_k"], tail=case["tail"], temperature=case["temperature"])
        st.update(loss=empty(T), stat=empty(T, 4), dlogits=torch.empty_like(st["logits"]))
    else:
        n, k = case["n_req"], case["n_out"]
        st["desc"] = lobra.make_beam_desc(case["dtype"], n, case["beams"], case["V"], k)
        st["ws"] = empty(max(lobra.lobra_beam_workspace_bytes(st["desc"]), 16), dtype=torch.uint8)
        st.update(out_score=empty(n, k), out_beam=empty(n, k, dtype=torch.int32), out_token=empty(n, k, dtype=torch.int32))
    return st


# ------------------------------------------------------------------------------------------------------------------
# one pass
# ------------------------------------------------------------------------------------------------------------------
def run(st):
    kind = st["case"]["kind"]
    if own:
        return {"q8": _own_q8, "distill": _own_distill, "beam": _own_beam}[kind](st)
    return {"q8": _plain_q8, "distill": _plain_distill, "beam": _plain_beam}[kind](st)


def _own_q8(st):
    from paper_2509_01193_amd import binding as lobra
    w = (st["x"], st["Wq"], st["w_scale"], st["A"], st["B"], st["s"])
    if not st["case"]["back"]:
        lobra.lobra_mlora_quant_fwd(st["plan"], *w, st["y"], None, st["ws"])
        return dict(y=st["y"])
    lobra.lobra_mlora_quant_fwd(st["plan"], *w, st["y"], st["h_save"], st["ws"])
    lobra.lobra_mlora_quant_bwd(st["plan"], *w, st["dy"], st["h_save"], st["dx"], st["dA"], st["dB"], 0, st["ws"])
    # the adapters' gradients: summed in 32 bits over a step's chunks, handed on in the adapters' type, as an exchange between replicas takes them
    return dict(y=st["y"], dx=st["dx"], dA=st["dA"].to(st["A"].dtype), dB=st["dB"].to(st["B"].dtype))


def _own_distill(st):
    from paper_2509_01193_amd import binding as lobra
    w = (st["desc"], st["logits"], st["teacher_logp"], st["teacher_id"])
    lobra.lobra_token_distill_fwd(*w, st["loss"], st["stat"])
    lobra.lobra_token_distill_bwd(*w, st["stat"], st["dloss"], st["dlogits"])
    return dict(loss=st["loss"], dlogits=st["dlogits"])


def _own_beam(st):
    from paper_2509_01193_amd import binding as lobra
    lobra.lobra_beam_select(st["desc"], st["logits"], st["score"], st["done"], DONE_TOKEN, st["out_score"], st["out_beam"], st["out_token"], st["ws"])
    lobra.lobra_beam_reorder(list(zip(st["states"], st["next"])), st["case"]["n_req"], st["case"]["beams"],
                             st["out_beam"][:, :st["case"]["beams"]], st["used"])
    return dict(score=st["out_score"], beam=st["out_beam"], token=st["out_token"], states=st["next"])


# ---- plain forms ---------------------------------------------------------------------------------------------------
def _plain_quantise(v):
    """Whole numbers between -127 and 127 and a 32-bit scale per row; a quotient half way between two goes to the even one, which takes 64 bits to
    see."""
    scale = (v.abs().amax(dim=1, keepdim=True).double() / 127).float()
    return torch.where(scale > 0, v.double() / scale.double(), 0.0).round().float(), scale


def _plain_q8(st):
    case, dt = st["case"], st["x"].dtype
    x, A, B = (st[k].float() for k in ("x", "A", "B"))
    xq, x_scale = _plain_quantise(st["x"])
    wq = st["Wq"].float()
    y = (xq @ wq) * x_scale * st["w_scale"]
    kept = []
    for t, rows in enumerate(st["rows"]):
        w = slice(int(st["rank_off"][t]), int(st["rank_off"][t + 1]))
        low = st["s"][t] * (x[rows] @ A[w].t())
        y[rows] += low @ B[w]
        kept.append((t, rows, w, low))
    out = dict(y=y.to(dt))
    if not case["back"]:
        return out
    dy = st["dy"].float()
    dx = dy @ (wq * st["w_scale"]).t()
    dA, dB = torch.zeros_like(A), torch.zeros_like(B)
    for t, rows, w, low in kept:
        back = st["s"][t] * (dy[rows] @ B[w].t())
        dx[rows] += back @ A[w]
        dA[w] = back.t() @ x[rows]
        dB[w] = low.t() @ dy[rows]
    out.update(dx=dx.to(dt), dA=dA.to(dt), dB=dB.to(dt))
    return out


def _plain_distill(st):
    case = st["case"]
    inv = 1.0 / case["temperature"]
    z = st["logits"].float() * inv
    m = z.max(dim=1, keepdim=True).values
    e = (z - m).exp()
    total = e.sum(dim=1, keepdim=True)
    ids, used = st["teacher_id"].clamp(min=0).long(), st["teacher_id"] >= 0
    tl = torch.where(used, st["teacher_logp"], torch.full_like(st["teacher_logp"], float("-inf")))
    zero = torch.zeros_like(tl)
    any_ = used.any(dim=1, keepdim=True)
    if case["tail"]:
        ln_q = tl
    else:
        tl = tl * inv
        top = torch.where(any_, tl.max(dim=1, keepdim=True).values, zero[:, :1])
        ln_q = tl - (top + (tl - top).exp().sum(dim=1, keepdim=True).log())
        ln_q = torch.where(used, ln_q, torch.full_like(ln_q, float("-inf")))
    q = ln_q.exp()
    ln_p = z.gather(1, ids) - m - total.log()
    loss = torch.where(used, q * (ln_q - ln_p), zero).sum(dim=1)
    p = e / total
    if case["tail"]:
        rest = e.scatter(1, ids, torch.where(used, zero, e.gather(1, ids)))      # what the list leaves out
        # (an unused place points at token 0, which another place may have taken out)
        first = (used & (ids == 0)).any(dim=1)
        rest[:, 0] = torch.where(first, torch.zeros_like(first, dtype=rest.dtype), rest[:, 0])
        left = 1 - q.double().sum(dim=1, keepdim=True)
        qr = torch.where(left > 2.0 ** -20, left, 0.0).float()
        sum_rest = rest.sum(dim=1, keepdim=True)
        has = qr > 0
        loss += torch.where(has, qr * (qr.log() - (sum_rest.log() - total.log())), zero[:, :1])[:, 0]
        grad = (q.sum(dim=1, keepdim=True) + qr) * p - torch.where(has & (sum_rest > 0), qr / sum_rest, zero[:, :1]) * rest
    else:
        grad = q.sum(dim=1, keepdim=True) * p
    grad.scatter_add_(1, ids, -torch.where(used, q, zero))
    grad *= st["dloss"][:, None] * inv
    live = any_[:, 0]
    return dict(loss=torch.where(live, loss, torch.zeros_like(loss)), dlogits=torch.where(any_, grad, torch.zeros_like(grad[:1, :1])).to(st["logits"].dtype))


def _plain_beam(st):
    case = st["case"]
    n, b, k, V = case["n_req"], case["beams"], case["n_out"], case["V"]
    z = st["logits"].float()
    # a request's continuations lie close together: their order is that of sums in 64 bits
    m = z.max(dim=1, keepdim=True).values.double()
    lse = m + (z.double() - m).exp().sum(dim=1, keepdim=True).log()
    # the k largest of each row by value, the lowest index first among equals: one whole number that orders like that
    bits = (z + 0.0).view(torch.int32).long()
    order = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits) * (1 << 20) + (V - 1 - torch.arange(V, device=DEV))
    kk = min(k, V)
    at = V - 1 - (order.topk(kk, dim=1).values & ((1 << 20) - 1))
    score = st["score"].double().view(n * b, 1)
    value = score + (z.gather(1, at).double() - lse)
    # a beam that is done goes on as it is
    done = st["done"].view(n * b, 1) != 0
    alone = torch.cat([score, torch.full((n * b, kk - 1), float("-inf"), dtype=torch.float64, device=DEV)], dim=1)
    value = torch.where(done, alone, value)
    at = torch.where(done, torch.full_like(at, DONE_TOKEN), at)
    best, place = torch.sort(value.view(n, b * kk), dim=1, descending=True, stable=True)
    best, place = best[:, :k], place[:, :k]
    some = best > float("-inf")
    beam = torch.where(some, place // kk, -1)
    token = torch.where(some, at.view(n, b * kk).gather(1, place), -1)
    out = dict(score=best.float(), beam=beam.int(), token=token.int())
    # the states: position after position of the beam that goes on, as far as the request has got
    parent = beam[:, :b]
    rows = (torch.arange(n, device=DEV)[:, None] * b + parent.clamp(min=0)).view(-1)
    live = (torch.arange(case["length"], device=DEV)[None, :] < st["used"][:, None]).repeat_interleave(b, dim=0) & (parent.reshape(-1, 1) >= 0)
    out["states"] = [torch.where(live[:, :, None], s[rows], d) for s, d in zip(st["states"], st["next"])]
    return out


# ------------------------------------------------------------------------------------------------------------------
# what a pass cannot do without
# ------------------------------------------------------------------------------------------------------------------
def work(case):
    kind, e = case["kind"], 4 if case.get("dtype") == "f32" else 2
    if kind == "q8":
        T, d, f, ranks = case["T"], case["d_in"], case["d_out"], _ranks(case)
        off, tk = _table(case)
        weighted = sum((off[k + 1] - off[k]) * ranks[t] for k, t in enumerate(tk) if t >= 0)
        adapters = sum(ranks) * (d + f) * 2
        nbytes, flops = T * (d + f) * 2 + d * f + 4 * f + adapters, 2 * T * d * f + 2 * weighted * (d + f)
        if case["back"]:
            # dy, the weight and the adapters -> dx, dA, dB
            nbytes += T * (d + f) * 2 + d * f + 2 * adapters
            flops += 2 * T * d * f + 4 * weighted * (d + f)
        return dict(bytes=nbytes, flops=flops)
    if kind == "distill":
        n, k = case["T"] * case["V"], case["T"] * case["top_k"]
        return dict(bytes=2 * n * e + 8 * k + 24 * case["T"], flops=8 * n + 16 * k)
    rows = case["n_req"] * case["beams"]
    per = case["length"] * case["width"] * e
    # half of the positions are in use on average: read and written
    return dict(bytes=rows * (case["V"] * e + 8) + 12 * case["n_req"] * case["n_out"] + case["states"] * rows * per, flops=5 * rows * case["V"])


# ------------------------------------------------------------------------------------------------------------------
# the operators' definition in 64 bits
# ------------------------------------------------------------------------------------------------------------------
def exact(case, seed):
    v = _inputs(case, seed)
    return {"q8": _exact_q8, "distill": _exact_distill, "beam": _exact_beam}[case["kind"]](case, v)


def _exact_rounded(v, dim):
    """v as the whole multiples of a 32-bit step that stand for it: 127 steps are the largest magnitude along `dim`."""
    step = (v.abs().max(dim=dim, keepdim=True).values.double() / 127.0).to(torch.float32).double()
    return torch.round(v.double() / torch.where(step == 0, 1.0, step)) * step


def _exact_q8(case, v):
    off, tk = _table(case)
    x, A, B, dy = v["x"].double(), v["A"].double(), v["B"].double(), v["dy"].double() if case["back"] else None
    W = _exact_rounded(v["W"], 0)
    y = _exact_rounded(v["x"], 1) @ W
    dx = dy @ W.T if case["back"] else None
    dA, dB = torch.zeros_like(A), torch.zeros_like(B)
    of = torch.tensor(np.repeat(np.asarray(tk), np.diff(np.asarray(off))), device=DEV)
    row = 0
    for t, r in enumerate(_ranks(case)):
        idx, a, b, s = (of == t).nonzero().flatten(), A[row:row + r], B[row:row + r], float(v["s"][t])
        if len(idx):
            y[idx] += s * ((x[idx] @ a.T) @ b)
            if case["back"]:
                low = dy[idx] @ b.T
                dx[idx] += s * (low @ a)
                dA[row:row + r] = s * (low.T @ x[idx])
                dB[row:row + r] = s * ((x[idx] @ a.T).T @ dy[idx])
        row += r
    return dict(y=y, dx=dx, dA=dA, dB=dB) if case["back"] else dict(y=y)


def _exact_distill(case, v):
    t, losses, grads = case["temperature"], [], []
    for r0 in range(0, case["T"], 512):
        part = slice(r0, r0 + 512)
        z = v["logits"][part].double() / t
        lp = torch.log_softmax(z, dim=1)
        ids, tl = v["teacher_id"][part].long(), v["teacher_logp"][part].double()
        used = ids >= 0
        q = torch.zeros_like(z)                      # the teacher's probabilities, spread out over the vocabulary
        listed_ = torch.zeros_like(z, dtype=torch.bool)
        r, c = used.nonzero(as_tuple=True)
        w = torch.where(used, tl, float("-inf")) if case["tail"] else torch.log_softmax(torch.where(used, tl / t, float("-inf")), dim=1)
        q[r, ids[r, c]] = w[r, c].exp()
        listed_[r, ids[r, c]] = True
        loss = torch.where(q > 0, q * (q.clamp(min=1e-300).log() - lp), 0.0).sum(dim=1)
        p = lp.exp()
        mass = q.sum(dim=1, keepdim=True)
        grad = mass * p - q
        if case["tail"]:
            qr = 1 - mass
            qr = torch.where(qr > 2.0 ** -20, qr, 0.0)
            ln_r = torch.logsumexp(torch.where(listed_, float("-inf"), lp), dim=1, keepdim=True)
            loss += torch.where(qr > 0, qr * (qr.clamp(min=1e-300).log() - ln_r), 0.0)[:, 0]
            grad += qr * (p - torch.where(listed_, 0.0, (lp - ln_r).exp()))
        live = used.any(dim=1)
        losses.append(torch.where(live, loss, 0.0))
        grads.append(torch.where(live[:, None], grad * (v["dloss"][part].double()[:, None] / t), 0.0))
    return dict(loss=torch.cat(losses), dlogits=torch.cat(grads))


def _exact_beam(case, v):
    n, b, k, V = case["n_req"], case["beams"], case["n_out"], case["V"]
    neg = float("-inf")
    score, beam, token = [], [], []
    for i in range(n):
        lp = torch.log_softmax(v["logits"][i * b:(i + 1) * b].double(), dim=1)
        total = v["score"][i].double()[:, None] + lp
        for j in range(b):
            if int(v["done"][i, j]):
                total[j] = neg
                total[j, DONE_TOKEN] = v["score"][i, j].double()
        best, at = torch.sort(total.flatten(), descending=True, stable=True)
        best, at = best[:k], at[:k]
        if len(best) < k:
            best, at = (torch.nn.functional.pad(best, (0, k - len(best)), value=neg), torch.nn.functional.pad(at, (0, k - len(at))))
        score.append(best)
        beam.append(torch.where(best > neg, at // V, -1))
        token.append(torch.where(best > neg, at % V, -1))
    beam = torch.stack(beam)
    states = []
    for s in v["states"]:
        new = torch.zeros_like(s)
        for i, used in enumerate(v["used"].tolist()):
            for j, p in enumerate(beam[i, :b].tolist()):
                if p >= 0:
                    new[i * b + j, :used] = s[i * b + p, :used]
        states.append(new)
    return dict(score=torch.stack(score), beam=beam.int(), token=torch.stack(token).int(), states=states)
