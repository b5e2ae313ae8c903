"""One replica's joint fine-tuning step, end to end: several tasks' sequences packed into one batch, through a stack of residual blocks.

    x = norm(r);  [g | u] = x W_gu + adapters;  h = silu(g) u;  b = h W_down + adapters;  r = r + gate_t * norm(b);  next block ...
    logits = norm(r) W_head;  loss of a task = - mean of the log probabilities of its targets

Embedding, base weights, head and the norms' gains are frozen; every task trains its own adapters and gates, clipped to its own gradient
norm, so that no task's spike touches another's step.  A block's second norm, its gate, the residual and the next block's first norm are
one call.  Attention is not part of it: the next token is learnt from the token alone.

The base of the down projections and the head can be put into 8-bit integers (quantise_base); adapters on it learn from the likeliest tokens of
another model, the one before for instance (teacher = ...), and prompts are continued by beam search (search).

    python -m paper_2509_01193_amd.joint_step --steps 30          # trains, then continues a prompt of every task token by token
    python -m paper_2509_01193_amd.joint_step --steps 30 --distill-steps 10 --beams 4       # then an 8-bit base, distillation, beam search
"""
import argparse
import math

import torch

from paper_2509_01193_amd import binding as lobra

LR_GATE = 0.02


def not_8_bits(dtype, d, f):
    """Why a base of this type and these widths is not put into 8 bits; None if it is."""
    if dtype != "bf16":
        return "a base in 8-bit integers is one of bf16 layers"
    return "layers wider than %d are not put into 8-bit integers" % lobra.MAX_QUANT_IN if max(d, f) > lobra.MAX_QUANT_IN else None


class JointStep:
    """Buffers and plans of a batch whose packing stays: seg_off / seg_task as in the plan (-1: tokens without an adapter)."""

    def __init__(self, dtype, d, f, vocab, layers, ranks, seg_off, seg_task, lr=2e-3, max_norm=1.0, eps=1e-5, seed=0, device="cuda:0"):
        self.dtype, self.edt = dtype, {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
        self.d, self.f, self.vocab, self.layers, self.n_tasks = d, f, vocab, layers, len(ranks)
        self.dev = torch.device(device)
        gen = torch.Generator().manual_seed(seed)

        def normal(*shape, std):
            return torch.randn(*shape, generator=gen) * std

        off = [0]
        for r in ranks:
            off.append(off[-1] + r)
        self.rank_off, self.rank_off2 = off, [2 * r for r in off]       # (gate and up projection: stacked)
        self.embedding = normal(vocab, d, std=1.0).to(self.dev, self.edt)
        self.head = normal(d, vocab, std=1 / math.sqrt(d)).to(self.dev, self.edt)
        self.gain = torch.ones(d, dtype=self.edt, device=self.dev)
        self.s = torch.full((self.n_tasks,), 2.0, device=self.dev)
        self.cfg = lobra.BlockNormConfig(eps, 1.0)
        self.adam = lobra.AdamConfig(0.9, 0.95, 1e-8, 0.0)
        self.lr = torch.full((self.n_tasks,), lr, device=self.dev)
        self.max_norm = torch.full((self.n_tasks,), max_norm, device=self.dev)
        self.steps = torch.zeros(self.n_tasks, dtype=torch.int32, device=self.dev)
        self.blocks, grads = [], []
        for _ in range(layers):
            blk = {"W_gu": normal(d, 2 * f, std=1 / math.sqrt(d)).to(self.dev, self.edt),
                   "W_down": normal(f, d, std=1 / math.sqrt(f)).to(self.dev, self.edt),
                   "gate32": torch.full((self.n_tasks, d), 0.5, device=self.dev)}
            blk["gate"] = blk["gate32"].to(self.edt)
            for name, R, d_in, d_out in (("gu", 2 * off[-1], d, f), ("down", off[-1], f, d)):
                for m, shape, std in (("A", (R, d_in), 1 / math.sqrt(d_in)), ("B", (R, d_out), 0.0)):
                    k = m + "_" + name
                    blk["master_" + k] = normal(*shape, std=std).to(self.dev)
                    blk[k] = blk["master_" + k].to(self.edt)
                    for what in ("m_", "v_", "d"):
                        blk[what + k] = torch.zeros(*shape, device=self.dev)
                    grads.append((blk["d" + k], None, self.rank_off2 if name == "gu" else self.rank_off))
            blk["dgate"] = torch.zeros(self.n_tasks, d, device=self.dev)
            grads.append((blk["dgate"], None, list(range(self.n_tasks + 1))))     # one row a task, as of rank 1
            self.blocks.append(blk)
        self.head8 = None
        self.grads = lobra.GradSet(grads, self.n_tasks)
        self.norm, self.clip_scale = (torch.empty(self.n_tasks, device=self.dev) for _ in range(2))
        self.step_now = torch.empty_like(self.steps)
        self.batch(seg_off, seg_task)

    def quantise_base(self):
        """The frozen weights of the down projections and the head in 8-bit integers from here on; the others are not kept.  ValueError, and the weights as
        they are, where that can't be."""
        why = not_8_bits(self.dtype, self.d, self.f) if self.head8 is None else "the base is in 8-bit integers already"
        if why:
            raise ValueError(why)

        def quantised(W):
            d_in, d_out = W.shape
            q = torch.empty(d_out, lobra.lobra_quant_pitch(d_in), dtype=torch.int8, device=self.dev), torch.empty(d_out, device=self.dev)
            lobra.lobra_quantise_weight(W, *q)
            return q

        for blk in self.blocks:
            blk["W_down8"] = quantised(blk.pop("W_down"))
        self.head8, self.head = quantised(self.head), None
        self.batch(*self.packing)

    def restart(self):
        """Adapters that add nothing yet, and gates, as at the beginning (the down factors stay)."""
        for blk in self.blocks:
            for k in ("A_gu", "B_gu", "A_down", "B_down"):
                for what in ("m_", "v_") + (("master_", "") if k[0] == "B" else ()):
                    blk[what + k].zero_()
            blk["gate32"].fill_(0.5)
            blk["gate"].copy_(blk["gate32"])
        self.steps.zero_()

    def _fwd(self, plan, x, W, W8, A, B, s, y, h_save):
        if W8 is None:
            lobra.lobra_mlora_plan_fwd(plan, x, W, A, B, s, y, h_save, self.ws)
        else:
            lobra.lobra_mlora_quant_fwd(plan, x, *W8, A, B, s, y, h_save, self.ws)

    def _bwd(self, plan, x, W, W8, A, B, s, dy, h_saved, dx, dA, dB):
        if W8 is None:
            lobra.lobra_mlora_plan_bwd(plan, x, W, A, B, s, dy, h_saved, dx, dA, dB, 0, self.ws)
        else:
            lobra.lobra_mlora_quant_bwd(plan, x, *W8, A, B, s, dy, h_saved, dx, dA, dB, 0, self.ws)

    def batch(self, seg_off, seg_task, train=True):
        """Plans and buffers for another packing (train=False: of a serving step, which keeps nothing for backward)."""
        T, d, f, dev, edt = int(seg_off[-1]), self.d, self.f, self.dev, self.edt
        self.T, self.train, self.packing = T, train, (seg_off, seg_task, train)
        self.p_gu = lobra.Plan(self.dtype, T, d, 2 * f, self.rank_off2, seg_off, seg_task, n_proj=2)
        self.p_down = lobra.Plan(self.dtype, T, f, d, self.rank_off, seg_off, seg_task)
        self.p_head = lobra.Plan(self.dtype, T, d, self.vocab, None, [0, T], [-1])
        plans = (self.p_gu, self.p_down, self.p_head)
        need = [p.fwd_ws_bytes for p in plans] + [lobra.lobra_mlora_gated_workspace_bytes(self.p_gu, train), 16]
        if self.head8 is not None:
            need += [n[k] for n in (lobra.lobra_mlora_quant_workspace_bytes(p) for p in (self.p_down, self.p_head)) for k in ((0, 1) if train else (0,))]
        if train:
            need += [p.bwd_ws_bytes for p in plans] + [self.grads.ws_bytes, lobra.lobra_mlora_block_norm_workspace_bytes(self.p_gu)]
        self.ws = torch.empty(max(need), dtype=torch.uint8, device=dev)

        def buf(*shape, dtype=edt):
            return torch.empty(*shape, dtype=dtype, device=dev)

        kept = self.layers if train else 1            # (serving: one block's buffers, used again by the next)
        self.act = [{"x": buf(T, d), "h": buf(T, f), "b": buf(T, d), "r": buf(T, d),
                     "gu": buf(T, 2 * f) if train else None,
                     "rstd_post": buf(T, dtype=torch.float32) if train else None,
                     "rstd_pre": buf(T, dtype=torch.float32) if train else None,
                     "h_gu": buf(self.p_gu.h_save_bytes, dtype=torch.uint8) if train else None,
                     "h_down": buf(self.p_down.h_save_bytes, dtype=torch.uint8) if train else None} for _ in range(kept)]
        self.x_out = buf(T, d)
        self.logits = buf(T, self.vocab)
        self.logp, self.lse, self.lse_rest, self.entropy = (buf(T, dtype=torch.float32) for _ in range(4))
        self.loss, self.stat = buf(T, dtype=torch.float32), buf(T, 4, dtype=torch.float32)
        if train:
            self.dr, self.dx, self.dh = buf(T, d), buf(T, d), buf(T, f)

    def forward(self, tokens, target=None, top=None, teacher=None):
        """logp [T] of target (int32 [T]; outside the vocabulary: not counted).  top = (logp [T, k], id [T, k]): receives the likeliest.
        teacher = (logp [T, k], id [T, k]), another model's likeliest: the loss [T] against them instead, what they leave out as one more token."""
        self.logits_of(tokens)
        lo = lobra
        if teacher is not None:
            desc = lo.make_distill_desc(self.dtype, self.T, self.vocab, teacher[0].shape[1], tail=True)
            lo.lobra_token_distill_fwd(desc, self.logits, *teacher, self.loss, self.stat)
            return self.loss
        desc = lo.make_logprob_desc(self.dtype, self.T, self.vocab, top_k=0 if top is None else top[0].shape[1])
        lo.lobra_token_logprob_fwd(desc, self.logits, target, self.logp, self.lse, self.lse_rest, self.entropy, *(top or (None, None)))
        return self.logp

    def logits_of(self, tokens):
        lo = lobra
        r = self.embedding.index_select(0, tokens)
        for l, blk in enumerate(self.blocks):
            a = self.act[l if self.train else 0]
            if l == 0:
                lo.lobra_mlora_block_norm_fwd(self.p_gu, self.cfg, r, None, None, None, self.gain, None, a["x"])
            x_next = self.x_out if l + 1 == self.layers else self.act[l + 1 if self.train else 0]["x"]
            lo.lobra_mlora_gated_fwd(self.p_gu, lo.ACT_SILU, a["x"], blk["W_gu"], blk["A_gu"], blk["B_gu"], self.s, a["gu"], a["h"], a["h_gu"], self.ws)
            self._fwd(self.p_down, a["h"], blk.get("W_down"), blk.get("W_down8"), blk["A_down"], blk["B_down"], self.s, a["b"], a["h_down"])
            lo.lobra_mlora_block_norm_fwd(self.p_gu, self.cfg, r, a["b"], self.gain, blk["gate"], self.gain, a["r"], x_next,
                                          a["rstd_post"], a["rstd_pre"])
            r = a["r"]
        self._fwd(self.p_head, self.x_out, self.head, self.head8, None, None, None, self.logits, None)

    def backward(self, target, dlogp, teacher=None):
        """Gradients of sum(dlogp * logp), or with the teacher that forward had of sum(dlogp * loss), into every block's dA_*, dB_*, dgate.  The logits'
        gradient takes the logits' place."""
        lo = lobra
        if teacher is not None:
            desc = lo.make_distill_desc(self.dtype, self.T, self.vocab, teacher[0].shape[1], tail=True)
            lo.lobra_token_distill_bwd(desc, self.logits, *teacher, self.stat, dlogp, self.logits)
        else:
            desc = lo.make_logprob_desc(self.dtype, self.T, self.vocab)
            lo.lobra_token_logprob_bwd(desc, self.logits, target, self.lse, self.lse_rest, None, dlogp, None, self.logits)
        self._bwd(self.p_head, self.x_out, self.head, self.head8, None, None, None, self.logits, None, self.dx, None, None)
        dr = None
        for l in reversed(range(self.layers)):
            blk, a = self.blocks[l], self.act[l]
            db = self.dx                                      # (each element is read before it is written)
            lo.lobra_mlora_block_norm_bwd(self.p_gu, self.cfg, a["r"], a["b"], self.gain, blk["gate"], self.gain, a["rstd_post"], a["rstd_pre"],
                                          dr, self.dx, self.dr, db, blk["dgate"], None, None, 0, self.ws)
            dr = self.dr
            self._bwd(self.p_down, a["h"], blk.get("W_down"), blk.get("W_down8"), blk["A_down"], blk["B_down"], self.s, db, a["h_down"], self.dh,
                      blk["dA_down"], blk["dB_down"])
            lo.lobra_mlora_gated_bwd(self.p_gu, lo.ACT_SILU, a["x"], blk["W_gu"], blk["A_gu"], blk["B_gu"], self.s, a["gu"], self.dh, a["h_gu"],
                                     a["gu"], self.dx if l else None, blk["dA_gu"], blk["dB_gu"], 0 if l else lo.FLAG_NO_DX, self.ws)

    def update(self):
        """Clips every task's gradients to its max_norm and takes a step: Adam for the adapters, plain descent for the gates.  A task whose norm is
        not finite is left out: its parameters, moments and count stay."""
        torch.add(self.steps, 1, out=self.step_now)
        lobra.lobra_grad_clip(self.grads, self.max_norm, None, self.step_now, self.norm, self.clip_scale, self.step_now, 0, self.ws)
        self.steps += self.step_now > 0               # (a task that is left out has not taken its step)
        for blk in self.blocks:
            for name, plan in (("gu", self.p_gu), ("down", self.p_down)):
                a, b = "A_" + name, "B_" + name
                lobra.lobra_mlora_adam_step(plan, self.adam, self.lr, self.step_now, self.clip_scale, blk["d" + a], blk["d" + b],
                                            blk["master_" + a], blk["master_" + b], blk["m_" + a], blk["v_" + a], blk["m_" + b], blk["v_" + b],
                                            blk[a], blk[b])
            scale = self.clip_scale[:, None]
            blk["gate32"] -= torch.where(scale > 0, LR_GATE * scale * blk["dgate"], 0.0)
            blk["gate"].copy_(blk["gate32"])


    def search(self, tokens, tasks, beams, new_tokens, end=-1):
        """Beam search from one token per request: (scores [n, beams], tokens [n, beams, new_tokens]), the best first.  A beam that has come to the token
        `end` is finished; what follows it is `end` again.  The batch is a serving one from here on."""
        n, lo = len(tasks), lobra
        self.batch([beams * i for i in range(n + 1)], tasks, train=False)
        desc = lo.make_beam_desc(self.dtype, n, beams, self.vocab)
        ws = torch.empty(lo.lobra_beam_workspace_bytes(desc), dtype=torch.uint8, device=self.dev)
        score = torch.full((n, beams), -math.inf, device=self.dev)
        score[:, 0] = 0.0                             # one beam to begin with
        parent, token = (torch.empty(n, beams, dtype=torch.int32, device=self.dev) for _ in range(2))
        seen = torch.zeros(n * beams, new_tokens, dtype=torch.int32, device=self.dev)
        done = torch.zeros(n * beams, 1, dtype=torch.int32, device=self.dev)
        now = tokens.repeat_interleave(beams)
        for k in range(new_tokens):
            self.logits_of(now)
            lo.lobra_beam_select(desc, self.logits, score, done.view(n, beams), end, score, parent, token, ws)
            lo.lobra_beam_reorder([(seen, seen), (done, done)], n, beams, parent)
            seen[:, k] = token.view(-1)
            done |= token.view(-1, 1) == end
            now = token.view(-1).long().clamp(min=0)
        return score, seen.view(n, beams, new_tokens)


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--dtype", choices=("bf16", "f32"), default="bf16")
    ap.add_argument("--steps", type=int, default=30)
    ap.add_argument("--layers", type=int, default=2)
    ap.add_argument("--width", type=int, default=512)
    ap.add_argument("--ffn", type=int, default=1408)
    ap.add_argument("--vocab", type=int, default=1000)
    ap.add_argument("--tokens", type=int, default=600, help="per task")
    ap.add_argument("--ranks", type=int, nargs="+", default=[8, 16, 8])
    ap.add_argument("--new-tokens", type=int, default=5)
    ap.add_argument("--distill-steps", type=int, default=0, help="steps of new adapters on an 8-bit base, against the trained model's likeliest tokens")
    ap.add_argument("--beams", type=int, default=0, help="continue the prompts by beam search")
    args = ap.parse_args(argv)
    why = not_8_bits(args.dtype, args.width, args.ffn) if args.distill_steps else None
    if why:
        ap.error("--distill-steps: " + why)
    if not 0 <= args.beams <= lobra.MAX_TOP:
        ap.error("--beams: 0 to %d" % lobra.MAX_TOP)
    n, T = len(args.ranks), len(args.ranks) * args.tokens
    gen = torch.Generator().manual_seed(1)
    # every task has a map of its own from a token to the next, over the tokens that occur
    occur = min(args.vocab, 64)
    maps = [torch.randperm(occur, generator=gen) for _ in range(n)]
    seg_off, seg_task = [t * args.tokens for t in range(n + 1)], list(range(n))
    step = JointStep(args.dtype, args.width, args.ffn, args.vocab, args.layers, args.ranks, seg_off, seg_task)
    task = torch.arange(n).repeat_interleave(args.tokens)
    used = torch.randint(occur, (T,), generator=gen)
    target = torch.stack([m[used] for m in maps])[task, torch.arange(T)].int().to(step.dev)
    tokens = used.to(step.dev)
    dlogp = torch.full((T,), -1.0 / args.tokens, device=step.dev)
    losses = []
    for k in range(args.steps):
        logp = step.forward(tokens, target)
        step.backward(target, dlogp)
        step.update()
        losses.append((-logp.view(n, args.tokens).mean(dim=1)).tolist())
        if k % 5 == 0 or k + 1 == args.steps:
            print("step %3d  losses %s  gradient norms %s" % (k, ["%.3f" % v for v in losses[-1]], ["%.3f" % v for v in step.norm.tolist()]), flush=True)
    if args.distill_steps:
        # what the model thinks likeliest, as the teacher of new adapters on an 8-bit base
        teacher = torch.empty(T, 16, device=step.dev), torch.empty(T, 16, dtype=torch.int32, device=step.dev)
        step.forward(tokens, target, teacher)
        step.quantise_base()
        step.restart()
        weight = torch.full((T,), 1.0 / args.tokens, device=step.dev)
        for k in range(args.distill_steps):
            loss = step.forward(tokens, teacher=teacher)
            step.backward(None, weight, teacher)
            step.update()
            if k % 5 == 0 or k + 1 == args.distill_steps:
                print("8-bit base, step %3d  losses %s" % (k, ["%.5f" % v for v in loss.view(n, args.tokens).mean(dim=1).tolist()]), flush=True)
    if args.beams:
        score, seen = step.search((torch.arange(n) % occur).to(step.dev), list(range(n)), args.beams, args.new_tokens)
        for t in range(n):
            for b in range(args.beams):
                print("task %d: %4d -> %s (%.2f)" % (t, t % occur, " ".join("%4d" % v for v in seen[t, b].tolist()), float(score[t, b])), flush=True)
    # one token per task at a time, all tasks in one call
    step.batch(list(range(n + 1)), list(range(n)), train=False)
    tokens = (torch.arange(n) % occur).to(step.dev)
    top = torch.empty(n, 3, device=step.dev), torch.empty(n, 3, dtype=torch.int32, device=step.dev)
    for _ in range(args.new_tokens):
        step.forward(tokens, None, top)
        now, nxt = tokens.tolist(), top[1].tolist()
        for t in range(n):
            print("task %d: %4d -> %s" % (t, now[t], "  ".join("%4d (%.2f)" % p for p in zip(nxt[t], top[0][t].exp().tolist()))), flush=True)
        tokens = top[1][:, 0].long()
    return losses


if __name__ == "__main__":
    main()
