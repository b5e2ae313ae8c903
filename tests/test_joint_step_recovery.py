"""The joint step on an 8-bit base, taught by likeliest tokens and answering by beam search: all calls together against 64 bits.

Tolerance as in bf16 without it: some 15 tensors rounded to 2^-8 of themselves at most lie between the embedding and a gradient of the first block and
back, 6e-2 of a tensor's largest; the whole numbers that tokens become are those of the same roundings, one in 127 of a token's largest off at most
where they differ."""
import math

import pytest

torch = pytest.importorskip("torch")
from test_joint_step import close  # noqa: E402

pytestmark = pytest.mark.gpu


def rounded(v, dim):
    """v as whole multiples of 127 steps, its gradient as if it were v."""
    step = (v.detach().abs().amax(dim=dim, keepdim=True) / 127).float().double()
    q = torch.where(step > 0, (v / torch.where(step > 0, step, 1.0)).round() * step, 0.0)
    return v + (q - v).detach()


def make(T=450):
    from paper_2509_01193_amd.joint_step import JointStep
    seg_off, seg_task = [0, 170, 300, 310, T], [1, 0, -1, 1]
    step = JointStep("bf16", 256, 384, 1000, 2, [8, 16], seg_off, seg_task)
    gen = torch.Generator().manual_seed(4)
    for blk in step.blocks:
        for k in ("B_gu", "B_down"):
            blk[k].copy_(torch.randn(blk[k].shape, generator=gen) * 0.1)
        blk["gate"].copy_(torch.randn(blk["gate"].shape, generator=gen))
    return step, gen, seg_off, seg_task


def test_gradients_of_the_loss_against_a_teacher_on_an_8_bit_base():
    step, gen, seg_off, seg_task = make()
    T, n, d, f, up = step.T, step.n_tasks, step.d, step.f, lambda t: t.detach().double().cpu()
    tokens = torch.randint(1000, (T,), generator=gen).cuda()
    weights = [up(b["W_down"]) for b in step.blocks], up(step.head)
    teacher = torch.empty(T, 12, device="cuda"), torch.empty(T, 12, dtype=torch.int32, device="cuda")
    step.forward(tokens, None, teacher)
    teacher[0].add_(0.3 * torch.randn(T, 12, generator=gen).cuda() - 0.5)            # (another model's, not the own)
    teacher[1][7] = -1
    step.quantise_base()
    dloss = torch.randn(T, generator=gen).cuda()
    got = step.forward(tokens, teacher=teacher).clone()
    step.backward(None, dloss, teacher)
    torch.cuda.synchronize()

    task = torch.full((T,), -1)
    for i, t in enumerate(seg_task):
        task[seg_off[i]:seg_off[i + 1]] = t
    norm = lambda v: v / torch.sqrt((v * v).mean(dim=1, keepdim=True) + 1e-5)

    def adapted(x, y, A, B, off, parts):
        for t in range(n):
            a, b = A[off[t]:off[t + 1]].chunk(parts), B[off[t]:off[t + 1]].chunk(parts)
            y = y + torch.cat([(x @ ai.T) @ bi for ai, bi in zip(a, b)], dim=1) * (2.0 * (task == t).double()[:, None])
        return y

    r, leaves = up(step.embedding)[tokens.cpu()], []
    for blk, W in zip(step.blocks, weights[0]):
        p = {k: up(blk[k]).requires_grad_() for k in ("A_gu", "B_gu", "A_down", "B_down", "gate")}
        leaves.append(p)
        x = norm(r)
        gu = adapted(x, x @ up(blk["W_gu"]), p["A_gu"], p["B_gu"], step.rank_off2, 2)
        h = torch.nn.functional.silu(gu[:, :f]) * gu[:, f:]
        b = adapted(h, rounded(h, 1) @ rounded(W, 0), p["A_down"], p["B_down"], step.rank_off, 1)
        r = r + torch.cat([p["gate"], torch.ones(1, d, dtype=torch.float64)])[task] * norm(b)
    lp = torch.log_softmax(rounded(norm(r), 1) @ rounded(weights[1], 0), dim=1)
    ids, q = teacher[1].cpu().long().clamp(min=0), teacher[0].double().cpu().exp()
    listed = torch.zeros_like(lp, dtype=torch.bool).scatter(1, ids, True)
    qr = 1 - q.sum(dim=1)
    rest = torch.logsumexp(lp.masked_fill(listed, -math.inf), dim=1)
    tail = torch.where(qr > 2.0 ** -20, qr.clamp(min=1e-9) * (qr.clamp(min=1e-9).log() - rest), 0.0)
    loss = (q * (q.log() - lp.gather(1, ids))).sum(dim=1) + tail
    loss = torch.where(torch.arange(T) == 7, 0.0, loss)
    (loss * dloss.double().cpu()).sum().backward()
    close(got, loss.detach(), "loss", 6e-2)
    for i, (blk, p) in enumerate(zip(step.blocks, leaves)):
        for k, v in p.items():
            close(blk["d" + k], v.grad, "block %d, d%s" % (i, k), 6e-2)


@pytest.mark.parametrize("base8", [False, True])
def test_beam_search(base8):
    """Against beam search over the table of the model's own answers to every token (a token's answer depends on nothing else)."""
    step, gen, _, _ = make()
    if base8:
        step.quantise_base()
    V, beams, new, tasks, start = 1000, 3, 4, [1, 0], torch.tensor([17, 400])
    score, seen = step.search(start.cuda(), tasks, beams, new, end=5)
    table = []
    for t in tasks:
        step.batch([0, V], [t], train=False)
        step.logits_of(torch.arange(V).cuda())
        table.append(torch.log_softmax(step.logits.double().cpu(), dim=1))
    for i in range(2):
        lp, live = table[i], [(0.0, [int(start[i])])]
        for _ in range(new):
            nxt = []
            for s, path in live:
                if path[-1] == 5 and len(path) > 1:
                    nxt.append((s, path + [5]))
                else:
                    nxt += [(s + float(lp[path[-1], j]), path + [j]) for j in lp[path[-1]].topk(beams + 1).indices.tolist()]
            live = sorted(nxt, key=lambda c: -c[0])[:beams]
        own = []
        for b in range(beams):
            path, s = [int(start[i])] + seen[i, b].tolist(), 0.0
            for a, c in zip(path, path[1:]):
                s += 0.0 if a == 5 else float(lp[a, c])
            own.append(s)
            # logits rounded to bf16 in one batch and in another: 2^-8 of up to 8, in every step
            assert abs(s - float(score[i, b])) <= new * 2 * 8 * 2.0 ** -8, (path, s, float(score[i, b]))
        for b in range(beams):
            assert abs(own[b] - live[b][0]) <= new * 2 * 8 * 2.0 ** -8 * 2, (own, live)


def test_the_command_runs(capsys):
    from paper_2509_01193_amd import joint_step
    joint_step.main(["--steps", "2", "--distill-steps", "2", "--beams", "3", "--width", "128", "--ffn", "256", "--tokens", "40", "--vocab", "200", "--new-tokens", "3"])
    out = capsys.readouterr().out
    assert out.count("8-bit base") == 2 and out.count("task 1:") == 3 + 3
