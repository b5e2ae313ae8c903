"""The calls on an 8-bit base, a teacher's tokens and beams refuse every tensor that does not lie where they are launched, each one by itself: nothing
here gets as far as a launch."""
import pytest

from paper_2509_01193_amd import binding as bd

torch = pytest.importorskip("torch")


class OnDevice(torch.Tensor):
    """A host tensor that says it lies on a device."""
    index = 0

    def get_device(self):
        return self.index


class OnAnother(OnDevice):
    index = 1


def calls():
    """(name, function, tensors by argument, other arguments); what is a list of pairs is one argument a tensor: src0, dst0, ..."""
    z = lambda *s, dt=torch.float32: torch.zeros(*s, dtype=dt)
    b16, i32, u8 = torch.bfloat16, torch.int32, torch.uint8
    plan = bd.Plan("bf16", 8, 64, 64, [0, 8, 24], [0, 4, 8], [0, 1], flags=bd.PLAN_HOST_ONLY)
    plan.host_only = False                           # (as one that runs)
    q8 = dict(x=z(8, 64, dt=b16), Wq=z(64, 256, dt=torch.int8), w_scale=z(64), A=z(24, 64, dt=b16), B=z(24, 64, dt=b16), s=z(2))
    ws, h = z(1 << 17, dt=u8), z(plan.h_save_bytes, dt=u8)
    dd, bm = bd.make_distill_desc("bf16", 3, 100, 5), bd.make_beam_desc("bf16", 1, 3, 100)
    t = dict(logits=z(3, 100, dt=b16), teacher_logp=z(3, 5), teacher_id=z(3, 5, dt=i32))
    states = {k + str(i): z(3, 4 + i) for i in range(3) for k in ("src", "dst")}

    def reorder(n_req, beams, parent, used=None, **kw):
        n = [k[3:] for k in kw if k.startswith("src")]
        bd.lobra_beam_reorder([(kw["src" + i], kw["dst" + i]) for i in n], n_req, beams, parent, used, stream=kw["stream"])

    return [
        ("quantise_weight", bd.lobra_quantise_weight, dict(W=z(8, 16), Wq=z(16, 256, dt=torch.int8), w_scale=z(16)), {}),
        ("quant_fwd", bd.lobra_mlora_quant_fwd, dict(q8, y=z(8, 64, dt=b16), h_save=h, ws=ws), dict(plan=plan)),
        ("quant_bwd", bd.lobra_mlora_quant_bwd, dict(q8, dy=z(8, 64, dt=b16), h_saved=h, dx=z(8, 64, dt=b16), dA=z(24, 64), dB=z(24, 64), ws=ws), dict(plan=plan)),
        ("distill_fwd", bd.lobra_token_distill_fwd, dict(t, loss=z(3), stat=z(3, 4)), dict(desc=dd)),
        ("distill_bwd", bd.lobra_token_distill_bwd, dict(t, stat=z(3, 4), dloss=z(3), dlogits=z(3, 100, dt=b16)), dict(desc=dd)),
        ("beam_select", bd.lobra_beam_select, dict(logits=z(3, 100, dt=b16), score=z(1, 3), done=z(1, 3, dt=i32), out_score=z(1, 3), out_beam=z(1, 3, dt=i32),
                                                   out_token=z(1, 3, dt=i32), ws=z(4096, dt=u8)), dict(desc=bm, done_token=2)),
        ("beam_reorder", reorder, dict(states, parent=z(1, 3, dt=i32), used=z(1, dt=i32)), dict(n_req=1, beams=3)),
    ]


CASES = [(c[0], k) for c in calls() for k in c[2]]


@pytest.mark.parametrize("name,operand", CASES, ids=["%s-%s" % c for c in CASES])
def test_one_operand_elsewhere(name, operand, monkeypatch):
    monkeypatch.setattr(bd, "_current_device", lambda: 0)
    _, call, tensors, other = next(c for c in calls() if c[0] == name)
    there = {k: v.as_subclass(OnDevice) for k, v in tensors.items()}
    with pytest.raises(AssertionError, match="host tensor"):
        call(**{**there, operand: tensors[operand]}, **other, stream=0)
    with pytest.raises(AssertionError, match="different devices"):
        call(**{**there, operand: tensors[operand].as_subclass(OnAnother)}, **other, stream=0)


@pytest.mark.parametrize("name", [c[0] for c in calls()])
def test_all_operands_on_another_device(name, monkeypatch):
    monkeypatch.setattr(bd, "_current_device", lambda: 0)
    _, call, tensors, other = next(c for c in calls() if c[0] == name)
    with pytest.raises(AssertionError, match="another device than the current one"):
        call(**{k: v.as_subclass(OnAnother) for k, v in tensors.items()}, **other, stream=0)


def test_types_are_looked_at_first():
    """What is of another type or too short is said to be that, wherever it lies."""
    for name, operand, bad, what in (("distill_fwd", "teacher_logp", lambda t: t.double(), "float64"), ("distill_bwd", "dloss", lambda t: t[:2], "2 elements"),
                                     ("beam_select", "out_token", lambda t: t[:, :2].contiguous(), "2 elements"), ("quant_fwd", "A", lambda t: t[:23], "elements")):
        _, call, tensors, other = next(c for c in calls() if c[0] == name)
        with pytest.raises(AssertionError, match=what):
            call(**{**tensors, operand: bad(tensors[operand])}, **other, stream=0)
