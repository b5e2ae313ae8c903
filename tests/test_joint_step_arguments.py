"""What the joint step refuses before it has changed, launched or trained anything."""
import pytest

torch = pytest.importorskip("torch")
from paper_2509_01193_amd import binding as bd  # noqa: E402
from paper_2509_01193_amd import joint_step  # noqa: E402


def bare(dtype="f32", d=16, f=24, head8=None):
    """A JointStep's weights without a device."""
    step = object.__new__(joint_step.JointStep)
    step.dtype, step.d, step.f, step.dev, step.head8 = dtype, d, f, torch.device("cpu"), head8
    step.blocks = [{"W_down": torch.ones(f, 4)} for _ in range(2)]
    step.head = torch.ones(4, 8)
    return step


@pytest.mark.parametrize("kw,what", [(dict(), "bf16"), (dict(dtype="bf16", f=bd.MAX_QUANT_IN + 8), "wider"), (dict(dtype="bf16", d=bd.MAX_QUANT_IN + 8), "wider"),
                                     (dict(dtype="bf16", head8=(None, None)), "already")])
def test_a_base_that_is_not_put_into_8_bits_keeps_its_weights(kw, what):
    step = bare(**kw)
    kept = [b["W_down"] for b in step.blocks], step.head
    with pytest.raises(ValueError, match=what):
        step.quantise_base()
    assert all(b["W_down"] is w for b, w in zip(step.blocks, kept[0])) and step.head is kept[1] and step.head8 == kw.get("head8")


@pytest.mark.parametrize("args,what", [
    (["--dtype", "f32", "--distill-steps", "1"], "--distill-steps"), (["--beams", "33"], "--beams"), (["--beams", "-1"], "--beams"),
    (["--ffn", "131080", "--distill-steps", "1"], "--distill-steps"), (["--width", "131080", "--distill-steps", "1"], "--distill-steps"),
])
def test_arguments_that_would_end_a_run_half_way(args, what, capsys):
    with pytest.raises(SystemExit) as e:
        joint_step.main(args)
    assert e.value.code == 2 and what in capsys.readouterr().err
