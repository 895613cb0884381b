"""What the calls that are made in C++ allocate is seen by torch: dispatch modes meet it, and where deterministic
algorithms are to find fresh memory filled it is."""
import pytest
import torch
from torch.utils._python_dispatch import TorchDispatchMode

from paper_2609_35587_amd import hwsel

pytestmark = pytest.mark.gpu


class Seen(TorchDispatchMode):
    def __init__(self):
        super().__init__()
        self.made = []

    def __torch_dispatch__(self, func, types, args=(), kwargs=None):
        out = func(*args, **(kwargs or {}))
        if func.overloadpacket is torch.ops.aten.empty:
            self.made.append(out)
        return out


def calls():
    x = torch.randn(5, 300, device="cuda")
    s, seg = torch.randn(90, device="cuda"), torch.tensor([0, 30, 90], device="cuda")
    picks = torch.zeros(2, 3, dtype=torch.int32, device="cuda")
    _, entropy, norm, _, _ = hwsel.hwsel_logprob_per_problem(s, seg, picks)
    d = torch.ones(2, 3, device="cuda")
    long = torch.randn(2 * 100_000, device="cuda")
    return dict(
        sample=lambda: hwsel.hwsel_sample_per_problem(s, seg, torch.full((2, 4), 0.5, device="cuda")),
        logprob=lambda: hwsel.hwsel_logprob_per_problem(s, seg, picks, top=2),
        in_parts=lambda: hwsel.hwsel_logprob_per_problem(long, torch.tensor([0, 100_000, 200_000], device="cuda"), top=2),
        logprob_gradient=lambda: (hwsel.hwsel_logprob_gradient(s, seg, norm, picks, d),),
        dropout=lambda: (hwsel.hwsel_dropout(x, 0.5),),
        join=lambda: hwsel.hwsel_block_join({}, x, x),
        join_gradient=lambda: tuple(t for t in hwsel.hwsel_block_join_gradient({}, x, x, d_x1=x) if t is not None))


@pytest.mark.parametrize("name", ["sample", "logprob", "in_parts", "logprob_gradient", "dropout", "join", "join_gradient"])
def test_a_dispatch_mode_sees_results(name):
    call = calls()[name]
    want = call()
    with Seen() as seen:
        got = call()
    made = {t.data_ptr() for t in seen.made}
    results = [t for t in got if t is not None]
    assert results and all(t.data_ptr() in made for t in results)
    assert all(torch.equal(a, b) for a, b in zip(want, got) if a is not None)


def test_a_dispatch_mode_sees_8_bit_matrices():
    x = torch.randn(5, 300, device="cuda")
    m = hwsel.hwsel_fp8_quantise(x)
    with Seen() as seen:
        hwsel.hwsel_fp8_dequantise(m)
    assert any(tuple(t.shape) == (5, 300) for t in seen.made)


def test_fresh_memory_is_filled_where_torch_fills():
    x = torch.randn(4, 3000, device="cuda")
    want = hwsel.hwsel_dropout(x, 0.5, seed=3)

    def events():
        with torch.profiler.profile(activities=[torch.profiler.ProfilerActivity.CPU]) as p:
            assert torch.equal(hwsel.hwsel_dropout(x, 0.5, seed=3), want)
        return [e.key for e in p.key_averages()]

    assert "aten::fill_" not in events()
    torch.use_deterministic_algorithms(True)
    try:
        assert torch.utils.deterministic.fill_uninitialized_memory
        assert "aten::fill_" in events()
        torch.utils.deterministic.fill_uninitialized_memory = False
        assert "aten::fill_" not in events()
    finally:
        torch.utils.deterministic.fill_uninitialized_memory = True
        torch.use_deterministic_algorithms(False)
