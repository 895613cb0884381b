"""Calls of log probabilities, dropout and joins: what they refuse with device
tensors in hand, streams of their own, captured graphs, results' places."""
import pytest
import torch

import test_gpu_foreign_streams as eight
from paper_2609_35587_amd import hwsel

pytestmark = pytest.mark.gpu


def x(rows=6, cols=200, dtype=torch.float32, seed=0):
    g = torch.Generator(device="cuda").manual_seed(rows * 1000 + cols + seed)
    return torch.randn(rows, cols, generator=g, device="cuda").to(dtype)


SEG = (0, 40, 100)


def scored():
    return x(1, 100).flatten(), torch.tensor(SEG, device="cuda"), torch.zeros(2, 3, dtype=torch.int32, device="cuda")


def test_log_probabilities_refuse():
    s, seg, picks = scored()
    call = lambda **kw: hwsel.hwsel_logprob_per_problem(**{**dict(scores=s, seg_offsets=seg, picks=picks, top=4), **kw})  # noqa: E731
    call()
    two, n = torch.ones(2, device="cuda"), lambda *k: torch.zeros(*k, device="cuda")  # noqa: E731
    for kw in (dict(scores=s.double()), dict(scores=s.cpu()), dict(scores=s[::2]), dict(scores=None), dict(seg_offsets=seg.int()),
               dict(seg_offsets=seg[:1]), dict(picks=picks.long()), dict(picks=picks[:1]), dict(picks=picks.flatten()), dict(picks=picks.cpu()),
               dict(picks=picks.t().contiguous().t()), dict(temperature=two[:1]), dict(temperature=two.double()), dict(logp=n(5)),
               dict(entropy=n(1)), dict(entropy=n(2).double()), dict(norm=n(3)), dict(top_idx=n(2, 4)), dict(top_logp=n(7)), dict(workspace=n(4))):
        with pytest.raises(ValueError):
            call(**kw)
    for kw in (dict(top=2.5), dict(temperature="hot"), dict(temperature=None)):
        with pytest.raises(TypeError):
            call(**kw)
    for top in (-1, 65):
        with pytest.raises(hwsel.HwselError):
            call(top=top)
    with pytest.raises(ValueError):
        call(top=1 << 40)


def test_gradient_refuses():
    s, seg, picks = scored()
    logp, entropy, norm, _, _ = hwsel.hwsel_logprob_per_problem(s, seg, picks)
    d, de = torch.ones(2, 3, device="cuda"), torch.ones(2, device="cuda")
    call = lambda **kw: hwsel.hwsel_logprob_gradient(**{**dict(scores=s, seg_offsets=seg, norm=norm, picks=picks, d_logp=d, entropy=entropy, d_entropy=de), **kw})  # noqa: E731
    call()
    for kw in (dict(norm=norm[:1]), dict(norm=norm.double()), dict(norm=None), dict(d_logp=None), dict(picks=None), dict(d_logp=d[:1]),
               dict(d_logp=d.double()), dict(entropy=entropy[:1]), dict(d_entropy=de.cpu()), dict(out=torch.zeros(99, device="cuda")),
               dict(out=torch.zeros(100, device="cuda").double())):
        with pytest.raises(ValueError):
            call(**kw)
    with pytest.raises(hwsel.HwselError):
        call(entropy=None)


def test_dropout_refuses():
    a = x()
    for kw in (dict(x=a.cpu()), dict(x=a.double()), dict(x=a.half()), dict(x=a[0]), dict(x=a.t()), dict(x=a[:, ::2]), dict(x=a[:0]), dict(x=None),
               dict(x=a[:1].expand(6, 200)), dict(x=a.flatten().unfold(0, 200, 7)), dict(residual=a[:5]), dict(residual=a[:, :199]), dict(residual=x(7)),
               dict(residual=a.cpu()), dict(residual=3.0), dict(out=a[:5]), dict(out=torch.empty(6, 199, device="cuda")), dict(seed=-1), dict(seed=1 << 64),
               dict(offset=-5), dict(state=torch.zeros(1, dtype=torch.int64, device="cuda")), dict(state=torch.zeros(2, device="cuda"))):
        with pytest.raises(ValueError):
            hwsel.hwsel_dropout(**{**dict(x=a, p=0.5), **kw})
    for p in (-0.1, 1.5, float("nan")):
        with pytest.raises(hwsel.HwselError):
            hwsel.hwsel_dropout(a, p)
    with pytest.raises(hwsel.HwselError):                   # results and residual have one type
        hwsel.hwsel_dropout(a, 0.5, residual=a, out=torch.empty(6, 200, dtype=torch.bfloat16, device="cuda"))
    for kw in (dict(p="half"), dict(seed=1.5), dict(seed="one")):
        with pytest.raises(TypeError):
            hwsel.hwsel_dropout(**{**dict(x=a, p=0.5), **kw})


def test_joins_refuse():
    a, w = x(), torch.ones(200, device="cuda")
    join = dict(post_norm=True, w_branch=w, w_pre=w)
    x1, _ = hwsel.hwsel_block_join(join, a, a)
    forward = lambda j=join, **kw: hwsel.hwsel_block_join(**{**dict(join=j, x=a, y=a), **kw})  # noqa: E731
    backward = lambda j=join, **kw: hwsel.hwsel_block_join_gradient(**{**dict(join=j, x1=x1, y=a, d_x1=a, d_z=a), **kw})  # noqa: E731
    for call in (forward, backward):
        for j in (None, 3, [], {**join, "w_brunch": w}, {**join, "w_pre": w[:199]}, {**join, "w_branch": w.bfloat16()}, {**join, "seed": -1},
                  {**join, "state": w}):
            with pytest.raises(ValueError):
                call(j)
        for j in ({**join, "eps": 0.0}, {**join, "eps": float("nan")}, {**join, "p": 2.0}, {**join, "stream_scale": float("inf")}):
            with pytest.raises(hwsel.HwselError):
                call(j)
        for j in ({**join, "eps": "small"}, {**join, "seed": 0.5}):
            with pytest.raises(TypeError):
                call(j)
        for kw in (dict(y=a[:5]), dict(y=a.cpu()), dict(y=a.half()), dict(y=a.t()), dict(gate=a[:, :2]), dict(gate=a[:5]), dict(gate=a[0]),
                   dict(gate=a[:1].expand(6, 200))):
            with pytest.raises(ValueError):
                call(**kw)
        with pytest.raises(hwsel.HwselError):               # the block's matrices have one type
            call(gate=a.bfloat16())
        with pytest.raises(hwsel.HwselError):               # a weight of the branch without one
            call(y=None)
    for kw in (dict(x=a.cpu()), dict(x=a.half()), dict(x1=a[:5]), dict(z=a[:, :100]), dict(dtype=torch.float16), dict(dtype="bf16")):
        with pytest.raises(ValueError):
            forward(**kw)
    for kw in (dict(with_x1=False, with_z=False), dict(x1=torch.empty(6, 200, dtype=torch.bfloat16, device="cuda")), dict(dtype=torch.bfloat16)):
        with pytest.raises(hwsel.HwselError):
            forward(**kw)
    n = hwsel.hwsel_block_join_gradient_workspace_bytes(6, 200)
    for kw in (dict(d_x1=a[:5]), dict(d_z=a[:, :5]), dict(dx=a[:5]), dict(dy=a[:5]), dict(dw_branch=w[:5]), dict(dw_pre=w.double()),
               dict(workspace=torch.zeros(n, device="cuda"))):
        with pytest.raises(ValueError):
            backward(**kw)
    for kw in (dict(d_x1=None, d_z=None), dict(d_z=a.bfloat16()), dict(workspace=torch.zeros(n - 1, dtype=torch.uint8, device="cuda")),
               dict(workspace=torch.zeros(n + 1, dtype=torch.uint8, device="cuda")[1:])):
        with pytest.raises(hwsel.HwselError):
            backward(**kw)


@pytest.fixture(scope="module")
def data():
    g = torch.Generator(device="cuda").manual_seed(1)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    d = dict(x=r(300, 1100), y=r(300, 1100).bfloat16(), gate=r(300, 1100).bfloat16(), dx=r(300, 1100), dz=r(300, 1100).bfloat16(),
             scores=r(3 * 200_000), seg=torch.arange(4, device="cuda") * 200_000, dl=r(3, 8), de=r(3),
             picks=torch.randint(0, 200_000, (3, 8), generator=g, device="cuda", dtype=torch.int32),
             big=torch.empty(1024 * eight.MB, dtype=torch.uint8, device="cuda"))
    w = lambda: 1 + 0.1 * r(1100)  # noqa: E731
    d["join"] = dict(post_norm=True, gate_sigmoid=True, w_branch=w(), w_pre=w(), p=0.3, seed=5)
    _, d["entropy"], d["norm"], _, _ = hwsel.hwsel_logprob_per_problem(d["scores"], d["seg"])
    assert hwsel.hwsel_logprob_workspace_bytes(600_000, 3, 9) > 0
    return d


CALLS = {
    "log probabilities": lambda d, s: hwsel.hwsel_logprob_per_problem(d["scores"], d["seg"], d["picks"], top=9, stream=s),
    "their gradient": lambda d, s: hwsel.hwsel_logprob_gradient(d["scores"], d["seg"], d["norm"], d["picks"], d["dl"], d["entropy"], d["de"], stream=s),
    "dropout": lambda d, s: hwsel.hwsel_dropout(d["y"], 0.2, 3, 4, residual=d["x"], stream=s),
    "join": lambda d, s: hwsel.hwsel_block_join(d["join"], d["x"], d["y"], d["gate"], stream=s),
    "join's gradient": lambda d, s: hwsel.hwsel_block_join_gradient(d["join"], d["x"], d["y"], d["gate"], d["dx"], d["dz"], stream=s),
}
WORK = lambda: [hwsel.hwsel_logprob_workspace_bytes(600_000, 3, 9), hwsel.hwsel_block_join_gradient_workspace_bytes(300, 1100)]  # noqa: E731


@pytest.fixture(params=["object", "number"])
def side(request):
    s = torch.cuda.Stream()
    return s, (s if request.param == "object" else s.cuda_stream)


@pytest.mark.parametrize("name", CALLS)
def test_workspace_is_not_handed_on(name, side, data):
    """The current stream allocates and writes while the given one has not begun."""
    call, (s, given) = CALLS[name], side
    want = [t.clone() for t in eight.tensors(call(data, None))]
    torch.cuda.synchronize()
    eight.busy(data, s)
    got = call(data, given)
    held = eight.overwrite(WORK() + [n // 2 for n in WORK()] + eight.sizes(got))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(eight.tensors(got), want))
    assert all(bool((h == 0xff).all()) for h in held)


@pytest.mark.parametrize("name", CALLS)
def test_memory_that_the_current_stream_still_writes(name, side, data):
    call, (s, given) = CALLS[name], side
    result = call(data, None)
    want, bytes_each = [t.clone() for t in eight.tensors(result)], eight.sizes(result)
    del result
    torch.cuda.synchronize()
    eight.busy(data, torch.cuda.current_stream())
    held = eight.overwrite(WORK() + bytes_each)
    del held
    got = call(data, given)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(eight.tensors(got), want))


@pytest.mark.parametrize("name", CALLS)
def test_replayed(name, data):
    """Captured on a stream that the capture has forked to; two graphs of one call in turn, eager calls in between."""
    want = [t.clone() for t in eight.tensors(CALLS[name](data, None))]
    graphs = []
    for _ in range(2):
        side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph):
            main = torch.cuda.current_stream()
            side.wait_stream(main)
            got = eight.tensors(CALLS[name](data, side))
            main.wait_stream(side)
        graphs.append((graph, got))
    for _ in range(3):
        for _, got in graphs:
            for t in got:
                t.zero_()
        for graph, _ in graphs:
            graph.replay()
        eager = eight.tensors(CALLS[name](data, None))
        torch.cuda.synchronize()
        for got in [eager] + [g for _, g in graphs]:
            assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_a_graph_drops_out_anew():
    """The state moves between replays, in the graph itself: each replay has the mask of its own offset."""
    a = x(40, 300, torch.bfloat16)
    state = torch.tensor([11, 0], device="cuda")
    one = torch.tensor([0, 1], device="cuda")
    graph = torch.cuda.CUDAGraph()
    hwsel.hwsel_dropout(a, 0.5, state=state)
    join = dict(p=0.25, state=state)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        state += one
        y = hwsel.hwsel_dropout(a, 0.5, state=state)
        x1, _ = hwsel.hwsel_block_join(join, a, a)
    state.copy_(torch.tensor([11, 0]))
    for turn in range(1, 4):
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, hwsel.hwsel_dropout(a, 0.5, 11, turn))
        assert torch.equal(x1, hwsel.hwsel_block_join(dict(p=0.25, seed=11, offset=turn), a, a)[0])


def test_results_go_where_they_are_wanted():
    s, seg, picks = scored()
    n = lambda *k, t=torch.float32: torch.empty(*k, dtype=t, device="cuda")  # noqa: E731
    out = dict(logp=n(2, 3), entropy=n(2), norm=n(2, 2), top_idx=n(2, 4, t=torch.int32), top_logp=n(2, 4))
    got, want = hwsel.hwsel_logprob_per_problem(s, seg, picks, top=4, **out), hwsel.hwsel_logprob_per_problem(s, seg, picks, top=4)
    assert all(a is b for a, b in zip(got, out.values())) and all(torch.equal(a, b) for a, b in zip(got, want))
    none = hwsel.hwsel_logprob_per_problem(s, seg)
    assert none[0] is None and none[3] is None and none[4] is None and torch.equal(none[1], want[1])
    empty = hwsel.hwsel_logprob_per_problem(s, seg, picks[:, :0])
    assert empty[0] is None and torch.equal(empty[2], want[2])


def test_no_scores():
    """Problems without a row, and no row at all."""
    seg = torch.zeros(4, dtype=torch.int64, device="cuda")
    picks = torch.zeros(3, 2, dtype=torch.int32, device="cuda")
    none = torch.empty(0, device="cuda")
    logp, entropy, norm, idx, lp = hwsel.hwsel_logprob_per_problem(none, seg, picks, top=2)
    assert not bool(logp.any()) and not bool(entropy.any()) and bool((norm == float("-inf")).all()) and bool((idx == -1).all())
    assert hwsel.hwsel_logprob_gradient(none, seg, norm, picks, torch.ones(3, 2, device="cuda")).numel() == 0


def test_two_calls_at_once(data):
    """On two streams, each with memory of its own."""
    want = {n: [t.clone() for t in eight.tensors(c(data, None))] for n, c in CALLS.items()}
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [(n, c(data, s)) for _ in range(3) for n, c in CALLS.items() for s in streams]
    torch.cuda.synchronize()
    for n, r in got:
        assert all(torch.equal(a, b) for a, b in zip(eight.tensors(r), want[n]))
