"""Calls given another stream than torch's current one.  What such a call
allocates must be that stream's: memory that the current stream has freed may
still be in use there, and what the call frees on return is in use on the
given stream until its kernels end.  Either stream is kept busy for some
milliseconds by fills of a large buffer, so that what is unordered overlaps."""
import pytest
import torch

from paper_2609_35587_amd import hwsel

pytestmark = pytest.mark.gpu
MB = 1 << 20


@pytest.fixture(scope="module")
def data():
    g = torch.Generator(device="cuda").manual_seed(1)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    d = dict(x=r(300, 700), a=hwsel.hwsel_fp8_quantise(r(40, 60_000)), b=hwsel.hwsel_fp8_quantise(r(200, 60_000), block_rows=128),
             scores=r(3 * 200_000), seg=torch.arange(4, device="cuda") * 200_000,
             u=torch.rand(3, 8, generator=g, device="cuda"), big=torch.empty(1024 * MB, dtype=torch.uint8, device="cuda"))
    assert hwsel.hwsel_fp8_matmul_workspace_bytes(d["a"], d["b"]) > 0
    assert hwsel.hwsel_sample_workspace_bytes(600_000, 3, 8) > 0
    return d


CALLS = {
    "quantise": lambda d, s: hwsel.hwsel_fp8_quantise(d["x"], stream=s),
    "dequantise": lambda d, s: hwsel.hwsel_fp8_dequantise(d["a"], stream=s),
    "transpose": lambda d, s: hwsel.hwsel_fp8_transpose(d["a"], stream=s),
    "matmul": lambda d, s: hwsel.hwsel_fp8_matmul(d["a"], d["b"], torch.float32, stream=s),
    "layer": lambda d, s: hwsel.hwsel_fp8_layer(d["a"], d["b"], stream=s),
    "draws": lambda d, s: hwsel.hwsel_sample_per_problem(d["scores"], d["seg"], d["u"], top_k=300, top_p=0.9, stream=s),
}


def tensors(result):
    if isinstance(result, dict):                            # (exponent bytes past the blocks may be anything)
        return [result["q"], result["scale"][:, :-(-result["cols"] // 128)]]
    return list(result) if isinstance(result, tuple) else [result]


def sizes(result):
    return [t.untyped_storage().nbytes() for t in tensors(result)]


def busy(d, stream):
    with torch.cuda.stream(stream):
        for _ in range(100):
            d["big"].fill_(1)


def overwrite(nbytes):
    """What the current stream would get of each size, and the sizes of a workspace, overwritten."""
    held = [torch.full((n,), 0xff, dtype=torch.uint8, device="cuda") for n in nbytes for _ in range(3)]
    return held


@pytest.fixture(params=["object", "number"])
def side(request):
    s = torch.cuda.Stream()
    return s, (s if request.param == "object" else s.cuda_stream)


@pytest.mark.parametrize("name", CALLS)
def test_workspace_is_not_handed_on(name, side, data):
    """The current stream allocates and writes while the given one has not begun."""
    call, (s, given) = CALLS[name], side
    want = [t.clone() for t in tensors(call(data, None))]
    work = [hwsel.hwsel_fp8_matmul_workspace_bytes(data["a"], data["b"]), hwsel.hwsel_sample_workspace_bytes(600_000, 3, 8)]
    torch.cuda.synchronize()
    busy(data, s)
    got = call(data, given)
    held = overwrite(work + [n // 2 for n in work] + sizes(got))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(tensors(got), want))
    assert all(bool((h == 0xff).all()) for h in held)       # and the call wrote to none of it


@pytest.mark.parametrize("name", CALLS)
def test_memory_that_the_current_stream_still_writes(name, side, data):
    """Freed on the current stream before the work that writes it has begun there."""
    call, (s, given) = CALLS[name], side
    result = call(data, None)
    want, bytes_each = [t.clone() for t in tensors(result)], sizes(result)
    work = [hwsel.hwsel_fp8_matmul_workspace_bytes(data["a"], data["b"]), hwsel.hwsel_sample_workspace_bytes(600_000, 3, 8)]
    del result
    torch.cuda.synchronize()
    busy(data, torch.cuda.current_stream())
    held = overwrite(work + bytes_each)
    del held
    got = call(data, given)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(tensors(got), want))


@pytest.mark.parametrize("name", CALLS)
def test_a_result_dropped_early(name, side, data):
    """Its memory is not the current stream's to reuse while the given one has yet to write it."""
    call, (s, given) = CALLS[name], side
    torch.cuda.synchronize()
    busy(data, s)
    got = call(data, given)
    nbytes, was = sizes(got), [t.data_ptr() for t in tensors(got)]
    del got
    now = [t.data_ptr() for t in overwrite(nbytes)]
    assert not set(was) & set(now)
    torch.cuda.synchronize()


@pytest.mark.parametrize("name", CALLS)
def test_a_result_that_the_current_stream_still_reads(name, side, data):
    """Dropped while a copy of it waits on the current stream: the next call on the given stream takes other memory."""
    call, (s, given) = CALLS[name], side
    want = [t.clone() for t in tensors(call(data, None))]
    torch.cuda.synchronize()
    got = call(data, given)
    s.synchronize()
    busy(data, torch.cuda.current_stream())
    copies, was = [t.clone() for t in tensors(got)], [t.data_ptr() for t in tensors(got)]
    del got
    other = call(data, given)
    assert not set(was) & {t.data_ptr() for t in tensors(other)}
    torch.cuda.synchronize()
    for got in (copies, tensors(other)):
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_the_current_stream_stays_current(side, data):
    before = torch.cuda.current_stream()
    for call in CALLS.values():
        call(data, side[1])
        assert torch.cuda.current_stream() == before
    with pytest.raises(ValueError):
        hwsel.hwsel_fp8_quantise(data["x"], mean=data["u"], stream=side[1])
    assert torch.cuda.current_stream() == before
    torch.cuda.synchronize()
