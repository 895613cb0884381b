"""The scoring, ranking and evaluation calls given another stream than torch's
current one: their workspaces and results are that stream's memory, as for the
8-bit calls.  Streams are kept busy by fills so that what is unordered overlaps."""
import pytest
import torch

import synth
from _gpu_util import Dev
from paper_2609_35587_amd import hwsel

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def data():
    w = synth.workload("tiny")
    d = Dev(w)
    X = d.features(64)
    packed = hwsel.hwsel_forest_pack(d.forest)
    scores = hwsel.hwsel_forest_score(d.forest, X, packed=packed)
    idx, _ = hwsel.hwsel_topk_per_problem(scores, d.seg, w.cfg.k)
    big = torch.empty(1 << 30, dtype=torch.uint8, device="cuda")
    ids = torch.arange(X.shape[0], device="cuda", dtype=torch.int32) % 64
    return dict(w=w, d=d, X=X, packed=packed, scores=scores, idx=idx, big=big, ids=ids)


CALLS = {
    "features": lambda m, s: (hwsel.hwsel_features(m["w"].hw, m["d"].problems, m["d"].seg, m["d"].cands, 64, stream=s),),
    "forest": lambda m, s: (hwsel.hwsel_forest_score(m["d"].forest, m["X"], packed=m["packed"], stream=s),),
    "topk": lambda m, s: hwsel.hwsel_topk_per_problem(m["scores"], m["d"].seg, m["w"].cfg.k, stream=s),
    "regret": lambda m, s: hwsel.hwsel_regret(m["d"].runtimes, m["d"].seg, m["idx"], stream=s),
    "select": lambda m, s: hwsel.hwsel_select_forest(m["w"].hw, m["d"].problems, m["d"].seg, m["d"].cands, 64, m["d"].forest,
                                                     m["packed"], m["w"].cfg.k, stream=s)[:2],
    "evaluate": lambda m, s: hwsel.hwsel_evaluate(m["d"].runtimes, m["d"].seg, m["idx"], stream=s),
    "static": lambda m, s: hwsel.hwsel_static_config(m["d"].runtimes, m["d"].seg, m["ids"], 64, stream=s),
}


def busy(m, stream):
    with torch.cuda.stream(stream):
        for _ in range(100):
            m["big"].fill_(1)


def workspaces(m):
    return [hwsel.hwsel_forest_workspace_bytes(m["d"].forest, m["X"].shape[0]),
            hwsel.hwsel_select_forest_workspace_bytes(m["d"].forest, m["X"].shape[0])]


def same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("number", [False, True])
@pytest.mark.parametrize("name", CALLS)
def test_memory_is_the_given_streams(name, number, data):
    call, s = CALLS[name], torch.cuda.Stream()
    given = s.cuda_stream if number else s
    want = [t.clone() for t in call(data, None)]
    sizes = workspaces(data) + [t.untyped_storage().nbytes() for t in want]
    torch.cuda.synchronize()
    # the current stream allocates and writes before the given one has begun
    busy(data, s)
    got = call(data, given)
    held = [torch.full((n,), 0xff, dtype=torch.uint8, device="cuda") for n in sizes for _ in range(3)]
    torch.cuda.synchronize()
    assert same(got, want) and all(bool((h == 0xff).all()) for h in held)
    # what it freed is still to be written there when the call comes
    busy(data, torch.cuda.current_stream())
    held = [torch.full((n,), 0xff, dtype=torch.uint8, device="cuda") for n in sizes for _ in range(3)]
    del held
    got = call(data, given)
    torch.cuda.synchronize()
    assert same(got, want)
    # results dropped early, and results that the current stream still reads
    busy(data, torch.cuda.current_stream())
    copies, was = [t.clone() for t in got], {t.data_ptr() for t in got}
    del got
    other = call(data, given)
    assert not was & {t.data_ptr() for t in other}
    torch.cuda.synchronize()
    assert same(copies, want) and same(other, want)
    assert torch.cuda.current_stream() == torch.cuda.default_stream()
