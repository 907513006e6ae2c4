"""The library's passes of perf/operators.py run on the stream that is current when they are called."""

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from perf import operators  # noqa: E402

CASES = [
    {"op": "norm", "tokens": 65, "n": 1000, "x": "bf16", "format": "mxfp8", "residual": True, "gain": True},
    {"op": "quantize", "tokens": 65, "n": 1000, "x": "f32", "format": "mxfp4"},
    {"op": "objective", "b": 3, "tokens": 65, "n": 200, "grad": "bf16", "format": "mxfp4", "reduce": "sum"},
    {"op": "product", "m": 65, "n": 200, "k": 1000, "a": "mxfp8", "b": "mxfp4", "out": "bf16"},
]


def same(a, b):
    return a.keys() == b.keys() and all(torch.equal(a[k], b[k]) for k in a)


@pytest.mark.parametrize("case", CASES, ids=[c["op"] for c in CASES])
def test_a_pass_runs_on_the_current_stream(case):
    """Eagerly on the default stream, then on another, then captured there: replays of the graph follow new inputs."""
    state, other = operators.prepare(case, 1), operators.prepare(case, 2)
    want = [{k: v.clone() for k, v in operators._calls(s).items()} for s in (state, other)]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        assert operators._library()["ctx"].stream.cuda_stream == side.cuda_stream
        got = operators._calls(state)
    side.synchronize()
    assert same(got, want[0])
    inputs = {"norm": ("X", "R", "g"), "quantize": ("X",), "objective": ("Y",), "product": ("A", "As", "B", "Bs")}[case["op"]]
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        out = operators._calls(state)
    saved = [state[k].clone() for k in inputs]
    for turn in range(4):
        for k, first in zip(inputs, saved):
            state[k].copy_(other[k] if turn % 2 else first)
        for v in out.values():
            v.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert same(out, want[turn % 2])
    assert operators._library()["ctx"].stream.cuda_stream == torch.cuda.current_stream().cuda_stream
