"""A call that is cut off between its two launches (the second one refused by the runtime, say) leaves nothing behind that the next call on the
table would count on: its results have the same bits."""
import numpy as np
import pytest

from gpu_util import to_dev
from test_gpu_rows_grad import Case

pytestmark = pytest.mark.gpu


def _first_launch_alone(c, form):
    """The call, captured, with everything behind its first kernel taken out of the graph."""
    import torch
    from cuda.bindings import runtime as rt
    dA, dB = c.buffers()[2:]
    x, dy = c.rows(form), to_dev(c.dy)
    graph = torch.cuda.CUDAGraph(keep_graph=True)
    with torch.cuda.graph(graph):
        c.t.backward_adapters_rows(c.tT, x, dy, c.so, c.ids, c.ids_T, dA, dB, accumulate=False)
    raw = rt.cudaGraph_t(graph.raw_cuda_graph())
    err, nodes, n = rt.cudaGraphGetNodes(raw, 16)
    err2, roots, n_roots = rt.cudaGraphGetRootNodes(raw, 16)
    assert int(err) == int(err2) == 0 and n == 2 and n_roots == 1
    for node in nodes[:n]:
        if int(node) != int(roots[0]):
            assert int(rt.cudaGraphDestroyNode(node)[0]) == 0
    graph.instantiate()
    return graph, (x, dy, dA, dB)


@pytest.mark.parametrize("form", ("int8", "bf16"))
def test_the_second_launch_never_happens(form):
    import torch
    c = Case(700, 1032, 520, [32, 16], [400, 300], [0, 1])
    want = c.run(form, fill=0.5)
    c.check(want[0].copy(), want[1].copy(), form, base=0.5)
    cut, kept = _first_launch_alone(c, form)
    for _ in range(3):
        cut.replay()
    torch.cuda.synchronize()
    for _ in range(2):
        got = c.run(form, fill=0.5)
        assert np.array_equal(got[0], want[0]) and np.array_equal(got[1], want[1])
    del cut, kept
    c.close()
