"""What cb_append_kv_device reports when it runs beside other work: a slot that is left out is always heard of."""
import pytest

from paper_2511_21699_amd import binding as B
from .serving_gpu import Batch

pytestmark = pytest.mark.gpu


def _batch():
    b = Batch("bf16", 8, 2, 64, [14], [4], block=16, max_nodes=8)
    b.table[0, 1] = b.k.shape[0] + 3  # slots 16 and 17 are outside the pool
    return b


def _busy():
    """Some tens of milliseconds of work for the current stream."""
    import torch
    a = torch.zeros(8192, 8192, device="cuda")
    torch.cuda.synchronize()
    return lambda: [torch.mm(a, a) for _ in range(6)]


def test_the_status_waits_for_an_append_on_another_stream():
    import torch
    b, busy, side = _batch(), _busy(), torch.cuda.Stream()
    out = torch.empty_like(b.q)
    with torch.cuda.stream(side):
        busy()
        b.ver.append_kv(b.q, b.q[:, :2].contiguous(), b.q[:, 2:4].contiguous(), B.head_prep(), b.kv, b.kv_len, b.off, out)
    assert b.ver.device_status() == 64
    assert b.ver.device_status() == 0
    side.synchronize()
    assert b.ver.device_status() == 0


def test_the_status_of_a_replayed_append_is_kept_until_it_is_read():
    import torch
    b, busy, side = _batch(), _busy(), torch.cuda.Stream()
    k, v, out = b.q[:, :2].contiguous(), b.q[:, 2:4].contiguous(), torch.empty_like(b.q)
    call = b.ver.bind_append_kv(b.q, k, v, B.head_prep(), b.kv, b.kv_len, b.off, out, stream=side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        call()
    assert b.ver.device_status() == 0
    other = torch.cuda.Stream()
    for _ in range(3):
        with torch.cuda.stream(other):
            busy()
            graph.replay()
        early = b.ver.device_status()  # (the context does not know the replay's stream)
        other.synchronize()
        assert early | b.ver.device_status() == 64
        assert b.ver.device_status() == 0
