"""The first attention of a handle makes its tables: the same bits from several
host threads that come first together, inside a graph capture, and from a call
that asked for the workspace before.  Needs an MI355X."""
import threading

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

import paper_2603_28430_amd as iq  # noqa: E402
from test_gpu_kv_attn import device, setup  # noqa: E402

CASES = [(128, 3, "f16", [3, 2]), (128, 4, "f16", [40, 2]), (64, 2, "f32", [1, 1]), (70, 3, "f16", [2, 2])]


def fresh(d, bits, dtype, q_lens):
    return device(setup("full", d, bits, dtype, q_lens, 4, 2, 16, [900, 300], seed=7))


@pytest.mark.parametrize("d,bits,dtype,q_lens", CASES)
def test_host_threads_that_come_first_together(d, bits, dtype, q_lens):
    want = iq.isoq_kv_attn(**fresh(d, bits, dtype, q_lens))
    torch.cuda.synchronize()
    for _ in range(5):
        args = fresh(d, bits, dtype, q_lens)
        got, streams, gate = [None] * 4, [torch.cuda.Stream() for _ in range(4)], threading.Barrier(4)
        torch.cuda.synchronize()

        def work(i):
            gate.wait()
            got[i] = iq.isoq_kv_attn(**args, stream=streams[i])
            streams[i].synchronize()
        threads = [threading.Thread(target=work, args=(i,)) for i in range(4)]
        for t in threads:
            t.start()
        for t in threads:
            t.join()
        for o, l in got:
            assert torch.equal(o, want[0]) and torch.equal(l, want[1])


@pytest.mark.parametrize("d,bits,dtype,q_lens", CASES)
def test_first_in_a_capture(d, bits, dtype, q_lens):
    want = iq.isoq_kv_attn(**fresh(d, bits, dtype, q_lens))
    args = fresh(d, bits, dtype, q_lens)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, lse = iq.isoq_kv_attn(**args)
    for _ in range(3):
        out.fill_(0)
        lse.fill_(0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1])


def test_handles_destroyed_with_and_without_tables():
    for attends in (False, True):
        args = fresh(128, 3, "f16", [3, 2])
        if attends:
            iq.isoq_kv_attn(**args)
            torch.cuda.synchronize()
        for p in (args["pk"], args["pv"]):
            iq.isoq_params_destroy(p)
