"""The decoder's steps of test_gpu_step_run.py with prompts behind prefixes that are attended to in
launches of their own (a prefix table as for 100,000 positions) and own positions of 128 at
most: what a batch of requests behind one instruction takes, eagerly and as one replayed
graph.  References and tolerance as there.  Needs an MI355X."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

import test_gpu_step_run as steps  # noqa: E402
from test_gpu_kv_attn_shared import widen  # noqa: E402
from test_kv_attn_shared_launches import WIDE  # noqa: E402

STEPS = [
    [40, 1, 0, 17, 33, 0, 33],
    [41, 2, 60, 18, 34, 0, 34],
    [42, 3, 61, 9, 35, 18, 35],
    [43, 0, 62, 10, 36, 19, 0],
    [44, 64, 63, 11, 0, 20, 128],     # (the last sequence's blocks are not there)
    [0, 65, 64, 12, 40, 21, 90],
]
CASES = [(128, 3, torch.float16, 16, 2, 4, "full"), (64, 4, torch.float16, 8, 1, 2, "fast"), (80, 2, torch.float16, 16, 2, 1, "2d"),
         (96, 3, torch.float16, 16, 1, 3, "8d")]


def world(monkeypatch, *case):
    monkeypatch.setattr(steps, "STEPS", STEPS)
    monkeypatch.setattr(steps, "MAX_LEN", 128)
    w = steps.World(*case)
    w.prefix_table = widen(w.prefix_table, w.bs, WIDE)
    return w


@pytest.mark.parametrize("case", CASES)
def test_steps(monkeypatch, case):
    w = world(monkeypatch, *case)
    for new in STEPS:
        w.step(new, w.call)


@pytest.mark.parametrize("case", CASES[:2])
def test_steps_of_a_captured_graph(monkeypatch, case):
    w = world(monkeypatch, *case)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        w.call()                    # (no sequence has tokens: nothing changes)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = w.call()

    def replay():
        graph.replay()
        return got

    for new in STEPS:
        w.step(new, replay)
        torch.ones(1 << 20, device="cuda").sum().item()
