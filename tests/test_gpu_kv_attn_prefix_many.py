"""Prompts, chunks and drafts of fp16 rows behind shared prefixes (isoq_kv_attn_prefix), 32
rows a key head and more, against the definition in 64 bits with the tolerances of
test_gpu_kv_attn_shared.py, whose prefix_case runs each both with the prefix read anew
and with launches of its own.  Needs an MI355X."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

import paper_2603_28430_amd as iq  # noqa: E402
from test_gpu_kv_attn_shared import CANARY, check, prefix_case, reference, widen  # noqa: E402
from test_kv_attn_shared_launches import MANY, WIDE  # noqa: E402


@pytest.mark.parametrize("k", range(len(MANY)))
def test_many_rows(k):
    variant, d, bits, q_lens, kv, group, own, max_len, prefixes, counts = MANY[k]
    prefix_case(variant, d, bits, "f16", q_lens, kv * group, kv, 16, own, prefixes, counts, max_len=max_len, seed=k)


@pytest.mark.parametrize("own", [0, 1, 64, 128])
@pytest.mark.parametrize("rows", [32, 100, 150, 600])
@pytest.mark.parametrize("d", [64, 80, 96, 128])
def test_rows_and_own_positions(d, rows, own):
    """One key head, its rows as 2 heads of each token; fewer own positions than tokens among them (rows without a key there)."""
    prefix_case(("full", "fast", "2d")[(d // 16 + rows) % 3], d, 2 + (own + rows) % 3, "f16", [rows // 2, 3], 2, 1, 16, [own, 3],
                [64 + own % 7], max_len=max(own, 3), seed=d + rows + own)


def test_a_captured_step():
    """A graph of a chunk behind a prefix, replayed with other lengths and eager work between."""
    w, args, out, lse = prefix_case("full", 128, 3, "f16", [40, 1, 33], 8, 2, 16, [128, 40, 33], [150], max_len=128, seed=3)
    args["prefix_table"] = widen(args["prefix_table"], 16, WIDE)
    o, l = torch.empty_like(out), torch.empty_like(lse)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        iq.isoq_kv_attn_prefix(**args, out=o, lse=l)
    for plen, own in ((150, [128, 40, 33]), (64, [40, 1, 33]), (0, [100, 0, 20]), (133, [77, 40, 33])):
        args["prefix_lens"].fill_(plen)
        args["seq_lens"].copy_(torch.tensor(own, dtype=torch.int32))
        a, b = torch.full_like(out, CANARY), torch.full_like(lse, CANARY)
        iq.isoq_kv_attn_prefix(**args, out=a, lse=b)
        o.fill_(CANARY)
        l.fill_(CANARY)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(a, o) and torch.equal(b, l) and not a[:74].isnan().any()
        assert torch.equal(a[74:], torch.full_like(a[74:], CANARY)) and (b[74:] == CANARY).all()
        torch.ones(1 << 20, device="cuda").sum().item()


def test_rows_of_a_prefix_that_are_left_alone():
    """max_prefix_tokens below a prefix's tokens: those rows keep what they held, the others are what they are without."""
    w, args, out, lse = prefix_case("fast", 64, 4, "f16", [40, 9, 33], 4, 2, 16, [64, 9, 33], [150, 33], [2, 1], max_len=64, seed=4)
    args["prefix_table"] = widen(args["prefix_table"], 16, WIDE)
    ref = reference(w, 1.3, [3, 3, 4], max_len=64)
    for most in (16, 40, 48):
        o, l = torch.full_like(out, CANARY), torch.full_like(lse, CANARY)
        iq.isoq_kv_attn_prefix(**dict(args, max_prefix_tokens=most), out=o, lse=l)
        row = torch.arange(len(out), device="cuda")
        left = (row >= most) & (row < 49) | (row >= 49 + most)
        left[82:] = True
        assert torch.equal(o[left], torch.full_like(o[left], CANARY)) and (l[left] == CANARY).all()
        check(o, l, {(t, h): x for (t, h), x in ref.items() if not left[t]})
