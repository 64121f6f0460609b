"""Attention of 32 rows and more per key head where one split has all of a
sequence's positions and the kernel finishes its rows itself (8-D handles: joins
one part): every variant, width and number of bits, short prompts and calls of so
many workgroups that longer ones are not split, with and without lse.  That the
call is planned so is read from its workspace: none, or one part a row.  Reference
and tolerances of test_gpu_kv_attn.py and test_gpu_kv_attn_many.py.  Needs an
MI355X."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

import paper_2603_28430_amd as iq  # noqa: E402
from paper_2603_28430_amd import isoquant as binding  # noqa: E402
from test_gpu_kv_attn import CANARY, check, device, reference, setup  # noqa: E402


def workspace(w, args):
    """Bytes of the call's workspace, and of one part a row."""
    n, heads, d = w["q"].shape
    cap = args["block_table"].shape[1] * w["bs"]
    need = iq.isoq_kv_attn_workspace(args["pk"], args["pv"], torch.float16, n, args["max_q_len"], len(w["seq_lens"]), heads,
                                     w["n_kv"], w["bs"], args["block_table"].shape[1], cap)
    return need, n * heads * (d + 2) * 4


def run(w, scale=1.3):
    args = device(w)
    need, part = workspace(w, args)
    assert need == (part if w["variant"] == "8d" else 0), "not the path that this test is about"
    out = torch.full_like(args["q"], CANARY)
    lse = torch.full(args["q"].shape[:2], CANARY, device="cuda")
    iq.isoq_kv_attn(**args, scale=scale, out=out, lse=lse)
    n = sum(w["q_lens"])
    check(out, lse, reference(w, scale))
    assert torch.all(out[n:] == torch.full_like(out[n:], CANARY)) and torch.all(lse[n:] == CANARY)
    # without lse the same bits
    other, ws = torch.full_like(out, CANARY), torch.zeros(max(need, 1), dtype=torch.uint8, device="cuda")
    n_seqs, blocks = args["block_table"].shape
    st = binding.lib.isoq_kv_attn(
        args["pk"].handle, args["pv"].handle, binding._dtype_code(torch.float16), args["q"].data_ptr(),
        args["q_start"].data_ptr(), out.shape[0], args["max_q_len"], n_seqs, out.shape[1], w["n_kv"], args["k_idx"].data_ptr(),
        args["k_rho"].data_ptr(), args["v_idx"].data_ptr(), args["v_rho"].data_ptr(), args["k_idx"].shape[0], w["bs"],
        args["block_table"].data_ptr(), blocks, args["seq_lens"].data_ptr(), blocks * w["bs"], scale, other.data_ptr(), None,
        ws.data_ptr(), need, binding._stream_ptr(None))
    assert st == 0
    torch.cuda.synchronize()
    assert torch.equal(out, other)


@pytest.mark.parametrize("bits", [2, 3, 4])
@pytest.mark.parametrize("d", [64, 80, 96, 128])
@pytest.mark.parametrize("variant", ["full", "fast", "2d", "8d"])
def test_short_prompts(variant, d, bits):
    """Whole prompts of up to 112 positions, a row tile and more of them, one that is
    shorter than its tokens, and rows behind the last sequence."""
    run(setup(variant, d, bits, "f16", [100, 33, 20], 4, 2, 16, [112, 33, 7], seed=d + bits, pad_rows=3))


@pytest.mark.parametrize("variant,d,bits", [("full", 128, 3), ("fast", 96, 4), ("2d", 80, 2), ("8d", 64, 3), ("fast", 64, 4)])
def test_many_workgroups(variant, d, bits):
    """Several hundred positions in one split, ragged, an empty sequence and one without tokens."""
    rng = np.random.default_rng(d)
    # (more workgroups than half of what the plan wants: 512, or 768 at d = 64)
    seqs = 50 if d == 64 else 34
    lens = rng.integers(300, 700, seqs)
    lens[3] = 0
    new = rng.integers(5, 9, seqs)
    new[5], new[-1] = 0, 8
    run(setup(variant, d, bits, "f16", list(new), 32, 8, 16, [int(x) for x in lens], seed=d, pad_rows=1))
