"""Calls of isoq_kv_attn that its documentation allows and that are easy to get
wrong: token ranges that leave rows before, between and behind them, lengths
past the table and below zero, many sequences, blocks of one position, no lse,
queries overwritten behind the call, host threads.  Reference and tolerances of
test_gpu_kv_attn.py.  Needs an MI355X."""
import threading

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

import paper_2603_28430_amd as iq  # noqa: E402
from paper_2603_28430_amd import isoquant as binding  # noqa: E402
from test_gpu_kv_attn import CANARY, check, device, reference, run_case, setup  # noqa: E402

KERNELS = [(128, 3, "f16", 2), (128, 3, "f16", 40), (96, 2, "f32", 10), (70, 3, "f16", 2)]   # digits, fp16, 12 rows, generic


def empty(args):
    return torch.full_like(args["q"], CANARY), torch.full(args["q"].shape[:2], CANARY, device="cuda")


@pytest.mark.parametrize("d,bits,dtype,n", KERNELS)
def test_rows_outside_the_sequences(d, bits, dtype, n):
    """Rows before the first sequence and behind the last one stay; a range that runs past the rows is cut."""
    w = setup("full", d, bits, dtype, [n, 3], 2, 2, 16, [300, 20], seed=3, pad_rows=5)
    args = device(w)
    q = args["q"].clone()
    args["q"] = torch.cat([q[n + 3:n + 5], q[:n + 3], q[n + 5:]])
    args["q_start"] = args["q_start"] + 2
    out, lse = empty(args)
    iq.isoq_kv_attn(**args, scale=1.3, out=out, lse=lse)
    torch.cuda.synchronize()
    check(out[2:], lse[2:], reference(w, 1.3))
    for rows in (slice(0, 2), slice(n + 5, None)):
        assert torch.all(out[rows] == torch.full_like(out[rows], CANARY)) and torch.all(lse[rows] == CANARY)
    # ranges past the rows, descending ones, negative ones: nothing outside q is touched
    for bad in ([0, n, 10 ** 9], [n, 0, 2], [-7, -3, 1], [2 ** 31 - 1, -2 ** 31, 4]):
        args["q_start"].copy_(torch.tensor(bad, dtype=torch.int64).to(torch.int32))
        iq.isoq_kv_attn(**args, scale=1.3)
    torch.cuda.synchronize()


@pytest.mark.parametrize("d,bits,dtype,n", KERNELS)
def test_lengths_past_the_table_and_below_zero(d, bits, dtype, n):
    """A length past what the table holds: the causal border counts from the length, the positions end with the table."""
    w = setup("full", d, bits, dtype, [n, 2], 2, 2, 16, [300, 48], seed=4)
    args = device(w)
    cap = args["block_table"].shape[1] * 16
    args["seq_lens"].copy_(torch.tensor([2 ** 31 - 1, -5], dtype=torch.int32))
    table = w["sides"][0][2].table
    assert cap == 304 and (table[0] >= 0).all()
    for side, name in enumerate(("k", "v")):   # (the positions 300 .. 303 are the last page's)
        args[name + "_rho"][int(table[0, 18]), :, 12:] = 0.0
        c = w["sides"][side][2]
        for h in (0, 1):
            c.idx[0, h] = np.concatenate([c.idx[0, h], np.zeros((4, c.idx[0, h].shape[1]), np.uint8)])
            c.norms[0, h] = np.concatenate([c.norms[0, h], np.zeros(4, np.float32)])
    out, lse = iq.isoq_kv_attn(**args, scale=1.3)
    w["seq_lens"] = [2 ** 31 - 1, 0]
    check(out, lse, {k: v for k, v in reference(w, 1.3).items() if k[0] < n})
    assert torch.all(out[n:n + 2] == 0) and torch.all(lse[n:n + 2] == -np.inf)


def test_many_sequences():
    """As many sequences as the grid takes, of one position each."""
    n = 65535
    rng = np.random.default_rng(0)
    pk, pv = (iq.isoq_params_init("fast", 64, 3, 1, seed=s) for s in (1, 2))
    idx = [torch.from_numpy(rng.integers(0, 256, (64, 1, 16, pk.record_bytes), dtype=np.uint8)).cuda() for _ in (0, 1)]
    rho = [torch.from_numpy(rng.uniform(0.5, 2.0, (64, 1, 16)).astype(np.float32)).cuda() for _ in (0, 1)]
    q = torch.randn((n, 1, 64), device="cuda").half()
    table = torch.randint(0, 64, (n, 1), device="cuda", dtype=torch.int32)
    lens = torch.ones(n, device="cuda", dtype=torch.int32)
    out, lse = iq.isoq_kv_attn(pk, q, idx[0], rho[0], pv, idx[1], rho[1], table, lens)
    # one position: out is its value, whatever the query (records of position 0 of the 64 blocks)
    first = [x[:, 0].reshape(64, -1) for x in idx]
    rec = first[1].reshape(64, pk.record_bytes // 8, 16, 8)[:, :, 0].reshape(64, -1).contiguous()   # pieces of 8 bytes
    v = iq.isoq_dequantize(pv, rec, rho[1][:, 0, 0].contiguous(), dtype=torch.float32)
    want = v[table[:, 0].long()]
    # a level off by 1 / 32639 of the largest and half a step of fp16, of the value's norm (at most sqrt(64) times its largest coordinate)
    err = (out[:, 0].float() - want).norm(dim=1)
    assert torch.all(err <= (2.0 ** -11 + 3.0 / 32639) * want.norm(dim=1)), float((err / want.norm(dim=1)).max())
    assert torch.isfinite(lse).all()


@pytest.mark.parametrize("d,bits,dtype,n", KERNELS)
def test_blocks_of_one_position(d, bits, dtype, n):
    run_case("fast", d, bits, dtype, [n, 3], n_q=2, n_kv=2, bs=1, seq_lens=[200, 70], seed=5)


@pytest.mark.parametrize("length", [300, 3000])
@pytest.mark.parametrize("d,bits,dtype,n", KERNELS)
def test_without_lse(d, bits, dtype, n, length):
    w = setup("full", d, bits, dtype, [n, 3], 2, 2, 16, [length, 20], seed=6)
    a = device(w)
    out, lse = iq.isoq_kv_attn(**a)
    other = torch.full_like(out, CANARY)
    pk, pv, q = a["pk"], a["pv"], a["q"]
    cap = a["block_table"].shape[1] * 16
    code, most = binding._dtype_code(q.dtype), a["max_q_len"]
    sizes = (pk.handle, pv.handle, code, n + 3, most, 2, 2, 2, 16, cap // 16, cap)
    need = binding.lib.isoq_kv_attn_workspace(*sizes)
    ws = torch.zeros(max(need, 1), dtype=torch.uint8, device="cuda")
    st = binding.lib.isoq_kv_attn(pk.handle, pv.handle, code, q.data_ptr(), a["q_start"].data_ptr(), n + 3, most, 2, 2, 2,
                                  a["k_idx"].data_ptr(), a["k_rho"].data_ptr(), a["v_idx"].data_ptr(), a["v_rho"].data_ptr(),
                                  a["k_idx"].shape[0], 16, a["block_table"].data_ptr(), cap // 16, a["seq_lens"].data_ptr(),
                                  cap, 1.0, other.data_ptr(), None, ws.data_ptr(), need, binding._stream_ptr(None))
    assert st == 0
    torch.cuda.synchronize()
    assert torch.equal(out, other)


def test_buffers_reused_behind_the_call():
    """What the binding allocated on another stream is not handed out while the call still runs there."""
    w = setup("fast", 128, 3, "f16", [1, 1], 8, 2, 16, [20000, 9000], seed=13)
    args = device(w)
    want = iq.isoq_kv_attn(**args)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = []
    for _ in range(20):
        got.append(iq.isoq_kv_attn(**args, stream=side))
        for _ in range(4):   # the current stream takes and fills memory of the workspace's size
            torch.full((1 << 20,), 7, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    for o, l in got:
        assert torch.equal(o, want[0]) and torch.equal(l, want[1])


def test_host_threads():
    """Calls from several host threads at once, each with a stream of its own, sharing the handles."""
    ws = [setup("full", 128, 3, "f16", [40 * (i % 2) + 1, 2], 4, 2, 16, [900, 300], seed=20) for i in range(4)]
    args = [device(w) for w in ws]
    for a in args[1:]:
        a["pk"], a["pv"] = args[0]["pk"], args[0]["pv"]   # (of the same draws)
    want = [iq.isoq_kv_attn(**a) for a in args]
    torch.cuda.synchronize()
    got, streams = [[] for _ in args], [torch.cuda.Stream() for _ in args]

    def work(i):
        for _ in range(10):
            got[i].append(iq.isoq_kv_attn(**args[i], stream=streams[i]))
        streams[i].synchronize()
    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(args))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    for i, (o, l) in enumerate(want):
        assert len(got[i]) == 10
        for x, y in got[i]:
            assert torch.equal(x, o) and torch.equal(y, l)
