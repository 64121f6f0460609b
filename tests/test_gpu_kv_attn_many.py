"""Attention of 32 rows and more per key head (the fp16 matrix cores; widths up
to 128, fp16 queries) where it can go wrong, against the definition in 64 bits;
reference and tolerance of test_gpu_kv_attn.py.  In its terms: a query's two fp16
parts are off by 2^-22 of its largest coordinate, inside (pw + 8) 2^-23.  A key's
level is fp16 plus what that leaves (at most 1e-4 of the levels' root mean square
at 4 bits) in e4m3, times the query in e4m3: both off by 2^-4 / sqrt(3) = 3.6% of
that at most in the root mean square, so a coordinate's product by 5e-6, and the
sum of d of them with independent signs by 5e-6 / sqrt(d) of ||q|| ||c[idx]||: 6.4e-7
at d = 64, of which (64 + 8) 2^-23 is 13 times, and more above.  A value's level is
off by at most 7e-5 of the levels' root mean square at 4 bits and 8e-6 at 3, inside
1 / 32639 of the largest level (2.7 and 2.2 times that) times sqrt(pw); a weight by
2^-4 of the 2^-11 that fp16 leaves of it, times a level off by 2^-4: 2^-14 of an
independent sum, inside what is allowed for the output's own rounding.  For other
codebooks the level's error is worked out from the levels (test_many_codebooks).
Needs an MI355X."""
import numpy as np
import pytest

import oracle

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

import paper_2603_28430_amd as iq  # noqa: E402
from test_gpu_kv_attn import CANARY, check, device, reference, run_case, setup  # noqa: E402


@pytest.mark.parametrize("bits", [2, 3, 4])
@pytest.mark.parametrize("variant", ["full", "fast", "2d", "8d"])
def test_many_d128(variant, bits):
    run_case(variant, 128, bits, "f16", [9, 40, 1], n_q=8, n_kv=2, bs=16, seq_lens=[1300, 50, 300], seed=bits)


@pytest.mark.parametrize("bits", [2, 3, 4])
@pytest.mark.parametrize("d", [64, 80, 96])
def test_many_widths(d, bits):
    """Blocks that end inside a tile, records stored whole among them (d = 80, 3 bits)."""
    run = d // 16 + bits
    run_case(("full", "fast", "2d", "8d")[run % 4], d, bits, "f16", [33, 70], n_q=6, n_kv=2, bs=(16, 7)[run % 2],
             seq_lens=[530, 80], seed=run)


@pytest.mark.parametrize("group", [32, 33, 64, 129])
def test_many_groups(group):
    """Rows of one token: every query head of a key head (one key head; an odd number)."""
    run_case("fast", 128, 3, "f16", [1, 1], n_q=group, n_kv=1, bs=16, seq_lens=[1000, 77], seed=group)
    run_case("full", 64, 4, "f16", [2, 3], n_q=3 * group, n_kv=3, bs=16, seq_lens=[90, 3], seed=group)


@pytest.mark.parametrize("d,bs", [(128, 16), (96, 5)])
def test_many_lengths(d, bs):
    """Around tiles of 64 positions and chunks of 256, with rows that end on both
    sides of a border, sequences shorter than their tokens (rows without a key),
    without tokens, empty; a max_len that cuts."""
    lens = [0, 1, 2, 31, 63, 64, 65, 66, 127, 128, 130, 255, 256, 257, 513, 1030]
    q_lens = [3, 1, 4, 33, 0, 5, 34, 2, 7, 40, 33, 1, 3, 60, 35, 36]
    run_case("full", d, 3, "f16", q_lens, n_q=2, n_kv=1, bs=bs, seq_lens=lens, seed=d)
    run_case("fast", d, 4, "f16", q_lens, n_q=2, n_kv=1, bs=bs, seq_lens=lens, max_len=200, seed=d + 1)


def test_many_splits():
    """A long cache and few rows: splits, joined; rows whose limits end in different ones."""
    run_case("fast", 64, 3, "f16", [40], n_q=1, n_kv=1, bs=16, seq_lens=[9000], scale=2.0, seed=3)
    run_case("full", 128, 4, "f16", [300], n_q=1, n_kv=1, bs=16, seq_lens=[1030], seed=4)


def test_many_heads_in_xcd_order():
    run_case("full", 128, 3, "f16", [16, 9], n_q=48, n_kv=16, bs=7, seq_lens=[300, 70], seed=4)
    run_case("fast", 96, 3, "f16", [16, 9], n_q=16, n_kv=8, bs=7, seq_lens=[300, 70], n_sets=1, seed=3)


def test_many_max_q_len_cuts():
    w = setup("full", 128, 3, "f16", [50, 2], 2, 2, 16, [60, 30], seed=2)
    args = device(w)
    args["max_q_len"] = 40
    out, lse = torch.full_like(args["q"], CANARY), torch.full(args["q"].shape[:2], CANARY, device="cuda")
    iq.isoq_kv_attn(**args, out=out, lse=lse)
    check(out, lse, {k: v for k, v in reference(w, 1.0).items() if not 40 <= k[0] < 50})
    assert torch.all(lse[40:50] == CANARY) and torch.all(out[40:50] == torch.full_like(out[40:50], CANARY))


@pytest.mark.parametrize("bits", [2, 4])
def test_many_invalid_pages(bits):
    """Pages outside the cache: single ones, a whole tile, the first and the last, all of a sequence."""
    w = setup("full", 128, bits, "f16", [9, 12, 40], 4, 1, 16, [400, 33, 48], seed=9)
    args = device(w)
    c = w["sides"][0][2]
    table = c.table.copy()
    table[0, [0, 3, 4, 5, 6, 7, 8, 24]] = [-1, c.n_blocks, -7, 2 ** 31 - 1, -2 ** 31, -1, -1, -1]
    table[1, :] = -1
    valid = np.repeat((table >= 0) & (table < c.n_blocks), 16, axis=1)
    args["block_table"] = torch.from_numpy(table).cuda()
    out, lse = iq.isoq_kv_attn(**args, scale=1.3)
    check(out, lse, reference(w, 1.3, valid=valid))


@pytest.mark.parametrize("bad", [np.inf, -np.inf, np.nan])
def test_many_nonfinite_queries(bad):
    w = setup("full", 128, 3, "f16", [20, 3], 6, 2, 16, [300, 40], seed=4)
    ref = reference(w, 1.0)
    rows = [(0, 1), (7, 5), (22, 3)]
    for t, hq in rows:
        w["q"][t, hq, 5 * t] = bad
    out, lse = iq.isoq_kv_attn(**device(w), scale=1.0)
    for t, hq in rows:
        assert torch.isnan(out[t, hq]).all() and torch.isnan(lse[t, hq])
        del ref[t, hq]
    check(out, lse, ref)


@pytest.mark.parametrize("bad", [np.inf, -np.inf, np.nan])
@pytest.mark.parametrize("side", ["k", "v"])
@pytest.mark.parametrize("d,bits,dtype,q_lens", [(128, 3, "f16", [40, 33]), (64, 4, "f16", [40, 33]), (128, 2, "f16", [3, 2]),
                                                 (96, 4, "f32", [7, 1]), (70, 3, "f16", [3, 9])])
def test_norms_that_are_no_numbers(d, bits, dtype, q_lens, side, bad):
    """NaN in the rows that attend to such a position, and others as if it were not there."""
    w = setup("full", d, bits, dtype, q_lens, 2, 2, 16, [300, 90], seed=4)
    ref = reference(w, 1.0)
    args = device(w)
    hit = set()
    at = 0
    for s, (n, pos) in enumerate(zip(q_lens, (298, 89))):   # inside a tile, and the last position
        c = w["sides"][0 if side == "k" else 1][2]
        args[side + "_rho"][int(c.table[s, pos // 16]), 1, pos % 16] = bad
        hit |= {(at + i, 1) for i in range(n) if w["seq_lens"][s] - (n - 1 - i) > pos}
        at += n
    out, lse = iq.isoq_kv_attn(**args, scale=1.0)
    assert 2 <= len(hit) < len(ref)
    for key in hit:
        assert torch.isnan(out[key]).all() and torch.isnan(lse[key]), key
        del ref[key]
    check(out, lse, ref)


@pytest.mark.parametrize("scale", [0.0, 300.0, -2.0])
def test_many_scales(scale):
    run_case("fast", 128, 3, "f16", [17, 20], n_q=4, n_kv=1, bs=16, seq_lens=[700, 40], scale=scale, seed=8)


def test_many_query_sizes():
    """Queries from fp16's smallest numbers to its largest in one call, zeros among them."""
    w = setup("full", 128, 3, "f16", [33, 40], 2, 2, 16, [300, 64], seed=5)
    size = np.array([2.0 ** -24, 1e-6, 1e-4, 1e-2, 1.0, 50.0, 3e4, 0.0])
    for t in range(73):
        q = w["q"][t].astype(np.float64)
        w["q"][t] = (q / np.abs(q).max() * size[t % 8]).astype(np.float16)
    out, lse = iq.isoq_kv_attn(**device(w), scale=0.7)
    check(out, lse, reference(w, 0.7))


@pytest.mark.parametrize("which", ["keys", "values", "both"])
@pytest.mark.parametrize("bits", [2, 3, 4])
def test_many_norms(which, bits):
    """Norms over eight orders of magnitude from tile to tile and inside tiles,
    zeros (whole tiles of them) among them: the units that sums are held in follow."""
    def keys(s, h, length):
        rng = np.random.default_rng(10 * s + h)
        rho = 10.0 ** rng.uniform(-2, 0, length) * np.repeat(10.0 ** rng.uniform(-5, 3, length // 64 + 1), 64)[:length]
        rho[64:192] = 0.0
        rho[rng.integers(0, length, length // 9)] = 0.0
        return rng.integers(0, 1 << bits, (length, 128)).astype(np.uint8), np.float32(rho)
    w = setup("full", 128, bits, "f16", [33, 20], 4, 2, 16, [1500, 700], keys=keys, seed=6)
    for i, side in enumerate(w["sides"]):
        c = side[2]
        c.rho = np.where(np.isnan(c.rho), np.float32(0), c.rho)
        if which != "both" and i == (which == "keys"):   # ordinary norms on the other side
            rho = np.random.default_rng(i).uniform(0.5, 2.0, c.rho.shape).astype(np.float32)
            c.rho = rho
            for s, length in enumerate(w["seq_lens"]):
                for h in range(2):
                    p = np.arange(length)
                    c.norms[s, h][:] = rho[c.table[s, p // 16], h, p % 16]
    out, lse = iq.isoq_kv_attn(**device(w), scale=0.05)
    check(out, lse, reference(w, 0.05))


@pytest.mark.parametrize("norm", [1e-15, 1e15])
def test_many_key_norms(norm):
    """Key norms at both ends of what the encoder takes, logits of ordinary size."""
    w = setup("full", 128, 3, "f16", [33], 2, 2, 16, [200], seed=3)
    c = w["sides"][0][2]
    c.rho = np.float32(c.rho * np.float32(norm))
    for h in range(2):
        p = np.arange(200)
        c.norms[0, h][:] = c.rho[c.table[0, p // 16], h, p % 16]
    out, lse = iq.isoq_kv_attn(**device(w), scale=1.0 / norm)
    check(out, lse, reference(w, 1.0 / norm))


def test_many_sink():
    """One position takes half of the weight, thousands share the rest (logits: the sink's ln 6000)."""
    n = 6000

    def keys(s, h, length):
        rng = np.random.default_rng(s + h)
        idx = rng.integers(0, 8, (length, 128)).astype(np.uint8)
        rho = np.full(length, 1e-3, np.float32)
        rho[17], idx[17] = 8.0, 7
        return idx, rho
    w = setup("full", 128, 3, "f16", [32], 1, 1, 16, [n], keys=keys, seed=1)
    (_, rot, c) = w["sides"][0]
    x = oracle.dequantize("full", 128, 3, rot, w["levels"], c.idx[0, 0][17:18], np.ones(1))[0]
    w["q"][:] = (x / (x @ x) * np.log(n) / 8.0)[None, None]
    cv = w["sides"][1][2]
    cv.norms[0, 0][:] = 1.0
    cv.rho = np.where(np.isnan(cv.rho), cv.rho, np.float32(1.0))
    out, lse = iq.isoq_kv_attn(**device(w), scale=1.0)
    check(out, lse, reference(w, 1.0))


@pytest.mark.parametrize("bits,ratio,scale", [(2, 3.0, 1.0), (3, 30.0, 1.0), (4, 30.0, 1.0), (3, 1e4, 1.0), (4, 300.0, 1.0),
                                              (3, 4.0, 2.0 ** -110), (4, 4.0, 2.0 ** 40)])
def test_many_codebooks(bits, ratio, scale):
    """Other codebooks: a level in one fp16 part is off by half a step, 2^-11 of
    itself, at most (codebooks of distant or of very small levels are decoded in
    fp32 by another kernel)."""
    k = 1 << (bits - 1)
    pos = 0.1 * ratio ** (np.arange(k) / (k - 1) - 1.0)
    lev = np.concatenate([-pos[::-1], pos]) * scale
    lev = np.float32(lev).astype(np.float64)
    w = setup("full", 128, bits, "f16", [20, 33], 4, 2, 16, [300, 90], levels=lev, seed=bits, norm=1.0)
    for _, _, c in w["sides"]:   # values and logits of ordinary size
        c.rho = np.float32(c.rho / np.float32(scale))
        for s in range(2):
            for h in range(2):
                p = np.arange(w["seq_lens"][s])
                c.norms[s, h][:] = c.rho[c.table[s, p // 16], h, p % 16]
    out, lse = iq.isoq_kv_attn(**device(w), scale=1.3)
    ref = {k: (o, l, bo + 2.0 ** -11 * vn, bl)
           for (k, (o, l, bo, bl)), vn in zip(reference(w, 1.3).items(), weighted_norms(w, 1.3))}
    check(out, lse, ref)


def weighted_norms(w, scale):
    """sum p rho ||c[idx]|| of the values per row, in reference()'s order."""
    g = w["q"].shape[1] // w["n_kv"]
    per = oracle.raw_params_per_set(w["variant"], w["d"])
    at = 0
    for s, n in enumerate(w["q_lens"]):
        for h in range(w["n_kv"]):
            (_, rk, ck), (_, _, cv) = w["sides"]
            kx = oracle.dequantize(w["variant"], w["d"], w["bits"], np.asarray(rk).reshape(-1)[h * per:][:per], w["levels"],
                                   ck.idx[s, h], ck.norms[s, h].astype(np.float64))
            vn = cv.norms[s, h].astype(np.float64) * np.linalg.norm(w["levels"][cv.idx[s, h]], axis=1)
            for i in range(n):
                lim = max(0, w["seq_lens"][s] - (n - 1 - i))
                for hq in range(h * g, h * g + g):
                    t = scale * (kx[:lim] @ w["q"][at + i, hq].astype(np.float64))
                    p = np.exp(t - t.max()) if lim else t
                    yield p @ vn[:lim] / p.sum() if lim else 0.0
        at += n


def test_many_streams_and_graphs():
    """Two streams at once and two graphs, each with buffers of its own: the bits of one call alone."""
    ws = [setup("fast", 128, 3, "f16", [40, 7], 8, 2, 16, [3000, 900], seed=s) for s in (12, 13)]
    args = [device(w) for w in ws]
    alone = [iq.isoq_kv_attn(**a) for a in args]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [[], []]
    for _ in range(3):
        for i in (0, 1):
            got[i].append(iq.isoq_kv_attn(**args[i], stream=streams[i]))
    torch.cuda.synchronize()
    for i in (0, 1):
        for o, l in got[i]:
            assert torch.equal(o, alone[i][0]) and torch.equal(l, alone[i][1])
    graphs, outs = [], []
    for i in (0, 1):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(iq.isoq_kv_attn(**args[i]))
        graphs.append(g)
    for _ in range(3):
        for o in outs:
            o[0].fill_(0)
            o[1].fill_(0)
        torch.cuda.synchronize()
        for i in (0, 1):
            with torch.cuda.stream(streams[i]):
                graphs[i].replay()
        torch.cuda.synchronize()
        again = iq.isoq_kv_attn(**args[0])
        torch.cuda.synchronize()
        for i in (0, 1):
            assert torch.equal(outs[i][0], alone[i][0]) and torch.equal(outs[i][1], alone[i][1])
        assert torch.equal(again[0], alone[0][0]) and torch.equal(again[1], alone[0][1])


def test_max_q_len_by_default():
    """Without max_q_len every token that q_start gives is computed."""
    w = setup("full", 128, 3, "f16", [9, 1, 30], 2, 2, 16, [50, 30, 300], seed=2)
    args = device(w)
    del args["max_q_len"]
    out, lse = iq.isoq_kv_attn(**args, scale=1.3)
    check(out, lse, reference(w, 1.3))
    none = iq.isoq_kv_attn(**dict(args, q=args["q"][:0], q_start=torch.zeros(4, dtype=torch.int32, device="cuda")))
    assert none[0].shape == (0, 2, 128) and none[1].shape == (0, 2)


def test_rows_do_not_depend_on_their_company():
    """A token's result is the same bits whatever other sequences the call has (splits alike)."""
    w = setup("full", 128, 3, "f16", [40, 40], 4, 2, 16, [500, 300], seed=2)
    args = device(w)
    both = iq.isoq_kv_attn(**args)
    start = torch.tensor([0, 40], dtype=torch.int32, device="cuda")
    one = iq.isoq_kv_attn(**dict(args, q=args["q"][:40].contiguous(), q_start=start,
                                 block_table=args["block_table"][:1].contiguous(), seq_lens=args["seq_lens"][:1]))
    assert torch.equal(one[0], both[0][:40]) and torch.equal(one[1], both[1][:40])
