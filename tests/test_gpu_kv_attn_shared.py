"""Attention behind shared prefixes (isoq_kv_attn_prefix) and to all positions
(isoq_kv_attn_cross) against the definition in 64 bits, with the tolerances that
test_gpu_kv_attn.py derives: the sums run over the prefix's and the sequence's own
positions together, joined once more (fp32, inside the 2^-19 of the weights).

Prefixes are further sequences of test_gpu_kv_attn.py's caches, without tokens.  Each case
runs twice: short prefixes are read anew by every sequence, and with a wide prefix table
(as for 100,000 positions) by launches of their own for the rows of all.
Slots that no position uses hold norms of NaN.  Needs an MI355X."""
import numpy as np
import pytest

import oracle

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

import paper_2603_28430_amd as iq  # noqa: E402
from test_gpu_kv_attn import CANARY, check, device, setup  # noqa: E402


def reference(w, scale, prefix_of=None, full=False, max_len=None, max_prefix_len=None):
    """Per (token, query head): (out, lse, bound of ||out||, bound of lse), as test_gpu_kv_attn.reference; prefix_of:
    each sequence's prefix, a sequence of the cache, or None."""
    f16 = w["dtype"] == "f16"
    lev, pw, bits, d = w["levels"], w["pw"], w["bits"], w["d"]
    g = w["q"].shape[1] // w["n_kv"]
    per = oracle.raw_params_per_set(w["variant"], d)
    rows = {}

    def cached(s, h):
        if (s, h) not in rows:
            got = []
            for p, rot, c in w["sides"]:
                r = np.asarray(rot).reshape(-1)[(h if w["n_sets"] > 1 else 0) * per:][:per]
                idx, rho = c.idx[s, h], c.norms[s, h].astype(np.float64)
                got.append((oracle.dequantize(w["variant"], d, bits, r, lev, idx, rho) if len(rho) else np.zeros((0, d)),
                            rho, np.linalg.norm(lev[idx], axis=1) if len(rho) else np.zeros(0)))
            rows[s, h] = got
        return rows[s, h]

    res, at = {}, 0
    for s, n in enumerate(w["q_lens"]):
        for i in range(n):
            lim = w["seq_lens"][s] - (0 if full else n - 1 - i)
            lim = max(0, lim if max_len is None else min(lim, max_len))
            for h in range(w["n_kv"]):
                take = [(s, lim)]
                if prefix_of is not None and prefix_of[s] is not None:
                    plen = w["seq_lens"][prefix_of[s]]
                    take.append((prefix_of[s], plen if max_prefix_len is None else min(plen, max_prefix_len)))
                (kx, krho, kc), (vx, vrho, vc) = [
                    [np.concatenate([cached(t, h)[side][k][:m] for t, m in take]) for k in range(3)] for side in (0, 1)]
                for hq in range(h * g, h * g + g):
                    q = w["q"][at + i, hq].astype(np.float64)
                    if not len(krho):
                        res[at + i, hq] = (np.zeros(d), -np.inf, 0.0, 0.0)
                        continue
                    t = scale * (kx @ q)
                    m = t.max()
                    p = np.exp(t - m)
                    lse = m + np.log(p.sum())
                    p /= p.sum()
                    o = p @ vx
                    ds = (pw + 8) * 2.0 ** -23 * abs(scale) * np.linalg.norm(q) * (krho * kc).max() + 2.0 ** -22 * np.abs(t).max()
                    vn = p @ (vrho * vc)
                    lv = (1 / 32639 if f16 else 2.0 ** -22) * lev.max() * np.sqrt(pw) * (p @ vrho)
                    step, sub = (2.0 ** -11, 2.0 ** -25 * np.sqrt(d)) if f16 else (2.0 ** -22, 0.0)
                    res[at + i, hq] = (o, lse, (2 * ds + 2.0 ** -19 + 2.0 ** -20) * vn + lv + step * np.linalg.norm(o) + sub,
                                       ds + 2.0 ** -19 + 2.0 ** -22 * abs(lse))
        at += n
    return res


def prefix_case(variant, d, bits, dtype, q_lens, n_q, n_kv, bs, seq_lens, prefix_lens, counts=None, first=0, pad_rows=2,
                scale=1.3, seed=0, **kw):
    """Sequences with prefixes of which the k-th is shared by counts[k] of them, from sequence `first` on (counts None:
    one, without prefix_start).  Returns (world, call arguments, tensors out and lse as the call left them)."""
    print(f"case {variant} d={d} b={bits} {dtype} q_lens={list(q_lens)[:6]} heads={n_q}/{n_kv} bs={bs} lens={list(seq_lens)[:6]} "
          f"prefixes={list(prefix_lens)} counts={counts} {kw}", flush=True)
    n, m = len(q_lens), len(prefix_lens)
    one = all(x == 1 for x in q_lens)
    w = setup(variant, d, bits, dtype, list(q_lens) + [0] * m, n_q, n_kv, bs, list(seq_lens) + list(prefix_lens), seed=seed,
              pad_rows=0 if one else pad_rows)
    args = device(w)
    table, lens = args["block_table"], args["seq_lens"]
    args.update(block_table=table[:n].contiguous(), seq_lens=lens[:n].contiguous(), prefix_table=table[n:].contiguous(),
                prefix_lens=lens[n:].contiguous(), scale=scale)
    if one:
        args.pop("q_start", None), args.pop("max_q_len", None)
    else:
        args["q_start"] = args["q_start"][:n + 1].contiguous()
    prefix_of = [n] * n
    if counts is not None:
        starts = first + np.concatenate([[0], np.cumsum(counts)])
        args["prefix_start"] = torch.from_numpy(starts.astype(np.int32)).cuda()
        prefix_of = [None] * n
        for p, c in enumerate(counts):
            prefix_of[starts[p]:starts[p + 1]] = [n + p] * c
        used = [sum(q_lens[starts[p]:starts[p + 1]]) for p in range(m)]
        args["max_prefix_tokens"] = max(1, max(used))
    args.update(kw)
    ref = reference(w, scale, prefix_of, max_len=kw.get("max_len"), max_prefix_len=kw.get("max_prefix_len"))
    total = sum(q_lens)
    narrow = args["prefix_table"]
    for table in (widen(narrow, bs), narrow):
        args["prefix_table"] = table
        out = torch.full_like(args["q"], CANARY)
        lse = torch.full(args["q"].shape[:2], CANARY, device="cuda")
        iq.isoq_kv_attn_prefix(**args, out=out, lse=lse)
        torch.cuda.synchronize()
        check(out, lse, ref)
        assert torch.all(out[total:] == torch.full_like(out[total:], CANARY)) and torch.all(lse[total:] == CANARY)
    return w, args, out, lse


def widen(table, bs, positions=100000):
    """A prefix table of so many positions, the further entries outside the cache."""
    more = max(0, -(-positions // bs) - table.shape[1])
    return torch.cat([table, table.new_full((table.shape[0], more), -5)], 1).contiguous()


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("bits", [2, 3, 4])
@pytest.mark.parametrize("variant", ["full", "fast", "2d", "8d"])
def test_one_prefix(variant, bits, dtype):
    prefix_case(variant, 128, bits, dtype, [1] * 5, 4, 2, 16, [60, 1, 130, 0, 17], [500], seed=bits)


@pytest.mark.parametrize("bits", [2, 3, 4])
@pytest.mark.parametrize("d", [64, 80, 96, 160, 192, 256, 512, 100, 7])
def test_widths(d, bits):
    run = d // 16 + bits
    prefix_case(("full", "fast", "2d", "8d")[run % 4], d, bits, "f16" if run % 2 else "f32", [1, 1, 1], 6, 2, (16, 7)[run % 2],
                [53, 65, 2], [330], seed=run)


@pytest.mark.parametrize("n", [1, 2, 3, 7, 16, 33, 70])
@pytest.mark.parametrize("d,dtype,group", [(128, "f16", 4), (64, "f16", 1), (96, "f32", 2), (192, "f16", 3)])
def test_numbers_of_sequences(n, d, dtype, group):
    """From a few rows to several workgroups of rows, own positions of 0 to 40."""
    rng = np.random.default_rng(n + d)
    prefix_case("fast", d, 3, dtype, [1] * n, 2 * group, 2, 16, list(rng.integers(0, 40, n)), [290], seed=n)


@pytest.mark.parametrize("plen", [0, 1, 15, 16, 17, 63, 64, 65, 127, 128, 129, 255, 257, 513, 767, 769, 1030])
def test_prefix_lengths(plen):
    prefix_case("full", 128, 3, "f16", [1] * 9, 4, 1, 16, [0, 1, 5, 16, 63, 64, 65, 128, 300], [plen], seed=plen)
    prefix_case("2d", 64, 4, "f32", [1] * 3, 2, 1, 5, [0, 3, 70], [plen], seed=plen + 1)


@pytest.mark.parametrize("counts,first", [([2, 3, 1], 0), ([1, 1, 1], 2), ([0, 6, 0], 0), ([3, 0, 2], 1), ([0, 0, 0], 4), ([6, 0, 0], 0)])
@pytest.mark.parametrize("d,dtype", [(128, "f16"), (80, "f32"), (90, "f16")])
def test_groups_of_sequences(counts, first, d, dtype):
    """Several prefixes, of none, one or more sequences, an empty prefix, and sequences of no prefix on either side."""
    prefix_case("full", d, 3, dtype, [1] * 6, 4, 2, 16, [30, 0, 100, 7, 0, 64], [200, 0, 77], counts, first, seed=d)


@pytest.mark.parametrize("q_lens,seq_lens", [([3, 1, 5, 2], [100, 1, 300, 64]), ([4, 0, 7, 1], [3, 50, 7, 0]), ([40, 1, 33], [130, 40, 33])])
@pytest.mark.parametrize("d,bits,dtype,group", [(128, 3, "f16", 4), (64, 2, "f32", 1), (80, 4, "f16", 3), (256, 3, "f16", 2), (70, 3, "f32", 2)])
def test_several_tokens(q_lens, seq_lens, d, bits, dtype, group):
    """Drafts and chunks: causal among themselves, all of the prefix; rows without a key, sequences without tokens."""
    n = len(q_lens)
    prefix_case("full", d, bits, dtype, q_lens, 2 * group, 2, 16, seq_lens, [150], seed=d)
    prefix_case("fast", d, bits, dtype, q_lens, 2 * group, 2, 16, seq_lens, [150, 0, 33], [1, 1, n - 2], seed=d + 1)


def test_many_splits():
    """More splits than the join of few takes, of the prefix, of the sequences and of both."""
    prefix_case("fast", 128, 3, "f16", [1] * 40, 2, 1, 16, [5] * 39 + [4000], [12000], seed=5)   # (both launches, both with splits)
    prefix_case("full", 192, 4, "f32", [1] * 9, 2, 1, 16, [5] * 8 + [2000], [9000], seed=6)
    prefix_case("fast", 128, 3, "f16", [1], 2, 1, 16, [30], [20000], seed=1)
    prefix_case("fast", 64, 4, "f32", [1], 2, 1, 16, [15000], [20], seed=2)
    prefix_case("fast", 128, 2, "f16", [1, 1], 2, 1, 16, [9000, 3], [12000], seed=3)
    prefix_case("full", 90, 3, "f16", [1, 1], 2, 1, 16, [3000, 0], [5000], seed=4)


def test_bounds_that_cut():
    """max_len and max_prefix_len below the lengths; max_prefix_tokens below a prefix's tokens: those rows are left alone."""
    prefix_case("full", 128, 3, "f16", [1] * 3, 4, 2, 16, [100, 30, 65], [300], max_len=64, max_prefix_len=130, seed=1)
    w, args, out, lse = prefix_case("full", 128, 3, "f16", [2, 3, 2, 1], 4, 2, 16, [100, 30, 65, 9], [300, 40], [3, 1], seed=2)
    narrow = args["prefix_table"]
    for most, table in ((m, x) for m in (1, 2, 5, 6) for x in (narrow, widen(narrow, 16))):
        args["max_prefix_tokens"], args["prefix_table"] = most, table
        o, l = torch.full_like(out, CANARY), torch.full_like(lse, CANARY)
        iq.isoq_kv_attn_prefix(**args, out=o, lse=l)
        left = torch.arange(len(out), device="cuda")
        left = (left >= most) & (left < 7) | (left >= 8)
        assert torch.equal(o[~left].isnan(), out[~left].isnan()) and torch.all(l[left] == CANARY)
        assert torch.all(o[left] == torch.full_like(o[left], CANARY))
        assert (l[~left] - lse[~left]).abs().max() < 1e-4


def test_no_prefix_is_isoq_kv_attn():
    w, args, out, lse = prefix_case("full", 128, 3, "f16", [1] * 3, 4, 2, 16, [100, 0, 700], [0], seed=1)
    plain = {k: v for k, v in args.items() if not k.startswith("prefix")}
    ref = iq.isoq_kv_attn(**plain)
    for kw in (dict(prefix_table=args["prefix_table"][:, :0].contiguous()), dict(max_prefix_len=0),
               dict(prefix_table=args["prefix_table"][:0], prefix_lens=args["prefix_lens"][:0])):   # (no prefix at all)
        got = iq.isoq_kv_attn_prefix(**dict(args, **kw))
        assert torch.equal(got[0], ref[0]) and torch.equal(got[1], ref[1])


@pytest.mark.parametrize("wide", [False, True])
def test_bounds_of_tokens_and_an_empty_cache(wide):
    """No tokens of a prefix are refused (they would be left out), more than there are are as many as there are; a
    cache without blocks gives 0 and -inf, with the workspace that the call asks for."""
    w, args, out, lse = prefix_case("full", 128, 3, "f16", [1] * 5, 4, 2, 16, [100, 0, 70, 9, 40], [200, 40], [3, 1], seed=2)
    if wide:
        args["prefix_table"] = widen(args["prefix_table"], 16)
    for most in (0, -1):
        with pytest.raises(iq.IsoqError):
            iq.isoq_kv_attn_prefix(**dict(args, max_prefix_tokens=most))
    a, b = (iq.isoq_kv_attn_prefix(**dict(args, max_prefix_tokens=most)) for most in (2 ** 40, 5))
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    none = {x: args[x][:0] for x in ("k_idx", "k_rho", "v_idx", "v_rho")}
    for kw in ({}, dict(block_table=widen(args["block_table"], 16))):
        got = iq.isoq_kv_attn_prefix(**dict(args, **none, **kw))
        assert (got[0] == 0).all() and (got[1] == -float("inf")).all()


def test_empty_rows_whatever_the_query_holds():
    """Neither prefix nor own positions: out 0 and lse -inf, also of a query that is no number; with a position, NaN."""
    w, args, out, lse = prefix_case("full", 128, 3, "f16", [1] * 4, 4, 2, 16, [0, 0, 3, 0], [0, 20], [3, 1], seed=5)
    args["q"][0] = float("nan")
    args["q"][2, 1] = float("inf")
    args["q"][3, 0] = float("nan")
    for table in (args["prefix_table"], widen(args["prefix_table"], 16)):
        out, lse = iq.isoq_kv_attn_prefix(**dict(args, prefix_table=table))
        empty_rows(out, lse)


def empty_rows(out, lse):
    assert (out[:2] == 0).all() and (lse[:2] == -float("inf")).all()
    assert lse[2, 1].isnan() and lse[3, 0].isnan() and out[3, 0].isnan().all()
    assert lse[2, 0].isfinite() and lse[3, 1:].isfinite().all()


@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("d", [128, 90])
def test_invalid_pages_and_odd_norms(d, wide):
    """Prefix blocks outside the cache are left out; a norm that is no number reaches the rows that share it, not others."""
    w, args, out, lse = prefix_case("full", d, 3, "f16", [1] * 4, 4, 2, 16, [20, 5, 40, 0], [100, 64], [2, 2], seed=d)
    if wide:
        args["prefix_table"] = widen(args["prefix_table"], 16)
    good = iq.isoq_kv_attn_prefix(**args)
    bad = args["prefix_table"].clone()
    bad[0, 1:6] = torch.tensor([-1, 10 ** 6, -7, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32)
    cut = iq.isoq_kv_attn_prefix(**dict(args, prefix_table=bad))
    short = iq.isoq_kv_attn_prefix(**dict(args, prefix_table=torch.where(bad < 0, -1, bad), prefix_lens=args["prefix_lens"]))
    assert torch.equal(cut[0], short[0]) and torch.equal(cut[0][2:], good[0][2:])
    only = iq.isoq_kv_attn_prefix(**dict(args, prefix_lens=torch.tensor([16, 64], dtype=torch.int32, device="cuda")))
    # (blocks 1 .. 5 are gone, block 6 holds positions 96 .. 99)
    assert not torch.equal(cut[0][:2], only[0][:2])
    bad[0, 6] = -1
    cut = iq.isoq_kv_attn_prefix(**dict(args, prefix_table=bad))
    assert (cut[1] - only[1])[:2].abs().max() < 1e-4
    rho = args["k_rho"].clone()
    rho[int(args["prefix_table"][0, 0]), 0, 3] = float("nan")
    got = iq.isoq_kv_attn_prefix(**dict(args, k_rho=rho))
    assert got[1][:2, :2].isnan().all() and got[1][:2, 2:].isfinite().all() and torch.equal(got[0][2:], good[0][2:])


@pytest.mark.parametrize("wide", [False, True])
def test_streams_workspaces_and_graphs(wide):
    """A stream and a workspace of its own; two graphs with a workspace each, replayed with other lengths and eager work between."""
    w, args, out, lse = prefix_case("full", 128, 3, "f16", [1] * 20, 8, 2, 16, list(range(20)), [700], seed=7)
    if wide:
        args["prefix_table"] = widen(args["prefix_table"], 16)
        out, lse = iq.isoq_kv_attn_prefix(**args)
    n_seqs, blocks = args["block_table"].shape
    shared = args["prefix_table"].shape[1]
    need = iq.isoq_kv_attn_prefix_workspace(args["pk"], args["pv"], torch.float16, 20, 1, n_seqs, 8, 2, 16, blocks,
                                            blocks * 16, 1, 20, shared, shared * 16)
    assert need > 0
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = iq.isoq_kv_attn_prefix(**args, workspace=ws, stream=stream)
    stream.synchronize()
    assert torch.equal(got[0], out) and torch.equal(got[1], lse)
    with pytest.raises(ValueError):
        iq.isoq_kv_attn_prefix(**args, workspace=ws[:need - 1])
    graphs = []
    for _ in range(2):
        wsg = torch.empty(need, dtype=torch.uint8, device="cuda")
        o, l = torch.empty_like(out), torch.empty_like(lse)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            iq.isoq_kv_attn_prefix(**args, workspace=wsg, out=o, lse=l)
        graphs.append((graph, o, l))
    for k in range(4):
        args["prefix_lens"].fill_((700, 64, 0, 333)[k])
        args["seq_lens"].copy_(torch.arange(20, device="cuda", dtype=torch.int32).flip(0) if k % 2 else
                               torch.arange(20, device="cuda", dtype=torch.int32))
        ref = iq.isoq_kv_attn_prefix(**args)
        for graph, o, l in graphs:
            o.fill_(CANARY)
            graph.replay()
        torch.cuda.synchronize()
        for graph, o, l in graphs:
            # (lengths past what the cache was filled to reach norms of NaN, whose rows are NaN in both)
            for a, b in ((o, ref[0]), (l, ref[1])):
                assert torch.equal(a.isnan(), b.isnan()) and torch.equal(a.nan_to_num(7.0), b.nan_to_num(7.0))


# ---- all positions -----------------------------------------------------------------------

def cross_case(variant, d, bits, dtype, q_lens, n_q, n_kv, bs, seq_lens, pad_rows=2, scale=1.3, seed=0, **kw):
    print(f"case {variant} d={d} b={bits} {dtype} q_lens={list(q_lens)[:6]} heads={n_q}/{n_kv} bs={bs} lens={list(seq_lens)[:6]}", flush=True)
    pad_rows = 0 if all(n == 1 for n in q_lens) else pad_rows
    w = setup(variant, d, bits, dtype, q_lens, n_q, n_kv, bs, seq_lens, pad_rows=pad_rows, seed=seed)
    args = dict(device(w), scale=scale, **kw)
    out = torch.full_like(args["q"], CANARY)
    lse = torch.full(args["q"].shape[:2], CANARY, device="cuda")
    iq.isoq_kv_attn_cross(**args, out=out, lse=lse)
    torch.cuda.synchronize()
    check(out, lse, reference(w, scale, full=True, max_len=kw.get("max_len")))
    n = sum(q_lens)
    assert torch.all(out[n:] == torch.full_like(out[n:], CANARY)) and torch.all(lse[n:] == CANARY)
    return w, args, out, lse


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("bits", [2, 3, 4])
@pytest.mark.parametrize("variant", ["full", "fast", "2d", "8d"])
def test_cross_variants(variant, bits, dtype):
    cross_case(variant, 128, bits, dtype, [3, 1, 9], 4, 2, 16, [300, 17, 5], seed=bits)


@pytest.mark.parametrize("bits", [2, 3, 4])
@pytest.mark.parametrize("d", [64, 80, 96, 160, 192, 256, 512, 100, 7])
def test_cross_widths(d, bits):
    run = d // 16 + bits
    cross_case(("full", "fast", "2d", "8d")[run % 4], d, bits, "f16" if run % 2 else "f32", [1, 5], 6, 2, (16, 7)[run % 2], [130, 65], seed=run)


@pytest.mark.parametrize("q_len", [1, 2, 12, 31, 32, 33, 64, 128, 129, 260])
@pytest.mark.parametrize("d,dtype", [(128, "f16"), (64, "f16"), (80, "f32"), (192, "f16")])
def test_cross_lengths(q_len, d, dtype):
    """Targets longer and shorter than their inputs, empty and one-position inputs among them."""
    cross_case("fast", d, 3, dtype, [q_len] * 5, 2, 2, 16, [0, 1, 63, 129, 40], seed=q_len)


def test_cross_no_targets_and_bounds():
    cross_case("full", 128, 3, "f16", [0, 4, 0, 33], 4, 2, 16, [50, 50, 0, 770], seed=1)
    cross_case("full", 128, 3, "f16", [2, 40], 4, 2, 16, [500, 200], max_len=100, seed=2)
    cross_case("full", 128, 3, "f16", [1, 1, 1], 4, 2, 16, [5000, 200, 0], seed=3)


def test_cross_of_one_token_is_causal():
    w, args, out, lse = cross_case("full", 96, 3, "f16", [1, 1, 1], 4, 2, 16, [500, 20, 0], seed=3)
    ref = iq.isoq_kv_attn(**args)
    assert torch.equal(out, ref[0]) and torch.equal(lse, ref[1])
