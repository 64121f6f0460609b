"""Attention over the paged quantized cache (isoq_kv_attn) against its
definition in 64 bits: every key and value dequantized by the oracle, then
logits, softmax and the weighted sum in numpy.

Caches are built on the host (indices packed by the oracle's packer); slots
that no position uses hold norms of NaN, so a kernel that lets them in shows.

Tolerance, per row, against s_t, p_t (softmax) and ||v_t|| of the reference:
  logits    |ds| <= (pw + 8) 2^-23 max_t scale rho ||q|| ||c[idx]||, the bound
            of an fp32 sum of pw products (test_gpu_kv_scores.py; the digits of
            the matrix-core kernel stay inside it), + 4 2^-24 max |s| for the
            logit in units of ln 2;
  weights   relative 2 |ds| + 2^-19 (two exponentials, rescalings of the running
            maximum and a sum over lanes, splits and positions in fp32);
  values    a level is off by at most 1 / (2^15 - 129) of the largest one (two
            digits, fp16) or 2^-22 of it (fp32): rho c_max sqrt(pw) times that;
  the sum   2^-20 of sum p ||v||, and half a step of fp16, 2^-11, of the output
            (fp32: 2^-22, with the rotation back);
lse: |ds| + 2^-19 (a sum of exponentials) + 2^-22 |lse|.
Needs an MI355X."""
import numpy as np
import pytest

import oracle
import workloads

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

import paper_2603_28430_amd as iq  # noqa: E402
from paper_2603_28430_amd import isoquant as binding  # noqa: E402
import test_gpu_kv_scores as plain  # noqa: E402

CANARY = -12345.0


def setup(variant, d, bits, dtype, q_lens, n_q, n_kv, bs, seq_lens, n_sets=None, seed=0, levels=None, keys=None,
          norm=1.0, pad_rows=0):
    """One call's data: handles, host caches, queries (host), device arguments."""
    rng = np.random.default_rng(seed)
    n_sets = n_kv if n_sets is None else n_sets
    pw = oracle.padded_width(variant, d)
    levels = oracle.codebook(bits, d) if levels is None else levels
    sides = []
    for k in (0, 1):
        rot = workloads.rotation_draws(variant, d, n_sets, seed + 1 + k)
        p = iq.isoq_params_init(variant, d, bits, n_sets, rot=rot, codebook=levels)
        c = plain.Cache(rng, d, bits, len(seq_lens), n_kv, bs, seq_lens, keys=keys, pw=pw)
        if k:   # one block table serves both caches: the values' own, moved
            c.rec, c.rho = c.rec.copy(), c.rho.copy()
            new_rec, new_rho = np.zeros_like(c.rec), np.zeros_like(c.rho)
            for s, row in enumerate(c.table):
                for j, b in enumerate(row):
                    if b >= 0:
                        new_rec[sides[0][2].table[s, j]], new_rho[sides[0][2].table[s, j]] = c.rec[b], c.rho[b]
            c.rec, c.rho, c.table = new_rec, new_rho, sides[0][2].table
        c.rho = np.where(c.rho == 0, np.float32(np.nan), c.rho)
        sides.append((p, rot, c))
    ndt = np.float16 if dtype == "f16" else np.float32
    n = sum(q_lens)
    q = (workloads.unit_gaussian_rows((n + pad_rows) * n_q, d, seed=seed + 7, dtype=np.float64) *
         rng.uniform(0.5, 4.0 * norm, ((n + pad_rows) * n_q, 1))).astype(ndt).reshape(n + pad_rows, n_q, d)
    return dict(sides=sides, q=q, levels=np.float32(levels).astype(np.float64), n_sets=n_sets, variant=variant, d=d,
                bits=bits, q_lens=q_lens, seq_lens=seq_lens, n_kv=n_kv, bs=bs, pw=pw, dtype=dtype)


def device(w):
    (pk, _, ck), (pv, _, cv) = w["sides"]
    k_idx, k_rho, table, lens = ck.device()
    v_idx, v_rho, _, _ = cv.device()
    kw = dict(pk=pk, q=torch.from_numpy(w["q"]).cuda(), k_idx=k_idx, k_rho=k_rho, pv=pv, v_idx=v_idx, v_rho=v_rho,
              block_table=table, seq_lens=lens)
    if any(n != 1 for n in w["q_lens"]):
        kw["q_start"] = torch.from_numpy(np.concatenate([[0], np.cumsum(w["q_lens"])]).astype(np.int32)).cuda()
        kw["max_q_len"] = max(1, max(w["q_lens"]))
    return kw


def reference(w, scale, max_len=None, valid=None):
    """Per (token, query head): (out, lse, bound of ||out||, bound of lse).  valid: [seqs, positions], pages there."""
    f16 = w["dtype"] == "f16"
    lev, pw, bits, d = w["levels"], w["pw"], w["bits"], w["d"]
    g = w["q"].shape[1] // w["n_kv"]
    per = oracle.raw_params_per_set(w["variant"], d)
    res, at = {}, 0
    for s, n in enumerate(w["q_lens"]):
        length = w["seq_lens"][s]
        for h in range(w["n_kv"]):
            rows = []
            for p, rot, c in w["sides"]:
                r = np.asarray(rot).reshape(-1)[(h if w["n_sets"] > 1 else 0) * per:][:per]
                idx, rho = c.idx[s, h], c.norms[s, h].astype(np.float64)
                rows.append((oracle.dequantize(w["variant"], d, bits, r, lev, idx, rho) if len(rho)
                             else np.zeros((0, d)), rho, np.linalg.norm(lev[idx], axis=1) if len(rho) else np.zeros(0)))
            (kx, krho, kc), (vx, vrho, vc) = rows
            for i in range(n):
                lim = length - (n - 1 - i)
                lim = max(0, lim if max_len is None else min(lim, max_len))
                on = np.arange(len(krho)) < lim
                if valid is not None:
                    on &= valid[s, :len(krho)]
                for hq in range(h * g, h * g + g):
                    q = w["q"][at + i, hq].astype(np.float64)
                    if not on.any():
                        res[at + i, hq] = (np.zeros(d), -np.inf, 0.0, 0.0)
                        continue
                    t = scale * (kx[on] @ q)
                    m = t.max()
                    p = np.exp(t - m)
                    lse = m + np.log(p.sum())
                    p /= p.sum()
                    o = p @ vx[on]
                    ds = (pw + 8) * 2.0 ** -23 * abs(scale) * np.linalg.norm(q) * (krho[on] * kc[on]).max() + \
                        2.0 ** -22 * np.abs(t).max()
                    vn = p @ (vrho[on] * vc[on])
                    lv = (1 / 32639 if f16 else 2.0 ** -22) * lev.max() * np.sqrt(pw) * (p @ vrho[on])
                    step = 2.0 ** -11 if f16 else 2.0 ** -22
                    # (fp16 below its smallest normal number: half of 2^-24 a coordinate)
                    sub = 2.0 ** -25 * np.sqrt(d) if f16 else 0.0
                    res[at + i, hq] = (o, lse, (2 * ds + 2.0 ** -19 + 2.0 ** -20) * vn + lv + step * np.linalg.norm(o) + sub,
                                       ds + 2.0 ** -19 + 2.0 ** -22 * abs(lse))
        at += n
    return res


def check(out, lse, ref):
    out, lse = out.cpu().numpy().astype(np.float64), lse.cpu().numpy().astype(np.float64)
    for (t, hq), (o, l, bo, bl) in ref.items():
        if np.isinf(l):
            assert lse[t, hq] == -np.inf and np.all(out[t, hq] == 0), (t, hq, lse[t, hq])
            continue
        err = np.linalg.norm(out[t, hq] - o)
        assert err <= bo, (t, hq, err, bo, np.linalg.norm(o))
        assert abs(lse[t, hq] - l) <= bl, (t, hq, lse[t, hq], l, bl)


def run_case(variant, d, bits, dtype, q_lens, n_q, n_kv, bs, seq_lens, scale=None, max_len=None, pad_rows=2, **kw):
    print(f"case {variant} d={d} b={bits} {dtype} q_lens={list(q_lens)[:6]} heads={n_q}/{n_kv} bs={bs} "
          f"lens={list(seq_lens)[:6]} max_len={max_len} {kw}", flush=True)
    pad_rows = 0 if all(n == 1 for n in q_lens) else pad_rows
    w = setup(variant, d, bits, dtype, q_lens, n_q, n_kv, bs, seq_lens, pad_rows=pad_rows, **kw)
    scale = 1.3 if scale is None else scale
    args = device(w)
    out = torch.full_like(args["q"], CANARY)
    lse = torch.full(args["q"].shape[:2], CANARY, device="cuda")
    iq.isoq_kv_attn(**args, scale=scale, max_len=max_len, out=out, lse=lse)
    torch.cuda.synchronize()
    n = sum(q_lens)
    check(out, lse, reference(w, scale, max_len))
    assert torch.all(out[n:] == torch.full_like(out[n:], CANARY)) and torch.all(lse[n:] == CANARY), \
        "rows behind the last sequence were written"
    return w, args, out, lse


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("bits", [2, 3, 4])
@pytest.mark.parametrize("variant", ["full", "fast", "2d", "8d"])
def test_attn_d128(variant, bits, dtype):
    run_case(variant, 128, bits, dtype, [1, 1, 1], n_q=4, n_kv=2, bs=16, seq_lens=[1100, 17, 300], seed=bits)


@pytest.mark.parametrize("bits", [2, 3, 4])
@pytest.mark.parametrize("d", [64, 80, 96, 160, 192, 256, 512])
def test_attn_widths(d, bits):
    run = d // 16 + bits
    run_case(("full", "fast", "2d", "8d")[run % 4], d, bits, "f16" if run % 2 else "f32", [1, 1], n_q=6, n_kv=2,
             bs=(16, 7)[run % 2], seq_lens=[530, 65], seed=run)


@pytest.mark.parametrize("variant,d,bits,dtype", [("full", 100, 3, "f16"), ("2d", 98, 4, "f16"), ("2d", 7, 3, "f32"),
                                                  ("8d", 9, 2, "f32"), ("full", 13, 4, "f32"), ("fast", 1000, 3, "f16"),
                                                  ("full", 1, 2, "f16"), ("8d", 1024, 4, "f16"), ("2d", 250, 2, "f32"),
                                                  ("fast", 1024, 2, "f32"), ("8d", 40, 3, "f16")])
def test_attn_any_width(variant, d, bits, dtype):
    """Widths without a tuned kernel: zero-padded records, several tokens, more than one split."""
    run_case(variant, d, bits, dtype, [1, 3], n_q=6, n_kv=3, bs=16, seq_lens=[600, 37], seed=d + bits)


@pytest.mark.parametrize("group", [1, 2, 3, 4, 5, 7, 8, 9, 16, 17])
def test_attn_groups(group):
    run_case("fast", 128, 3, "f16", [1, 1], n_q=2 * group, n_kv=2, bs=16, seq_lens=[260, 77], seed=group)


@pytest.mark.parametrize("rows", [7, 10, 12, 19])
@pytest.mark.parametrize("bits", [2, 3, 4])
@pytest.mark.parametrize("d", [64, 80, 96, 128, 160, 192, 256])
def test_attn_rows_per_workgroup(d, bits, rows):
    """Row counts on both sides of what a workgroup takes, tokens of one head and heads of one token."""
    run = d // 16 + bits + rows
    dtype, variant = ("f16", "f32")[run % 2], ("full", "fast", "2d", "8d")[run % 4]
    run_case(variant, d, bits, dtype, [rows, 3], n_q=2, n_kv=2, bs=16, seq_lens=[330, 3], seed=run)
    run_case(variant, d, bits, dtype, [1, 1], n_q=rows, n_kv=1, bs=7, seq_lens=[270, 41], seed=run)


@pytest.mark.parametrize("d,dtype", [(128, "f16"), (96, "f32"), (100, "f16")])
def test_attn_lengths(d, dtype):
    """Around the tiles of 64 and 256 positions, empty and one-token sequences, a max_len that cuts."""
    lens = [0, 1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 255, 256, 257, 511, 513, 1025]
    run_case("full", d, 3, dtype, [1] * len(lens), n_q=2, n_kv=1, bs=16, seq_lens=lens, seed=d)
    run_case("full", d, 3, dtype, [1] * len(lens), n_q=2, n_kv=1, bs=5, seq_lens=lens, max_len=300, seed=d + 1)


def test_attn_one_rotation_set_and_xcd_order():
    """n_sets 1, and heads whose records do not end on a 128-byte line (heads in XCD order)."""
    run_case("fast", 96, 3, "f16", [1, 1], n_q=8, n_kv=8, bs=7, seq_lens=[300, 70], n_sets=1, seed=3)
    run_case("full", 128, 3, "f16", [1, 1], n_q=32, n_kv=16, bs=7, seq_lens=[300, 70], seed=4)


@pytest.mark.parametrize("d,bits,dtype", [(128, 3, "f16"), (64, 4, "f32"), (90, 2, "f16")])
def test_attn_many_splits(d, bits, dtype):
    """One sequence, one head, a long cache: many splits, joined."""
    run_case("fast", d, bits, dtype, [1], n_q=2, n_kv=1, bs=16, seq_lens=[20000], scale=2.0, seed=d)


@pytest.mark.parametrize("q_lens,seq_lens", [([3, 1, 5, 2], [100, 1, 300, 64]), ([4, 0, 7], [3, 50, 7]),
                                             ([16, 1, 33], [530, 40, 33]), ([5, 130], [1000, 140])])
@pytest.mark.parametrize("d,bits,dtype,group", [(128, 3, "f16", 4), (64, 2, "f32", 1), (80, 4, "f16", 3),
                                                (256, 3, "f16", 2), (70, 3, "f32", 2)])
def test_attn_chunks(q_lens, seq_lens, d, bits, dtype, group):
    """Several new tokens a sequence, causal; more tokens than positions (rows
    without a key), sequences without tokens, rows behind the last one."""
    run_case("full", d, bits, dtype, q_lens, n_q=2 * group, n_kv=2, bs=16, seq_lens=seq_lens, seed=d)


def test_attn_chunk_prefill():
    """A whole prompt as one chunk."""
    run_case("fast", 128, 3, "f16", [300, 77], n_q=4, n_kv=2, bs=16, seq_lens=[300, 700], seed=5)


def test_attn_max_q_len_cuts():
    """Tokens of a sequence from max_q_len on are left as they were; the others keep their places."""
    w = setup("full", 128, 3, "f16", [6, 2], 2, 1, 16, [50, 30], seed=2)
    args = device(w)
    args["max_q_len"] = 4
    out, lse = torch.full_like(args["q"], CANARY), torch.full(args["q"].shape[:2], CANARY, device="cuda")
    iq.isoq_kv_attn(**args, out=out, lse=lse)
    ref = reference(w, 1.0)
    check(out, lse, {k: v for k, v in ref.items() if not 4 <= k[0] < 6})
    assert torch.all(lse[4:6] == CANARY) and torch.all(out[4:6] == torch.full_like(out[4:6], CANARY))


@pytest.mark.parametrize("d", [128, 90])
def test_attn_invalid_pages(d):
    """Pages outside the cache are left out, alone, in rows, and all of them."""
    w = setup("full", d, 3, "f16", [1, 1, 1], 4, 2, 16, [400, 33, 48], seed=9)
    args = device(w)
    table = w["sides"][0][2].table.copy()
    table[0, [0, 3, 4, 5, 6, 24]] = [-1, w["sides"][0][2].n_blocks, -7, 2 ** 31 - 1, -2 ** 31, -1]
    table[1, :] = -1
    valid = np.repeat((table >= 0) & (table < w["sides"][0][2].n_blocks), 16, axis=1)
    args["block_table"] = torch.from_numpy(table).cuda()
    out, lse = iq.isoq_kv_attn(**args, scale=1.3)
    check(out, lse, reference(w, 1.3, valid=valid))


@pytest.mark.parametrize("d,dtype", [(128, "f16"), (128, "f32"), (100, "f16")])
def test_attn_sink(d, dtype):
    """One position takes half of the weight, thousands share the rest: small
    weights are not lost next to a large one.  (Logits: the sink's ln 6000.)"""
    n = 6000

    def keys(s, h, length):
        rng = np.random.default_rng(s + h)
        idx = rng.integers(0, 8, (length, oracle.padded_width("full", d))).astype(np.uint8)
        rho = np.full(length, 1e-3, np.float32)
        rho[17] = 8.0
        idx[17] = 7
        return idx, rho
    w = setup("full", d, 3, dtype, [1], 2, 1, 16, [n], keys=keys, seed=1)
    # queries along the sink's key
    (p, rot, c) = w["sides"][0]
    lev = w["levels"]
    x = oracle.dequantize("full", d, 3, rot, lev, c.idx[0, 0][17:18], np.ones(1))[0]
    x /= x @ x
    w["q"][:] = (x * np.log(n) / 8.0)[None, None]
    # values all of norm one
    cv = w["sides"][1][2]
    cv.norms[0, 0][:] = 1.0
    cv.rho = np.where(np.isnan(cv.rho), cv.rho, np.float32(1.0))
    args = device(w)
    out, lse = iq.isoq_kv_attn(**args, scale=1.0)
    check(out, lse, reference(w, 1.0))


@pytest.mark.parametrize("scale", [0.0, 300.0, -2.0])
def test_attn_scales(scale):
    """Uniform weights, one-hot weights, a negative scale."""
    run_case("fast", 128, 3, "f32", [1, 1], n_q=4, n_kv=1, bs=16, seq_lens=[700, 40], scale=scale, seed=8)


@pytest.mark.parametrize("d,bits,ratio", [(128, 3, 1e4), (64, 4, 300.0), (128, 2, 1e6)])
def test_attn_wide_codebook(d, bits, ratio):
    """Codebooks whose levels differ much in size."""
    k = 1 << (bits - 1)
    pos = 0.1 * ratio ** (np.arange(k) / (k - 1) - 1.0)
    lev = np.concatenate([-pos[::-1], pos]).astype(np.float32).astype(np.float64)
    run_case("full", d, bits, "f32", [1], n_q=4, n_kv=2, bs=16, seq_lens=[300], levels=lev, seed=bits)


@pytest.mark.parametrize("norm", [1e-15, 1e15])
def test_attn_norms(norm):
    """Norms at both ends of what the encoder takes, logits of ordinary size."""
    def keys(s, h, length):
        rng = np.random.default_rng(s + 2 * h)
        return rng.integers(0, 8, (length, 128)).astype(np.uint8), rng.uniform(0.5, 2.0, length) * norm
    run_case("full", 128, 3, "f32", [1], n_q=2, n_kv=2, bs=16, seq_lens=[200], scale=1.0 / norm, keys=keys, seed=3)


@pytest.mark.parametrize("d", [128, 90])
@pytest.mark.parametrize("bad", [np.inf, -np.inf, np.nan])
def test_attn_nonfinite_query(d, bad):
    """NaN in the rows of such queries and nowhere else."""
    w = setup("full", d, 3, "f16", [1, 1], 6, 2, 16, [300, 40], seed=4)
    ref = reference(w, 1.0)
    w["q"][0, 1, 5] = bad
    w["q"][1, 3, 0] = bad
    out, lse = iq.isoq_kv_attn(**device(w), scale=1.0)
    for t, hq in ((0, 1), (1, 3)):
        assert torch.isnan(out[t, hq]).all() and torch.isnan(lse[t, hq])
        del ref[t, hq]
    check(out, lse, ref)


def test_attn_zero_rows():
    """Zero queries (uniform weights) and zero keys and values (norm 0)."""
    def keys(s, h, length):
        rng = np.random.default_rng(s)
        rho = rng.uniform(0.5, 1.0, length)
        rho[::3] = 0.0
        return rng.integers(0, 8, (length, 128)).astype(np.uint8), rho
    w = setup("full", 128, 3, "f16", [1, 1], 4, 2, 16, [200, 1], keys=keys, seed=6)
    for _, _, c in w["sides"]:
        c.rho = np.where(np.isnan(c.rho), np.float32(0), c.rho)
    w["q"][0, 2] = 0
    out, lse = iq.isoq_kv_attn(**device(w), scale=1.0)
    check(out, lse, reference(w, 1.0))


def test_attn_no_cache():
    """No cache blocks, no block-table columns, max_len 0: outputs of zero, lse -inf."""
    w = setup("full", 128, 3, "f16", [1, 1], 4, 2, 16, [20, 5], seed=6)
    args = device(w)
    for change in (dict(block_table=torch.zeros((2, 0), dtype=torch.int32, device="cuda")), dict(max_len=0),
                   {k: args[k][:0] for k in ("k_idx", "k_rho", "v_idx", "v_rho")}):
        out, lse = iq.isoq_kv_attn(**dict(args, **change))
        assert torch.all(out == 0) and torch.all(lse == -np.inf)


def test_attn_same_bits_twice_and_on_another_stream():
    """Results do not depend on the stream or on what ran before; a caller's
    workspace serves, and a workspace of another call's leftovers."""
    w = setup("fast", 128, 4, "f16", [1, 1], 16, 4, 16, [3000, 1111], seed=12)
    args = device(w)
    a = iq.isoq_kv_attn(**args)
    need = iq.isoq_kv_attn_workspace(args["pk"], args["pv"], torch.float16, 2, 1, 2, 16, 4, 16,
                                     args["block_table"].shape[1], args["block_table"].shape[1] * 16)
    assert need > 0
    ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    b = iq.isoq_kv_attn(**args, workspace=ws, stream=side)
    side.synchronize()
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    with torch.cuda.stream(side):
        c = iq.isoq_kv_attn(**args)
    side.synchronize()
    assert torch.equal(a[0], c[0]) and torch.equal(a[1], c[1])
    with pytest.raises(ValueError):
        iq.isoq_kv_attn(**args, workspace=ws[:need - 1])


def test_attn_graph():
    """Captured and replayed, with other queries and lengths and eager calls between."""
    w = setup("fast", 128, 3, "f16", [1, 1], 8, 2, 16, [2000, 900], seed=13)
    args = device(w)
    iq.isoq_kv_attn(**args)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, lse = iq.isoq_kv_attn(**args)
    gen = torch.Generator(device="cuda").manual_seed(1)
    for i in range(4):
        args["q"].copy_(torch.randn(args["q"].shape, generator=gen, device="cuda"))
        args["seq_lens"].copy_(torch.tensor([2000 - 300 * i, 900 - 400 * (i % 2)], dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        eager = iq.isoq_kv_attn(**args)
        torch.cuda.synchronize()
        assert torch.equal(out, eager[0]) and torch.equal(lse, eager[1]), i


def test_attn_refusals():
    """Argument values that the library refuses, by status."""
    lib, p = binding.lib, iq.isoq_params_init("full", 128, 3, 2)
    other = [iq.isoq_params_init(*x) for x in (("fast", 128, 3, 2), ("full", 64, 3, 2), ("full", 128, 2, 2),
                                               ("full", 128, 3, 3))]
    buf = torch.zeros(1 << 16, dtype=torch.uint8, device="cuda")
    b = buf.data_ptr()
    names = ("pk pv dtype q q_start n_tokens max_q_len n_seqs n_q_heads n_kv_heads k_idx k_rho v_idx v_rho n_blocks "
             "block_size table max_blocks lens max_len scale out lse ws ws_bytes stream").split()
    ok = dict(zip(names, (p.handle, p.handle, 1, b, None, 2, 1, 2, 4, 2, b, b, b, b, 1, 16, b, 1, b, 16, 1.0, b, b, b,
                          1 << 16, None)))

    def call(**kw):
        a = dict(ok, **kw)
        return lib.isoq_kv_attn(*(a[n] for n in names))
    for st, cases in ((3, [dict(pk=None), dict(pv=None), dict(q=None), dict(out=None), dict(lens=None), dict(table=None),
                           dict(k_idx=None), dict(k_rho=None), dict(v_idx=None), dict(v_rho=None),
                           dict(ws=None, max_len=4096, max_blocks=256)]),
                      (1, [dict(dtype=2), dict(n_tokens=-1), dict(n_seqs=-1), dict(max_q_len=0), dict(n_q_heads=3),
                           dict(n_q_heads=0), dict(n_kv_heads=0), dict(block_size=0), dict(max_blocks=-1),
                           dict(max_len=-1), dict(n_blocks=-1), dict(scale=float("inf")), dict(scale=float("nan")),
                           dict(n_tokens=3), dict(max_q_len=2), dict(n_kv_heads=4),
                           dict(ws_bytes=100, max_len=4096, max_blocks=256)] +
                       [dict(pv=o.handle) for o in other]),
                      (2, [dict(n_seqs=65536, n_tokens=65536), dict(max_blocks=1 << 28),
                           dict(q_start=b, max_q_len=1 << 22), dict(q_start=b, n_tokens=1 << 30)]),
                      (4, [{k: b + o} for k, o in (("q", 8), ("out", 8), ("k_idx", 8), ("v_idx", 4), ("k_rho", 2),
                                                   ("v_rho", 2), ("table", 2), ("lens", 1), ("lse", 2), ("ws", 4),
                                                   ("q_start", 2))])):
        for kw in cases:
            assert call(**kw) == st, (kw, st)
    assert call(n_tokens=0, n_seqs=0) == 0
