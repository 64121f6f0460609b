"""The cache's operators as a serving program runs them, one after the other on
one cache: prompts appended and attended as chunks, a sequence forked (its last
block copied, later all of them), tokens decoded one at a time by both, one of
them compacted by its own logits, and decoded further.  After each attention the
result is compared with the definition in 64 bits on what the cache holds then
(records dequantized by the oracle), within the tolerance of
test_gpu_kv_attn.py; the appended records are the ones isoq_quantize gives.
And the operators on caches whose byte offsets pass 2^32.  Needs an MI355X."""
import numpy as np
import pytest

import oracle
import workloads
from cache_layout import from_cache, to_cache

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

import paper_2603_28430_amd as iq  # noqa: E402
from test_gpu_kv_attn import check, device, reference, setup  # noqa: E402


class Server:
    """Host bookkeeping of a paged cache: block tables, lengths, and what each
    position holds (by the records that isoq_quantize gives)."""

    def __init__(self, variant, d, bits, dtype, n_q, n_kv, bs, n_blocks, max_blocks, seed):
        self.v, self.d, self.bits, self.n_q, self.n_kv, self.bs = variant, d, bits, n_q, n_kv, bs
        self.dtype, self.ndt = dtype, torch.float16 if dtype == "f16" else torch.float32
        self.levels = np.float32(oracle.codebook(bits, d)).astype(np.float64)
        self.pw = oracle.padded_width(variant, d)
        self.rot = [workloads.rotation_draws(variant, d, n_kv, seed + k) for k in (0, 1)]
        self.p = [iq.isoq_params_init(variant, d, bits, n_kv, rot=r) for r in self.rot]
        R = self.p[0].record_bytes
        self.idx = [torch.full((n_blocks, n_kv, bs, R), 255, dtype=torch.uint8, device="cuda") for _ in (0, 1)]
        self.rho = [torch.full((n_blocks, n_kv, bs), float("nan"), device="cuda") for _ in (0, 1)]
        self.free = list(np.random.default_rng(seed).permutation(n_blocks))
        self.table = np.full((0, max_blocks), -1, np.int32)
        self.lens = []
        self.gen = torch.Generator(device="cuda").manual_seed(seed)

    def rows(self, n, heads, size=1.0):
        return (torch.randn((n, heads, self.d), generator=self.gen, device="cuda") * size).to(self.ndt)

    def add(self):
        self.table = np.concatenate([self.table, np.full((1, self.table.shape[1]), -1, np.int32)])
        self.lens.append(0)
        return len(self.lens) - 1

    def fork(self, s, whole):
        """A sequence like s: sharing its full blocks, or with copies of all of them."""
        t = self.add()
        n = -(-self.lens[s] // self.bs)
        pairs = []
        for j in range(n):
            own = whole or (j + 1) * self.bs > self.lens[s]
            self.table[t, j] = self.free.pop() if own else self.table[s, j]
            if own:
                pairs.append((self.table[s, j], self.table[t, j]))
        iq.isoq_kv_copy_blocks(self.p[0], torch.tensor(pairs, dtype=torch.int32, device="cuda").reshape(-1, 2),
                               self.idx[0], self.rho[0], self.idx[1], self.rho[1])
        self.lens[t] = self.lens[s]
        return t

    def append(self, counts):
        """New tokens for the sequences (a dict), quantized into their slots."""
        slots = []
        for s, n in counts.items():
            for pos in range(self.lens[s], self.lens[s] + n):
                if self.table[s, pos // self.bs] < 0:
                    self.table[s, pos // self.bs] = self.free.pop()
                slots.append(int(self.table[s, pos // self.bs]) * self.bs + pos % self.bs)
            self.lens[s] += n
        k, v = self.rows(len(slots), self.n_kv), self.rows(len(slots), self.n_kv)
        iq.isoq_kv_append(self.p[0], k, torch.tensor(slots, device="cuda"), self.idx[0], self.rho[0], self.p[1], v,
                          self.idx[1], self.rho[1])
        slots = np.array(slots)
        for p, x, idx, rho in zip(self.p, (k, v), self.idx, self.rho):
            rec, norm = iq.isoq_quantize(p, x.reshape(-1, self.d), rows_per_set=1)
            rec, norm = rec.cpu().numpy().reshape(len(slots), self.n_kv, -1), norm.cpu().numpy().reshape(-1, self.n_kv)
            assert np.array_equal(from_cache(idx.cpu().numpy())[slots // self.bs, :, slots % self.bs], rec)
            assert np.array_equal(rho.cpu().numpy()[slots // self.bs, :, slots % self.bs], norm)

    def tables(self, seqs):
        return (torch.from_numpy(self.table[seqs]).cuda(),
                torch.tensor([self.lens[s] for s in seqs], dtype=torch.int32, device="cuda"))

    def attend(self, counts, scale):
        """Attention of the last tokens of the sequences, checked."""
        seqs, ns = list(counts), list(counts.values())
        q = self.rows(sum(ns), self.n_q, 2.0)
        table, lens = self.tables(seqs)
        more = {}
        if any(n != 1 for n in ns):
            more = dict(q_start=torch.tensor(np.concatenate([[0], np.cumsum(ns)]).astype(np.int32), device="cuda"),
                        max_q_len=max(ns))
        out, lse = iq.isoq_kv_attn(self.p[0], q, self.idx[0], self.rho[0], self.p[1], self.idx[1], self.rho[1], table,
                                   lens, scale=scale, **more)
        w = dict(sides=[(p, r, Held(self, i, seqs)) for i, (p, r) in enumerate(zip(self.p, self.rot))],
                 q=q.cpu().numpy(), levels=self.levels, n_sets=self.n_kv, variant=self.v, d=self.d, bits=self.bits,
                 q_lens=ns, seq_lens=[self.lens[s] for s in seqs], n_kv=self.n_kv, bs=self.bs, pw=self.pw, dtype=self.dtype)
        check(out, lse, reference(w, scale))
        return q, table, lens

    def compact(self, s, keep):
        """keep [heads or 1, n]: the positions of s that stay."""
        n = keep.shape[1]
        table, _ = self.tables([s])
        iq.isoq_kv_compact(self.p[0], torch.from_numpy(keep[None].astype(np.int32)).cuda(),
                           torch.tensor([n], dtype=torch.int32, device="cuda"), table, self.idx[0], self.rho[0],
                           self.idx[1], self.rho[1])
        self.lens[s] = n
        for j in range(-(-n // self.bs), self.table.shape[1]):
            if self.table[s, j] >= 0:
                self.free.append(self.table[s, j])
                self.table[s, j] = -1


class Held:
    """What the cache holds at the sequences' positions, as reference() reads it."""

    def __init__(self, srv, side, seqs):
        rec, rho = from_cache(srv.idx[side].cpu().numpy()), srv.rho[side].cpu().numpy()
        self.idx, self.norms = {}, {}
        for i, s in enumerate(seqs):
            pos = np.arange(srv.lens[s])
            blk = srv.table[s, pos // srv.bs]
            for h in range(srv.n_kv):
                self.idx[i, h] = oracle.unpack(rec[blk, h, pos % srv.bs], srv.pw, srv.bits).reshape(len(pos), srv.pw)
                self.norms[i, h] = rho[blk, h, pos % srv.bs]


@pytest.mark.parametrize("variant,d,bits,dtype,n_q,n_kv,bs", [("full", 128, 3, "f16", 8, 2, 16), ("fast", 64, 4, "f16", 4, 4, 7),
                                                              ("2d", 96, 2, "f32", 6, 2, 16), ("8d", 100, 3, "f16", 4, 1, 5)])
def test_a_run(variant, d, bits, dtype, n_q, n_kv, bs):
    srv = Server(variant, d, bits, dtype, n_q, n_kv, bs, n_blocks=200, max_blocks=-(-400 // bs), seed=d + bits)
    scale = d ** -0.5
    a, b = srv.add(), srv.add()
    srv.append({a: 150, b: 37})
    srv.attend({a: 150, b: 37}, scale)              # the prompts
    c = srv.fork(a, whole=False)
    held = from_cache(srv.idx[0].cpu().numpy())
    for _ in range(3):                              # three sequences, a token each
        srv.append({a: 1, b: 1, c: 1})
        srv.attend({a: 1, b: 1, c: 1}, scale)
    # (the fork's tokens went to its own block: the original's positions are as they were)
    now = from_cache(srv.idx[0].cpu().numpy())
    pos = np.arange(150)
    assert np.array_equal(now[srv.table[a, pos // bs], :, pos % bs], held[srv.table[a, pos // bs], :, pos % bs])
    e = srv.fork(c, whole=True)                     # blocks of its own: e can be compacted, c stays
    q, table, lens = srv.attend({e: 1}, scale)
    scores = iq.isoq_kv_scores(srv.p[0], q, srv.idx[0], srv.rho[0], table, lens, scale=scale)
    by_head = scores[0].reshape(n_kv, n_q // n_kv, -1).amax(1)[:, :srv.lens[e]]
    keep = np.sort(by_head.topk(61, dim=1).indices.cpu().numpy(), axis=1)
    before = Held(srv, 0, [e]), Held(srv, 1, [e])
    srv.compact(e, keep)
    for x, y in zip(before, (Held(srv, 0, [e]), Held(srv, 1, [e]))):
        for h in range(n_kv):
            assert np.array_equal(x.idx[0, h][keep[h]], y.idx[0, h]) and np.array_equal(x.norms[0, h][keep[h]], y.norms[0, h])
    for n in (1, 5, 1):                             # a draft of five among single tokens
        srv.append({a: 1, c: n, e: n})
        srv.attend({a: 1, c: n, e: n}, scale)
    srv.compact(e, np.arange(20, srv.lens[e] - 1)[None])   # a window, the same for every head
    srv.append({a: 30, b: 40, e: 45})
    srv.attend({a: 30, b: 40, e: 45}, scale)


def far(w, n_blocks):
    """The case's caches moved to the end of caches of n_blocks blocks (byte offsets past 2^32)."""
    args = device(w)
    shift = n_blocks - args["k_idx"].shape[0]
    for name in ("k_idx", "v_idx", "k_rho", "v_rho"):
        big = torch.zeros((n_blocks,) + args[name].shape[1:], dtype=args[name].dtype, device="cuda")
        big[shift:] = args[name]
        args[name] = big
    table = w["sides"][0][2].table
    args["block_table"] = torch.from_numpy(np.where(table >= 0, table + shift, table).astype(np.int32)).cuda()
    return args, shift


@pytest.mark.parametrize("d,bits,dtype,q_lens", [(128, 3, "f16", [1, 1]), (128, 4, "f32", [3, 1]), (64, 3, "f16", [40, 1]),
                                                 (100, 3, "f16", [2, 1])])
def test_attn_far_offsets(d, bits, dtype, q_lens):
    w = setup("full", d, bits, dtype, q_lens, 4, 4, 64, [500, 70], seed=d)
    block = 4 * 64 * w["sides"][0][0].record_bytes
    args, _ = far(w, (1 << 32) // block + 1000)
    assert args["k_idx"].numel() > 1 << 32
    out, lse = iq.isoq_kv_attn(**args, scale=1.3)
    check(out, lse, reference(w, 1.3))


@pytest.mark.parametrize("d,bits,q_len", [(64, 2, 1), (64, 3, 32), (16, 4, 1)])
def test_attn_longest_sequences(d, bits, q_len):
    """2,047 pages of 2^20 positions, all the same block: nearly 2^31 positions.
    Rows without a causal border inside the last page would be those of one page
    with lse + ln 2047; the last q_len - 1 - i positions that token i does not see
    are 1e-8 of the weights.  A lane adds up to 2^31 / 256 / 64 tiles' weights a
    split, an error of 2^17 2^-24 at most, of the output's norm too."""
    bs, pages = 1 << 20, 2047
    rng = np.random.default_rng(d)
    pk, pv = (iq.isoq_params_init("full", d, bits, 1, seed=s) for s in (1, 2))
    k_idx, v_idx = (torch.from_numpy(rng.integers(0, 256, (1, 1, bs, pk.record_bytes), dtype=np.uint8)).cuda() for _ in (0, 1))
    k_rho, v_rho = (torch.from_numpy(rng.uniform(0.5, 1.5, (1, 1, bs)).astype(np.float32)).cuda() for _ in (0, 1))
    q = torch.from_numpy(rng.standard_normal((q_len, 1, d)).astype(np.float16)).cuda()
    start = torch.tensor([0, q_len], dtype=torch.int32, device="cuda")

    def run(n):
        table = torch.zeros((1, n), dtype=torch.int32, device="cuda")
        lens = torch.tensor([n * bs], dtype=torch.int32, device="cuda")
        return iq.isoq_kv_attn(pk, q, k_idx, k_rho, pv, v_idx, v_rho, table, lens, scale=d ** -0.5, q_start=start,
                               max_q_len=q_len)
    (one, lse_one), (out, lse) = run(1), run(pages)
    torch.cuda.synchronize()
    assert ((lse - lse_one).double() - np.log(pages)).abs().max() < 2.0 ** -7
    assert (out.double() - one.double()).norm() < (2.0 ** -7 + 2.0 ** -10) * one.double().norm()


@pytest.mark.parametrize("d,dtype,q_len", [(64, "f32", 1), (64, "f16", 32), (60, "f32", 1)])
def test_attn_large_block(d, dtype, q_len):
    """One block of more than 2^28 positions, whose records' offsets in it pass 2^32.
    All but the last 64 have zero norms: logit 0, value 0, so they add their number
    to the sum of exponentials of those 64 alone.  Half a step of fp16 in both
    outputs, 2^-11 of the norm each (fp32: what a sum of 2^17 weights a lane and
    split takes, 2^-7 at most, of the zeros' share, which is below 2^-9)."""
    bs = (1 << 32) // 15 + 1000 if d == 60 else (1 << 28) + 1000
    rng = np.random.default_rng(d)
    pk, pv = (iq.isoq_params_init("fast", d, 2, 1, seed=s) for s in (1, 2))
    ndt = torch.float16 if dtype == "f16" else torch.float32
    q = torch.from_numpy(rng.standard_normal((q_len, 1, d))).to(ndt).cuda()
    start = torch.tensor([0, q_len], dtype=torch.int32, device="cuda")
    table = torch.zeros((1, 1), dtype=torch.int32, device="cuda")
    small, large = [], []
    for _ in (0, 1):
        rec = torch.from_numpy(rng.integers(0, 256, (1, 1, 64, pk.record_bytes), dtype=np.uint8)).cuda()
        rho = torch.from_numpy(rng.uniform(30, 60, (1, 1, 64)).astype(np.float32)).cuda()
        small += [rec, rho]
        idx, norm = torch.zeros((1, 1, bs, pk.record_bytes), dtype=torch.uint8, device="cuda"), torch.zeros((1, 1, bs), device="cuda")
        idx[:, :, -64:], norm[:, :, -64:] = rec, rho   # (one piece, or records stored whole: position after position)
        large += [idx, norm]
    assert large[0].numel() > 1 << 32

    def run(c, n):
        return iq.isoq_kv_attn(pk, q, c[0], c[1], pv, c[2], c[3], table, torch.tensor([n], dtype=torch.int32, device="cuda"),
                               scale=1.0, q_start=start, max_q_len=q_len)
    (o64, l64), (out, lse) = run(small, 64), run(large, bs)
    torch.cuda.synchronize()
    l64 = l64.double()
    want = torch.logaddexp(l64, torch.full_like(l64, np.log(bs - 64)))
    share = torch.exp(np.log(bs - 64) - want)
    assert share.max() < 2.0 ** -9, share.max()
    assert torch.all((lse.double() - want).abs() <= 2.0 ** -7 * share + 2.0 ** -16 + 2.0 ** -22 * want.abs())
    ref = o64.double() * torch.exp(l64 - want)[..., None]
    err = (out.double() - ref).norm(dim=-1)
    assert torch.all(err <= (2.0 ** -7 * share + (2.0 ** -10 if dtype == "f16" else 2.0 ** -15)) * ref.norm(dim=-1))


def test_pages_far_offsets():
    w = setup("full", 128, 3, "f16", [1, 1], 4, 4, 64, [500, 70], seed=1)
    n_blocks = (1 << 32) // (4 * 64 * 48) + 1000
    args, shift = far(w, n_blocks)
    planes = dict(k_idx=args["k_idx"], k_rho=args["k_rho"], v_idx=args["v_idx"], v_rho=args["v_rho"])
    src = int(args["block_table"][0, 0])
    pairs = torch.tensor([[src, 3], [3 + 1, src - 900], [src, src - 901]], dtype=torch.int32, device="cuda")
    planes["k_idx"][4] = 77
    iq.isoq_kv_copy_blocks(args["pk"], pairs, **planes)
    for x in planes.values():
        for a, b in pairs.tolist():
            assert torch.equal(x[a].view(torch.uint8), x[b].view(torch.uint8))
    keep = torch.arange(0, 500, 3, dtype=torch.int32, device="cuda")[None, None].contiguous()
    table = w["sides"][0][2].table
    was = {k: v[shift:].cpu().numpy() for k, v in planes.items()}
    iq.isoq_kv_compact(args["pk"], keep, torch.tensor([keep.shape[2]], dtype=torch.int32, device="cuda"),
                       args["block_table"][:1].contiguous(), **planes)
    i = np.arange(keep.shape[2])
    j = 3 * i
    for k, v in planes.items():
        old, new = was[k], v[shift:].cpu().numpy()
        if k.endswith("idx"):
            old, new = from_cache(old), from_cache(new)
        old[table[0, i // 64], :, i % 64] = old[table[0, j // 64], :, j % 64]
        np.testing.assert_array_equal(new, old)


def test_layout_round_trip():
    x = np.arange(2 * 3 * 48, dtype=np.uint8).reshape(2, 3, 48)
    assert np.array_equal(from_cache(to_cache(x)), x)
