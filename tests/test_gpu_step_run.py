"""Steps of a decoder as they are used together: isoq_kv_plan, isoq_qk_norm_rope on
a packed projection, isoq_kv_append, isoq_kv_attn_prefix behind two shared prefixes
and isoq_kv_attn_cross to encoder positions, over steps in which sequences start,
grow, are cut, end and are refused for want of blocks; called eagerly and as one
captured graph that is replayed with each step's lengths and rows.

The reference keeps every sequence's keys and values as Python lists of what was
appended (rows by themselves through isoq_qk_norm_rope, isoq_quantize and
isoq_dequantize, each tested against 64 bits elsewhere) and attends to them in 64 bits.

Tolerance: that of test_gpu_kv_attn.py's docstring, with vn the weighted norms of the
values; the fp32 rows of isoq_dequantize add an error as the kernel's own rotation has
it, (width + 8) 2^-23, to the scores (ds is taken twice) and to the values.
Needs an MI355X."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

import paper_2603_28430_amd as iq  # noqa: E402
from test_gpu_kv_plan import walk  # noqa: E402

CANARY = 77.0
PREFIX_LENS, PREFIX_START = [75, 33], [0, 4, 6]     # sequence 6 has none
ENC_LENS = [90, 0, 41, 64, 1, 130, 17]
STEPS = [  # every sequence's length after the step, without its prefix
    [20, 1, 0, 17, 5, 0, 33],
    [21, 2, 30, 18, 6, 0, 34],
    [22, 3, 31, 9, 7, 18, 35],
    [23, 0, 32, 10, 8, 19, 0],
    [24, 16, 33, 11, 0, 20, 140],    # (its last sequence's blocks are not there)
    [0, 17, 34, 12, 3, 21, 40],
    [1, 18, 64, 13, 4, 0, 41],
]
MAX_LEN, SPARE = 160, 16


class World:
    def __init__(self, d, bits, dtype, bs, n_kv, group, variant):
        rng = self.rng = np.random.default_rng(d + bits)
        self.d, self.dtype, self.bs, self.n_kv, self.n_q = d, dtype, bs, n_kv, n_kv * group
        self.scale, self.n = d ** -0.5, len(STEPS[0])
        self.pk, self.pv = (iq.isoq_params_init(variant, d, bits, seed=s) for s in (1, 2))
        self.level, self.pw = float(iq.isoq_codebook_lloyd(bits, d).max()), {"full": 4, "fast": 4, "2d": 2, "8d": 8}[variant]
        self.rope = iq.isoq_rope_init(d, d // 2 // 2 * 2, "halves")
        self.weights = [torch.from_numpy(1 + 0.2 * rng.standard_normal(d)).float().cuda() for _ in range(2)]
        rec = iq.isoq_record_bytes(variant, d, bits)
        pre, enc = (sum(-(-x // bs) for x in lens) for lens in (PREFIX_LENS, ENC_LENS))
        spare = SPARE * 16 // bs
        planes = lambda blocks: (torch.full((blocks, n_kv, bs, rec), 0xA5, dtype=torch.uint8, device="cuda"),   # noqa: E731
                                 torch.full((blocks, n_kv, bs), float("nan"), device="cuda"))
        self.k, self.v = planes(pre + spare), planes(pre + spare)
        self.ek, self.ev = planes(enc), planes(enc)
        ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")   # noqa: E731
        self.prefix_table, self.prefixes = self.fill(PREFIX_LENS, pre, self.k, self.v)
        self.enc_table, self.encoders = self.fill(ENC_LENS, enc, self.ek, self.ev)
        self.prefix_lens, self.enc_lens, self.prefix_start = ints(PREFIX_LENS), ints(ENC_LENS), ints(PREFIX_START)
        self.offset = [PREFIX_LENS[0]] * 4 + [PREFIX_LENS[1]] * 2 + [0]
        self.offsets = ints(self.offset)
        # the state of the sequences, on the device and as the test has it
        self.lens, self.n_free = ints([0] * self.n), ints([spare])
        self.table = torch.full((self.n, -(-MAX_LEN // bs)), -3, dtype=torch.int32, device="cuda")
        self.free = ints(list(pre + rng.permutation(spare)))
        self.kept = [[] for _ in range(self.n)]
        # a step's inputs and outputs, of fixed sizes
        most = lambda a, b: [max(0, y - x) for x, y in zip(a, b)]   # noqa: E731
        news = [most(a, b) for a, b in zip([[0] * self.n] + STEPS, STEPS)]
        self.max_q = max(max(x) for x in news)
        self.n_tokens = max(sum(x) for x in news) + 40
        self.new = ints([0] * self.n)
        self.proj = torch.zeros(self.n_tokens, (self.n_q + 2 * n_kv) * d, dtype=dtype, device="cuda")
        self.out, self.cross = (torch.zeros(self.n_tokens, self.n_q, d, dtype=dtype, device="cuda") for _ in range(2))
        self.step_no = torch.arange(self.n_tokens, device="cuda")

    def rows(self, n, heads):
        return torch.from_numpy(self.rng.standard_normal((n, heads, self.d))).cuda().to(self.dtype)

    def kv(self, k, v):
        """What a cache gives back for these rows: (kx, krho, vx, vrho), float64 [n, n_kv, ..]."""
        res = []
        for p, x in ((self.pk, k), (self.pv, v)):
            idx, rho = iq.isoq_quantize(p, x.reshape(-1, self.d))
            res.append(iq.isoq_dequantize(p, idx, rho, torch.float32).double().cpu().numpy().reshape(x.shape))
            res.append(rho.double().cpu().numpy().reshape(x.shape[:2]))
        return res

    def fill(self, lens, blocks, k, v):
        """Sequences of rows in the cache's first blocks, in an order of their own: (table, what they hold)."""
        perm = self.rng.permutation(blocks)
        table, slots, at = np.full((len(lens), max(-(-x // self.bs) for x in lens)), -9), [], 0
        for s, x in enumerate(lens):
            for j in range(-(-x // self.bs)):
                table[s, j] = perm[at]
                at += 1
            slots += [table[s, p // self.bs] * self.bs + p % self.bs for p in range(x)]
        kx, vx = self.rows(len(slots), self.n_kv), self.rows(len(slots), self.n_kv)
        iq.isoq_kv_append(self.pk, kx, torch.tensor(slots, device="cuda"), *k, self.pv, vx, *v)
        kv, start = self.kv(kx, vx), np.concatenate([[0], np.cumsum(lens)])
        held = [[tuple(a[i] for a in kv) for i in range(start[s], start[s + 1])] for s in range(len(lens))]
        return torch.tensor(table, dtype=torch.int32, device="cuda"), held

    def call(self):
        """One step, as a program that serves these sequences calls it."""
        n_q, n_kv, d = self.n_q, self.n_kv, self.d
        lens, q_start, slots, pos, _ = iq.isoq_kv_plan(self.lens, self.new, self.table, self.bs, self.free, self.n_free,
                                                       self.n_tokens, seq_lens=self.lens, n_free_out=self.n_free)
        seq = torch.searchsorted(q_start[1:].contiguous(), self.step_no, right=True).clamp(max=self.n - 1)
        pos = pos + self.offsets[seq]
        q, k, v = self.proj.view(self.n_tokens, n_q + 2 * n_kv, d).split([n_q, n_kv, n_kv], 1)
        q, k = iq.isoq_qk_norm_rope(self.rope, q, k, pos, *self.weights)
        iq.isoq_kv_append(self.pk, k, slots, *self.k, self.pv, v.contiguous(), *self.v)
        common = dict(scale=self.scale, q_start=q_start, max_q_len=self.max_q)
        iq.isoq_kv_attn_prefix(self.pk, q, *self.k, self.pv, *self.v, self.table, lens, self.prefix_table, self.prefix_lens,
                               self.prefix_start, **common, out=self.out)
        iq.isoq_kv_attn_cross(self.pk, self.out, *self.ek, self.pv, *self.ev, self.enc_table, self.enc_lens, **common,
                              out=self.cross)
        return q, q_start, slots

    def near(self, got, q, held):
        """One row of one query head against the definition; q and got float64, held: (kx, krho, vx, vrho)."""
        f16 = self.dtype == torch.float16
        if not len(held[1]):
            assert np.all(got == 0)
            return
        kx, krho, vx, vrho = held
        t = self.scale * (kx @ q)
        p = np.exp(t - t.max())
        p /= p.sum()
        o = p @ vx
        ds = (self.pw + 8) * 2.0 ** -23 * self.scale * np.linalg.norm(q) * np.linalg.norm(kx, axis=1).max() + 2.0 ** -22 * np.abs(t).max()
        vn = p @ np.linalg.norm(vx, axis=1)
        lv = (1 / 32639 if f16 else 2.0 ** -22) * self.level * np.sqrt(self.pw) * (p @ vrho)
        step, sub = (2.0 ** -11, 2.0 ** -25 * np.sqrt(self.d)) if f16 else (2.0 ** -22, 0.0)
        tol = (4 * ds + 2.0 ** -19 + 2.0 ** -20 + (self.pw + 8) * 2.0 ** -23) * vn + lv + step * np.linalg.norm(o) + sub
        off = np.linalg.norm(got - o)
        assert off <= tol, (off, tol)

    def step(self, new, call):
        """One step of the device's state, and the test's own of it."""
        old = [len(x) for x in self.kept]
        assert self.lens.tolist() == old
        table, free = self.table.cpu().numpy(), self.free.cpu().numpy()
        want = walk(old, new, table, self.bs, free, self.n_free.item(), self.n_tokens)
        self.new.copy_(torch.tensor(new, dtype=torch.int32))
        self.proj.copy_(self.rows(self.n_tokens, self.n_q + 2 * self.n_kv).flatten(1))
        self.out.fill_(CANARY)
        self.cross.fill_(CANARY)
        q, q_start, slots = call()
        torch.cuda.synchronize()
        assert self.lens.tolist() == list(want[0]) and q_start.tolist() == want[1] and self.n_free.tolist() == want[4]
        assert slots.tolist() == want[2]
        assert (self.table.cpu().numpy() == table).all() and (self.free.cpu().numpy() == free).all()
        # the rows by themselves, at positions that the test knows
        total = want[1][-1]
        body = self.proj.view(self.n_tokens, -1, self.d)[:total]
        seq = np.repeat(np.arange(self.n), np.diff(want[1]))
        pos = torch.tensor([p + self.offset[s] for p, s in zip(want[3], seq)], dtype=torch.int32, device="cuda")
        qx, kx = iq.isoq_qk_norm_rope(self.rope, body[:, :self.n_q].contiguous(),
                                      body[:, self.n_q:self.n_q + self.n_kv].contiguous(), pos, *self.weights)
        assert torch.equal(q[:total], qx)
        kv = self.kv(kx, body[:, self.n_q + self.n_kv:].contiguous())
        for s in range(self.n):
            del self.kept[s][want[0][s]:]
            if want[0][s] == max(new[s], 0):
                self.kept[s] += [tuple(a[i] for a in kv) for i in range(want[1][s], want[1][s + 1])]
            assert len(self.kept[s]) == want[0][s]
        qx, out, cross = qx.double().cpu().numpy(), self.out.double().cpu().numpy(), self.cross.double().cpu().numpy()
        for i in range(total):
            s = int(seq[i])
            n = max(0, want[0][s] - (want[1][s + 1] - 1 - i))
            shared = [] if s == 6 else self.prefixes[0 if s < 4 else 1]
            own, enc = (list(zip(*x)) or [[]] * 4 for x in (shared + self.kept[s][:n], self.encoders[s]))
            for h in range(self.n_q):
                kvh = h * self.n_kv // self.n_q
                for got, query, held in ((out, qx[i, h], own), (cross, out[i, h], enc)):
                    self.near(got[i, h], query, [np.array([x[kvh] for x in part]) for part in held])
        assert np.all(out[total:] == CANARY) and np.all(cross[total:] == CANARY)


CASES = [(128, 3, torch.float16, 16, 2, 4, "full"), (64, 4, torch.float32, 8, 1, 2, "fast"), (80, 2, torch.float16, 16, 2, 1, "2d")]


@pytest.mark.parametrize("d,bits,dtype,bs,n_kv,group,variant", CASES)
def test_steps(d, bits, dtype, bs, n_kv, group, variant):
    w = World(d, bits, dtype, bs, n_kv, group, variant)
    for new in STEPS:
        w.step(new, w.call)


@pytest.mark.parametrize("d,bits,dtype,bs,n_kv,group,variant", CASES[:2])
def test_steps_of_a_captured_graph(d, bits, dtype, bs, n_kv, group, variant):
    w = World(d, bits, dtype, bs, n_kv, group, variant)
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
