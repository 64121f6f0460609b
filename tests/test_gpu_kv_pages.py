"""Copies of cache blocks (isoq_kv_copy_blocks) and compaction of sequences
(isoq_kv_compact) against the same moves in numpy, byte for byte, over whole
caches (what is not named stays).  Needs an MI355X."""
import numpy as np
import pytest

import oracle
from cache_layout import from_cache, to_cache

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

import paper_2603_28430_amd as iq  # noqa: E402
from paper_2603_28430_amd import isoquant as binding  # noqa: E402


class Caches:
    """K (and V, and a sketch's) arrays of random bytes, on the host and on the GPU."""

    def __init__(self, variant, d, bits, n_blocks, heads, bs, values=True, m=0, seed=0):
        rng = np.random.default_rng(seed)
        self.p = iq.isoq_params_init(variant, d, bits, 1)
        self.sk = iq.isoq_sketch_init(self.p, m) if m else None
        R = self.p.record_bytes
        byte = lambda w: rng.integers(0, 256, (n_blocks, heads, bs, w), dtype=np.uint8)  # noqa: E731
        real = lambda: rng.standard_normal((n_blocks, heads, bs)).astype(np.float32)  # noqa: E731
        self.host = dict(k_idx=byte(R), k_rho=real())
        if values:
            self.host.update(v_idx=byte(R), v_rho=real())
        if m:
            self.host.update(k_signs=byte(m // 8), k_gamma=real())
        self.dev = {k: torch.from_numpy(v.copy()).cuda() for k, v in self.host.items()}
        self.kw = dict(self.dev, sketch=self.sk)

    def check(self, want):
        torch.cuda.synchronize()
        for k, v in self.dev.items():
            np.testing.assert_array_equal(v.cpu().numpy(), want[k], err_msg=k)


SHAPES = [("full", 128, 3, 8, 16, True, 0), ("full", 128, 4, 2, 16, True, 128), ("fast", 96, 3, 3, 16, True, 64),
          ("2d", 80, 3, 3, 7, True, 64), ("full", 100, 3, 1, 5, True, 0), ("2d", 7, 3, 5, 3, False, 0),
          ("2d", 1, 2, 1, 1, True, 0), ("full", 512, 4, 2, 64, True, 64), ("fast", 1000, 3, 3, 2, True, 0),
          ("8d", 1024, 4, 2, 16, False, 0), ("full", 64, 2, 32, 32, True, 0)]


@pytest.mark.parametrize("variant,d,bits,heads,bs,values,m", SHAPES)
def test_copy_blocks(variant, d, bits, heads, bs, values, m):
    c = Caches(variant, d, bits, 41, heads, bs, values, m, seed=d)
    rng = np.random.default_rng(d + bits)
    perm = rng.permutation(41)
    pairs = np.stack([perm[:14], perm[14:28]], 1).astype(np.int32)
    pairs[:3] = pairs[0, 0], pairs[1, 1]          # one source for several destinations
    pairs[0, 1], pairs[1, 1], pairs[2, 1] = perm[14], perm[15], perm[16]
    bad = np.array([[-1, perm[30]], [perm[31], 41], [perm[32], perm[32]], [2 ** 31 - 1, 0], [0, -2 ** 31]], np.int32)
    want = {k: v.copy() for k, v in c.host.items()}
    for v in want.values():
        v[pairs[:, 1]] = v[pairs[:, 0]]
    pairs = np.concatenate([pairs[:5], bad, pairs[5:]])
    iq.isoq_kv_copy_blocks(c.p, torch.from_numpy(pairs).cuda(), **c.kw)
    c.check(want)


@pytest.mark.parametrize("variant,d,bits,heads,bs,n", [("2d", 80, 3, 1, 3, 3000), ("2d", 7, 3, 1, 1, 5000), ("full", 128, 3, 1, 16, 2500),
                                                       ("2d", 1, 2, 1, 2, 9000), ("fast", 100, 3, 3, 13, 700)])
def test_copy_many_small_blocks(variant, d, bits, heads, bs, n):
    """Blocks of less than a workgroup's accesses, that end anywhere in them, and of less than 16 bytes."""
    c = Caches(variant, d, bits, 2 * n + 5, heads, bs, True, 64 if d == 80 else 0, seed=d)
    perm = np.random.default_rng(d).permutation(2 * n + 5)
    pairs = np.stack([perm[:n], perm[n:2 * n]], 1).astype(np.int32)
    pairs[5::97] = [-1, 3]
    want = {k: v.copy() for k, v in c.host.items()}
    good = pairs[pairs[:, 0] >= 0]
    for v in want.values():
        v[good[:, 1]] = v[good[:, 0]]
    iq.isoq_kv_copy_blocks(c.p, torch.from_numpy(pairs).cuda(), **c.kw)
    c.check(want)


def test_copy_blocks_none():
    c = Caches("full", 128, 3, 4, 2, 16)
    iq.isoq_kv_copy_blocks(c.p, torch.zeros((0, 2), dtype=torch.int32, device="cuda"), **c.kw)
    c.check(c.host)


def lists(rng, n_seqs, keep_heads, lens, max_keep, n_keep):
    keep = np.full((n_seqs, keep_heads, max_keep), -5, np.int32)   # (entries past n_keep are not looked at)
    for s in range(n_seqs):
        for h in range(keep_heads):
            keep[s, h, :n_keep[s]] = np.sort(rng.permutation(lens[s])[:n_keep[s]])
    return keep


def compacted(host, table, keep, n_keep, bs, n_blocks):
    """The definition: each list's entries in turn, from the contents before the call."""
    want = {k: v.copy() for k, v in host.items()}
    cap = table.shape[1] * bs

    def page(s, pos):
        if not 0 <= pos < cap or not 0 <= table[s, pos // bs] < n_blocks:
            return None
        return table[s, pos // bs], pos % bs
    for k, old in host.items():
        rows = from_cache(old) if k.endswith("idx") else old
        new = rows.copy()
        for s in range(keep.shape[0]):
            for h in range(old.shape[1]):
                ls = keep[s, 0 if keep.shape[1] == 1 else h]
                for i in range(min(max(n_keep[s], 0), keep.shape[2])):
                    a, b = page(s, int(ls[i])), page(s, i)
                    if a and b:
                        new[b[0], h, b[1]] = rows[a[0], h, a[1]]
        want[k] = to_cache(new) if k.endswith("idx") else new
    return want


def run_compact(c, table, keep, n_keep, bs):
    want = compacted(c.host, table, keep, n_keep, bs, c.host["k_rho"].shape[0])
    iq.isoq_kv_compact(c.p, torch.from_numpy(keep).cuda(), torch.from_numpy(n_keep).cuda(),
                       torch.from_numpy(table).cuda(), **c.kw)
    c.check(want)


@pytest.mark.parametrize("variant,d,bits,heads,bs,values,m", SHAPES)
@pytest.mark.parametrize("per_head", [False, True])
def test_compact(variant, d, bits, heads, bs, values, m, per_head):
    rng = np.random.default_rng(d + bits)
    lens = [300, 1, 77, 40]
    per = -(-300 // bs)
    n_blocks = 4 * per + 2
    c = Caches(variant, d, bits, n_blocks, heads, bs, values, m, seed=d)
    table = rng.permutation(n_blocks)[:4 * per].reshape(4, per).astype(np.int32)
    n_keep = np.array([133, 1, 77, 0], np.int32)   # (all of one sequence, none of another)
    run_compact(c, table, lists(rng, 4, heads if per_head else 1, lens, 150, n_keep), n_keep, bs)


@pytest.mark.parametrize("variant,d,bits,m", [("2d", 80, 3, 64), ("full", 100, 3, 0), ("full", 160, 3, 128), ("2d", 98, 4, 0),
                                              ("fast", 1000, 3, 0), ("2d", 7, 3, 0), ("2d", 1, 2, 0), ("fast", 80, 2, 64),
                                              ("full", 96, 3, 128), ("2d", 250, 2, 0), ("full", 172, 3, 0)])
def test_compact_many_heads(variant, d, bits, m):
    """Sequences and heads that fill the card: records stored whole (1 to 375
    bytes, with every remainder of 64 and 16 bytes) move as few chains."""
    rng = np.random.default_rng(d + bits)
    lens, heads, bs = [130, 40, 7], 22, 7
    per = -(-130 // bs)
    c = Caches(variant, d, bits, 3 * per + 1, heads, bs, True, m, seed=d)
    table = rng.permutation(3 * per + 1)[:3 * per].reshape(3, per).astype(np.int32)
    n_keep = np.array([61, 40, 3], np.int32)
    run_compact(c, table, lists(rng, 3, heads, lens, 70, n_keep), n_keep, bs)


def test_compact_long_whole_records():
    """More than one tile of a workgroup's positions, 2 and 4 a lane, in place."""
    rng = np.random.default_rng(1)
    for d, bits in ((80, 3), (160, 3), (100, 2)):
        per, heads = 626, 70
        c = Caches("full", d, bits, per, heads, 16, seed=d)
        table = rng.permutation(per).reshape(1, per).astype(np.int32)
        n_keep = np.array([9003], np.int32)
        run_compact(c, table, lists(rng, 1, heads, [10000], 9003, n_keep), n_keep, 16)


@pytest.mark.parametrize("length,count", [(9001, 8999), (9001, 4097), (20000, 8192), (4097, 4096), (13000, 12999)])
def test_compact_long(length, count):
    """Lists around and past a workgroup's 4,096 positions, nearly everything kept among them."""
    rng = np.random.default_rng(count)
    bs, heads = 16, 3
    per = -(-length // bs)
    c = Caches("full", 64, 3, per + 1, heads, bs, seed=1)
    table = rng.permutation(per + 1)[:per].reshape(1, per).astype(np.int32)
    n_keep = np.array([count], np.int32)
    run_compact(c, table, lists(rng, 1, heads, [length], count, n_keep), n_keep, bs)
    # dropping the first position moves every other one by one
    c = Caches("full", 64, 3, per + 1, heads, bs, seed=2)
    keep = np.arange(1, count + 1, dtype=np.int32)[None, None]
    run_compact(c, table, keep, n_keep, bs)


def test_compact_missing_pages_and_counts():
    """Entries without a page or outside the table are skipped; n_keep is cut to [0, max_keep]."""
    rng = np.random.default_rng(5)
    c = Caches("full", 128, 3, 30, 2, 16, m=64)
    table = np.stack([rng.permutation(30)[:10] for _ in range(1)] + [np.full(10, -1)] + [np.full(10, 99)]).astype(np.int32)
    table[0, [2, 7]] = [-1, 30]
    keep = lists(rng, 3, 1, [160, 160, 160], 60, [60, 60, 60])
    keep[0, 0, 58:] = [160, 2 ** 31 - 1]   # past the table
    for n_keep in ([60, 60, 60], [-3, 1, 1], [2 ** 31 - 1, 5, 5]):
        run_compact(c, table, keep, np.array(n_keep, np.int32), 16)
        c = Caches("full", 128, 3, 30, 2, 16, m=64)


def test_compact_unordered_lists_stay_inside():
    """A list that does not ascend leaves positions below its n_keep unspecified, and the rest as it was."""
    rng = np.random.default_rng(7)
    c = Caches("full", 128, 3, 24, 2, 16)
    table = rng.permutation(24)[:20].reshape(2, 10).astype(np.int32)
    keep = rng.integers(-100, 300, (2, 2, 70)).astype(np.int32)
    iq.isoq_kv_compact(c.p, torch.from_numpy(keep).cuda(), torch.tensor([50, 70], dtype=torch.int32, device="cuda"),
                       torch.from_numpy(table).cuda(), **c.kw)
    torch.cuda.synchronize()
    for name, v in c.dev.items():
        a, b = v.cpu().numpy(), c.host[name]
        if name.endswith("idx"):
            a, b = from_cache(a), from_cache(b)
        touched = np.zeros(b.shape[:3], bool)
        for s, n in ((0, 50), (1, 70)):
            i = np.arange(n)
            touched[table[s, i // 16], :, i % 16] = True
        np.testing.assert_array_equal(a[~touched], b[~touched])


def test_pages_refusals():
    lib, p = binding.lib, iq.isoq_params_init("full", 128, 3, 1)
    sk = iq.isoq_sketch_init(p, 64)
    other = iq.isoq_sketch_init(iq.isoq_params_init("fast", 128, 3, 1), 64)
    buf = torch.zeros(1 << 16, dtype=torch.uint8, device="cuda")
    b = buf.data_ptr()
    planes = dict(k_idx=b, k_rho=b, v_idx=b, v_rho=b, k_signs=None, k_gamma=None, n_blocks=1, bs=16, stream=None)
    copy = dict(pk=p.handle, sk=None, pairs=b, n_pairs=1, heads=2, **planes)
    comp = dict(pk=p.handle, sk=None, keep=b, keep_heads=1, max_keep=4, n_keep=b, n_seqs=1, table=b, max_blocks=1, heads=2,
                **planes)
    shared = [(3, dict(pk=None)), (3, dict(k_idx=None)), (3, dict(k_rho=None)), (3, dict(v_idx=None)),
              (3, dict(v_rho=None)), (3, dict(k_signs=b)), (3, dict(k_gamma=b)), (3, dict(sk=sk.handle)),
              (3, dict(sk=sk.handle, k_signs=b)), (1, dict(sk=other.handle, k_signs=b, k_gamma=b)),
              (1, dict(heads=0)), (1, dict(bs=0)), (1, dict(n_blocks=-1)), (2, dict(n_blocks=1 << 30)),
              (4, dict(k_idx=b + 4)), (4, dict(v_idx=b + 8)), (4, dict(k_rho=b + 2)), (4, dict(v_rho=b + 1)),
              (4, dict(sk=sk.handle, k_signs=b + 2, k_gamma=b)), (4, dict(sk=sk.handle, k_signs=b, k_gamma=b + 2))]
    for st, kw in shared + [(1, dict(n_pairs=-1)), (2, dict(n_pairs=1 << 24)), (3, dict(pairs=None)), (4, dict(pairs=b + 2))]:
        assert lib.isoq_kv_copy_blocks(*dict(copy, **kw).values()) == st, kw
    for st, kw in shared + [(1, dict(n_seqs=-1)), (1, dict(max_keep=-1)), (1, dict(keep_heads=3)), (1, dict(max_blocks=-1)),
                            (2, dict(n_seqs=65536)), (2, dict(max_blocks=1 << 28)), (2, dict(max_keep=2 ** 31 - 1)),
                            (2, dict(heads=1 << 22, keep_heads=1)),
                            (3, dict(keep=None)), (3, dict(n_keep=None)), (3, dict(table=None)), (4, dict(keep=b + 2)),
                            (4, dict(n_keep=b + 2)), (4, dict(table=b + 2))]:
        assert lib.isoq_kv_compact(*dict(comp, **kw).values()) == st, kw
    assert lib.isoq_kv_copy_blocks(*dict(copy, n_pairs=0).values()) == 0
    assert lib.isoq_kv_compact(*dict(comp, n_seqs=0).values()) == 0


def test_pages_graph_and_streams():
    """Captured and replayed: each replay compacts and copies what it finds."""
    c = Caches("full", 128, 3, 60, 4, 16, seed=3)
    rng = np.random.default_rng(3)
    table = rng.permutation(60)[:50].reshape(1, 50).astype(np.int32)
    free = [b for b in range(60) if b not in table][:1]
    pairs = np.array([[table[0, 0], free[0]]], np.int32)
    keep = np.sort(rng.permutation(800)[:500]).astype(np.int32)[None, None]
    n_keep = np.array([500], np.int32)
    g = [torch.from_numpy(x).cuda() for x in (pairs, keep, n_keep, table)]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    want = c.host
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        iq.isoq_kv_copy_blocks(c.p, g[0], **c.kw)
        iq.isoq_kv_compact(c.p, *g[1:], **c.kw)
    for i in range(4):
        if i % 2:
            graph.replay()
        else:
            iq.isoq_kv_copy_blocks(c.p, g[0], **c.kw, stream=s)
            iq.isoq_kv_compact(c.p, *g[1:], **c.kw, stream=s)
            s.synchronize()
        want = {k: v.copy() for k, v in want.items()}
        for v in want.values():
            v[pairs[:, 1]] = v[pairs[:, 0]]
        want = compacted(want, table, keep, n_keep, 16, 60)
        c.check(want)
