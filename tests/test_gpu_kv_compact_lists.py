"""isoq_kv_compact with lists that are not ascending positions: an entry takes what
its source held before the call if that lies at or behind its own place, and is
left out if not (negative ones among them), so the result is the same whatever
order workgroups and waves run in.  Needs an MI355X."""
import numpy as np
import pytest

from cache_layout import from_cache, to_cache

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

import paper_2603_28430_amd as iq  # noqa: E402
from test_gpu_kv_pages import Caches  # noqa: E402


def expected(host, table, keep, n_keep, bs):
    want = {}
    cap = table.shape[1] * bs
    for k, old in host.items():
        rows = from_cache(old) if k.endswith("idx") else old
        new = rows.copy()
        for s in range(keep.shape[0]):
            for h in range(old.shape[1]):
                j = keep[s, 0 if keep.shape[1] == 1 else h, :n_keep[s]].astype(np.int64)
                i = np.arange(len(j))
                on = (j >= i) & (j < cap) & (i < cap)
                i, j = i[on], j[on]
                new[table[s, i // bs], h, i % bs] = rows[table[s, j // bs], h, j % bs]
        want[k] = to_cache(new) if k.endswith("idx") else new
    return want


@pytest.mark.parametrize("variant,d,bits,heads", [("full", 128, 3, 3), ("2d", 80, 3, 2), ("full", 160, 3, 70), ("fast", 64, 4, 2)])
@pytest.mark.parametrize("kind", ["shifted", "far back", "random", "equal"])
def test_lists_that_do_not_ascend_from_zero(variant, d, bits, heads, kind):
    rng = np.random.default_rng(d)
    length, bs = 9300, 16
    per = -(-length // bs)
    c = Caches(variant, d, bits, per + 1, heads, bs, seed=d)
    table = rng.permutation(per + 1)[:per].reshape(1, per).astype(np.int32)
    i = np.arange(9200)
    keep = {"shifted": i - 1, "far back": i - 5000, "random": rng.integers(-200, length + 200, 9200),
            "equal": np.full(9200, 9000)}[kind]
    keep = keep.astype(np.int32)[None, None]
    n_keep = np.array([9200], np.int32)
    iq.isoq_kv_compact(c.p, torch.from_numpy(keep).cuda(), torch.from_numpy(n_keep).cuda(), torch.from_numpy(table).cuda(),
                       **c.kw)
    c.check(expected(c.host, table, keep, n_keep, bs))
