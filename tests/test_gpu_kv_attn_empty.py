"""Rows that attend to nothing: out 0 and lse -inf, whatever the query holds and
however many splits, waves and tiles there are, and with pages that are there for
others.  Needs an MI355X."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

import paper_2603_28430_amd as iq  # noqa: E402
from test_gpu_kv_attn import check, device, reference, setup  # noqa: E402

KERNELS = [(128, 3, "f16", 1), (128, 4, "f16", 9), (64, 2, "f32", 5), (256, 3, "f16", 2), (128, 3, "f16", 40), (64, 4, "f16", 33),
           (70, 3, "f16", 2)]


@pytest.mark.parametrize("bad", [np.inf, np.nan])
@pytest.mark.parametrize("length", [100, 5000])
@pytest.mark.parametrize("d,bits,dtype,n", KERNELS)
def test_queries_that_are_no_numbers_without_positions(d, bits, dtype, n, length, bad):
    """Sequence 0 has no valid page, 1 no position, 2 only a page far behind; each
    with such queries and ordinary ones.  NaN only where there is something to attend to."""
    q_lens = [n, n, n]
    w = setup("full", d, bits, dtype, q_lens, 2, 2, 16, [length, 0, length], seed=d + n)
    ref = reference(w, 1.0)
    args = device(w)
    table = w["sides"][0][2].table.copy()
    table[0, :] = -1
    valid = np.ones((3, table.shape[1] * 16), bool)
    valid[0] = False
    keep = table.shape[1] - 3   # (in the tokens' own reach: n <= 40 of 48 positions from its first on)
    table[2, :keep] = -1
    valid[2, :keep * 16] = False
    args["block_table"] = torch.from_numpy(table).cuda()
    ref = reference(w, 1.0, valid=valid)
    w["q"][:, 1, 3] = bad
    args["q"] = torch.from_numpy(w["q"]).cuda()
    out, lse = iq.isoq_kv_attn(**args, scale=1.0)
    torch.cuda.synchronize()
    for t in range(3 * n):
        some = ref[t, 1][3] > 0
        assert some == (ref[t, 0][3] > 0)
        if some:
            assert torch.isnan(out[t, 1]).all() and torch.isnan(lse[t, 1]), t
            del ref[t, 1]
    assert any(np.isinf(l) for _, l, _, _ in ref.values()) and any(not np.isinf(l) for _, l, _, _ in ref.values())
    check(out, lse, ref)


@pytest.mark.parametrize("d", [128, 70])
def test_scales_at_the_end_of_floats(d):
    """A scale whose multiple in units of ln 2 is no float is refused; the largest others are not."""
    w = setup("full", d, 3, "f16", [1, 1], 2, 2, 16, [40, 3], seed=1)
    w["q"][:] = 0
    args = device(w)
    for bad in (2.4e38, -3.4e38):
        with pytest.raises(iq.IsoqError):
            iq.isoq_kv_attn(**args, scale=bad)
    for good in (2.3e38, -2.3e38):
        out, lse = iq.isoq_kv_attn(**args, scale=good)
        check(out, lse, reference(w, good))
