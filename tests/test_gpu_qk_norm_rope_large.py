"""Calls of isoq_qk_norm_rope with more rows or tokens than one launch takes: tokens on both
sides of each launch's end, the first and the last are what calls of their own give, bit
for bit (a row's result does not depend on the others).  Needs an MI355X."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

import paper_2603_28430_amd as iq  # noqa: E402

WAVES = 2 ** 26 - 4   # of one launch


@pytest.mark.parametrize("d,rot,layout,n_tokens,hq,hk,a_token", [
    (3, 2, "pairs", 2 ** 20 + 41, 33, 32, 65),          # a wave a row
    (2, 2, "halves", 2 ** 26 + 1003, 1, 0, 1),          # a wave a token
])
def test_more_than_a_launch(d, rot, layout, n_tokens, hq, hk, a_token):
    gen = torch.Generator(device="cuda").manual_seed(d)
    wide = torch.randn(n_tokens, (hq + hk) * d, dtype=torch.float16, device="cuda", generator=gen)
    body = wide.unflatten(1, (hq + hk, d))
    q, k = body[:, :hq], body[:, hq:] if hk else None
    pos = torch.randint(-2 ** 31, 2 ** 31, (n_tokens,), dtype=torch.int32, device="cuda", generator=gen)
    w = torch.tensor([0.5, -1.5, 2.0], device="cuda")[:d].contiguous()
    rope = iq.isoq_rope_init(d, rot, layout)
    got = iq.isoq_qk_norm_rope(rope, q, k, pos, w, None if k is None else w)
    most = WAVES // a_token // 16 * 16
    assert most < n_tokens < 2 * most
    for lo, hi in ((0, 40), (most - 40, most + 40), (n_tokens - 40, n_tokens)):
        ref = iq.isoq_qk_norm_rope(rope, q[lo:hi], None if k is None else k[lo:hi], pos[lo:hi], w, None if k is None else w)
        for a, b in zip(got, ref):
            assert b is None if a is None else torch.equal(a[lo:hi], b) and b.abs().max() > 0.1
    # every token, in pieces that one launch takes
    for lo in range(0, n_tokens, most // 2 - 5):
        hi = min(n_tokens, lo + most // 2 - 5)
        ref = iq.isoq_qk_norm_rope(rope, q[lo:hi], None if k is None else k[lo:hi], pos[lo:hi], w, None if k is None else w)
        for a, b in zip(got, ref):
            assert b is None if a is None else torch.equal(a[lo:hi], b)
