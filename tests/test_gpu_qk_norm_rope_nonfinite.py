"""Infinities in rows of isoq_qk_norm_rope that are normed: by the definition, x / sqrt(mean x^2 +
eps), such a row is 0 where it is finite and NaN at the infinity and in the pair that it is
rotated with, at whatever coordinate it stands; a NaN reaches the whole row, no other.
Rows of an odd number of chunks, rotated and passed on, among them.  Needs an MI355X."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

import paper_2603_28430_amd as iq  # noqa: E402

CASES = [(128, 128, "halves"), (128, 64, "pairs"), (64, 24, "pairs"), (72, 72, "pairs"), (24, 16, "halves"), (20, 20, "pairs"),
         (20, 4, "pairs"), (12, 8, "halves"), (6, 2, "pairs"), (90, 44, "halves"), (7, 6, "halves"), (7, 4, "pairs"), (9, 0, "halves")]


@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
@pytest.mark.parametrize("d,rot,layout", CASES)
def test_one_infinity(d, rot, layout, dtype):
    gen = torch.Generator(device="cuda").manual_seed(d + rot)
    q = torch.randn(d, 3, d, device="cuda", generator=gen).to(dtype)
    pos = torch.arange(d, dtype=torch.int32, device="cuda") * 1001
    w = torch.randn(d, device="cuda", generator=gen)
    rope = iq.isoq_rope_init(d, rot, layout)
    clean = iq.isoq_qk_norm_rope(rope, q, q, pos, w, w)
    half, at = rot // 2, torch.arange(d, device="cuda")
    pair = at ^ 1 if layout == "pairs" else torch.where(at < half, at + half, at - half)
    for value in (float("inf"), -float("inf"), float("nan")):
        x = q.clone()
        x[at, 1, at] = value         # token t has it at coordinate t
        for got, ref in zip(iq.isoq_qk_norm_rope(rope, x, x, pos, w, w), clean):
            assert torch.equal(got[:, ::2], ref[:, ::2])
            row = got[:, 1]
            if value != value:
                assert row.isnan().all()
                continue
            odd = torch.eye(d, dtype=torch.bool, device="cuda")
            turned = at[at < rot]
            odd[turned, pair[turned]] = True
            assert torch.equal(row.isnan(), odd), (value, (row.isnan() != odd).nonzero()[:4].tolist())
            assert (row[~odd] == 0).all()
