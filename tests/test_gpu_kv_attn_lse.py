"""lse of attention, an fp32 output, held to what fp32 arithmetic leaves, whatever
the codebook: the root mean square of its error over a call's rows is at most
2^-22 of the root mean square of the rows' largest logit (in size).  Derivation,
relative to sum |q c[idx]| of a logit's products: a coordinate is held to 2^-23 and
a level to 2^-23 (two fp16 parts, or three digits of the largest one, 2^-23 of it),
products of what both leave are 2^-24; sums in fp32 round d / 16 steps of a few
instructions, sqrt(3 d / 16) 2^-25 at independent signs, 2^-22.7 at d = 128.  In the
root mean square these add to 2^-22.2 of the root of the sum of squares, which is
what the logits' size is; the exponentials, their sum and its logarithm are off by
2^-23 absolute, next to nothing here (logits of 5 and more).
A level without what fp16 leaves of it (2^-12), or with that in e4m3 (2.6%, times a
query rounded as much), is 5 to 40 times that.  Needs an MI355X."""
import numpy as np
import pytest

import oracle

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

import paper_2603_28430_amd as iq  # noqa: E402
from test_gpu_kv_attn import device, reference, setup  # noqa: E402


def levels_of(bits, kind, d):
    k = 1 << (bits - 1)
    if kind == "lloyd":
        return oracle.codebook(bits, d)
    if kind == "uniform":
        pos = (np.arange(k) + 0.5) / k
    else:
        pos = np.sort(np.random.default_rng(10 * bits + len(kind)).uniform(0.1, 1.0, k))
    return np.float32(np.concatenate([-pos[::-1], pos]) / np.sqrt(d)).astype(np.float64)


@pytest.mark.parametrize("kind", ["lloyd", "uniform", "other", "another"])
@pytest.mark.parametrize("bits", [2, 3, 4])
@pytest.mark.parametrize("d,dtype,n,group", [(128, "f16", 40, 2), (96, "f16", 33, 2), (80, "f16", 33, 2), (64, "f16", 50, 1),
                                             (128, "f16", 3, 2), (64, "f32", 5, 3)])
def test_lse_is_held_to_fp32(d, dtype, n, group, bits, kind):
    w = setup("full", d, bits, dtype, [n, n], 2 * group, 2, 16, [700, 300], seed=d + bits, levels=levels_of(bits, kind, d))
    w["q"] *= 12.0   # logits of 5 and more
    lse = iq.isoq_kv_attn(**device(w), scale=1.0)[1].cpu().numpy().astype(np.float64)
    ref = reference(w, 1.0)
    err = np.array([lse[k] - l for k, (_, l, _, _) in ref.items()])
    size = np.array([l for _, l, _, _ in ref.values()])
    ratio = np.sqrt(np.mean(err ** 2) / np.mean(size ** 2))
    print(f"{d} {dtype} {bits} {kind}: {ratio:.2e} of {np.sqrt(np.mean(size ** 2)):.1f}", flush=True)
    assert np.mean(size) > 5
    assert ratio <= 2.0 ** -22
