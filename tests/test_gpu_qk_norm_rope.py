"""Norms and rotary positions of queries and keys (isoq_qk_norm_rope) against
the definition in 64 bits (angles in 80).

Tolerance, per element, with (a, b) the normed pair:
  norm      the sum of d squares over lanes, its square root and the quotient:
            (d / 64 + 16) 2^-24 relative; the products with it and the weight 2 2^-24;
  angle     cos and sin off by 6 2^-24 (argument 3 roundings of at most pi / 4, the
            polynomials, the phase's 2^-31 turns);
  rotation  two products, a sum and the amplitude: 4 2^-24;
together amplitude (|a| + |b|) (d / 64 + 28) 2^-24, and half a step of fp16, 2^-11
of the result or 2^-25.
Needs an MI355X."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

import paper_2603_28430_amd as iq  # noqa: E402

L = np.longdouble
TWO_PI = L("6.283185307179586476925286766559005768")


def definition(x, pos, freqs, half, halves, weight, eps, amplitude):
    """(rows, their tolerance) of x [tokens, heads, d] float64."""
    d = x.shape[-1]
    if weight is not None:
        x = weight * x / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    turns = np.mod(pos.astype(L)[:, None] * (freqs.astype(L) / TWO_PI), L(1))
    angle = (turns * TWO_PI).astype(np.float64)[:, None]
    y, size = x.copy(), np.abs(x)
    lo, hi = (slice(0, half), slice(half, 2 * half)) if halves else (slice(0, 2 * half, 2), slice(1, 2 * half, 2))
    a, b = x[..., lo], x[..., hi]
    y[..., lo] = amplitude * (a * np.cos(angle) - b * np.sin(angle))
    y[..., hi] = amplitude * (a * np.sin(angle) + b * np.cos(angle))
    size[..., lo] = size[..., hi] = abs(amplitude) * (np.abs(a) + np.abs(b))
    return y, size * (d / 64 + 28) * 2.0 ** -24


def check(got, dtype, x, pos, freqs, half, halves, weight, eps, amplitude):
    ref, tol = definition(x, pos, freqs, half, halves, weight, eps, amplitude)
    off = np.abs(got.double().cpu().numpy() - ref)
    if dtype == torch.float16:
        tol = tol + np.maximum(2.0 ** -11 * np.abs(ref), 2.0 ** -25)
    bad = off > tol
    assert not bad.any(), (np.argwhere(bad)[:3], off[bad][:3], tol[bad][:3])


def positions(rng, n, far=2 ** 31):
    pos = rng.integers(-far, far, n)
    edge = [0, 1, 2 ** 31 - 1, -2 ** 31, -1, 2 ** 24 + 1, 131071]
    pos[:min(n, len(edge))] = edge[:n]
    return pos.astype(np.int32)


def rows(rng, shape, dtype):
    x = rng.standard_normal(shape) * np.exp(rng.standard_normal(shape[:-1] + (1,)))
    return torch.from_numpy(x).cuda().to(dtype)


CASES = [  # d, rot, layout
    (128, 128, "halves"), (128, 128, "pairs"), (128, 64, "halves"), (128, 32, "pairs"), (64, 64, "halves"),
    (64, 16, "pairs"), (80, 80, "halves"), (80, 32, "pairs"), (96, 48, "halves"), (160, 160, "pairs"), (192, 64, "halves"),
    (256, 256, "halves"), (512, 512, "pairs"), (1024, 1024, "halves"), (1024, 16, "pairs"), (90, 44, "halves"),
    (90, 90, "pairs"), (7, 4, "halves"), (7, 6, "pairs"), (2, 2, "pairs"), (1, 0, "halves"), (33, 0, "pairs"), (1000, 500, "halves"),
    (65, 2, "halves"), (48, 24, "pairs"), (112, 8, "halves"), (16, 16, "halves"), (32, 32, "pairs")]


@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
@pytest.mark.parametrize("d,rot,layout", CASES)
def test_rows(d, rot, layout, dtype):
    rng = np.random.default_rng(d * 3 + rot)
    for n, hq, hk, norm, amplitude in ((9, 5, 2, True, 1.0), (1, 1, 1, False, 1.3), (37, 8, 8, True, 0.7), (3, 33, 3, False, 1.0)):
        freqs = iq.isoq_rope_freqs(rot, 10000.0, factor=4.0, original=2048) if rot else np.zeros(0)
        rope = iq.isoq_rope_init(d, rot, layout, freqs=freqs, amplitude=amplitude)
        q, k, pos = rows(rng, (n, hq, d), dtype), rows(rng, (n, hk, d), dtype), positions(rng, n)
        w = [1 + 0.3 * rng.standard_normal(d).astype(np.float32) for _ in range(2)] if norm else [None, None]
        dev = [None if x is None else torch.from_numpy(x.astype(np.float32)).cuda() for x in w]
        got = iq.isoq_qk_norm_rope(rope, q, k, torch.from_numpy(pos).cuda(), *dev, eps=1e-5)
        for g, x, wt in zip(got, (q, k), w):
            assert g.is_contiguous() and g.shape == x.shape and g.dtype == dtype
            wt = None if wt is None else wt.astype(np.float32).astype(np.float64)
            check(g, dtype, x.double().cpu().numpy(), pos, freqs, rot // 2, layout == "halves", wt, np.float64(np.float32(1e-5)),
                  float(np.float32(amplitude)))
            if not norm:   # what is not rotated is passed on bit for bit
                assert torch.equal(g[..., rot:], x[..., rot:])


@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
@pytest.mark.parametrize("d,hq,hk,extra", [(128, 32, 8, 0), (64, 4, 2, 3), (96, 5, 1, 8), (90, 3, 3, 0), (128, 3, 1, 1)])
def test_parts_of_a_projection(d, hq, hk, extra, dtype):
    """Views whose tokens lie further apart, at any element's alignment, equal contiguous rows bit for bit; so do rows in place."""
    rng = np.random.default_rng(d + hq)
    n = 21
    wide = rows(rng, (n, (hq + 2 * hk) * d + extra), dtype)
    for shift in (0, 1, 8):
        if shift > extra:
            continue
        body = wide[:, shift:shift + (hq + 2 * hk) * d].unflatten(1, (hq + 2 * hk, d))
        q, k = body[:, :hq], body[:, hq:hq + hk]
        pos = torch.from_numpy(positions(rng, n)).cuda()
        w = torch.from_numpy(1 + 0.3 * rng.standard_normal(d)).float().cuda()
        rope = iq.isoq_rope_init(d, d // 4 * 2, "halves")
        before = wide.clone()
        got = iq.isoq_qk_norm_rope(rope, q, k, pos, w, None)
        assert torch.equal(wide, before)
        ref = iq.isoq_qk_norm_rope(rope, q.contiguous(), k.contiguous(), pos, w, None)
        qi, ki = q.contiguous(), k.contiguous()
        same = iq.isoq_qk_norm_rope(rope, qi, ki, pos, w, None, q_out=qi, k_out=ki)
        assert same[0] is qi and same[1] is ki
        check(ref[0], dtype, q.double().cpu().numpy(), pos.cpu().numpy(), iq.isoq_rope_freqs(d // 4 * 2), d // 4, True,
              w.double().cpu().numpy(), np.float64(np.float32(1e-6)), 1.0)
        # (another alignment may take another kernel, which sums squares in another order)
        for a, b, c in zip(got, ref, same):
            assert torch.equal(b, c)
            assert (a.double() - b.double()).abs().max() <= (2.0 ** -10 if dtype == torch.float16 else 2.0 ** -20) * b.double().abs().max()
        alone, none = iq.isoq_qk_norm_rope(rope, q, None, pos, w)
        assert none is None and torch.equal(alone, got[0])


@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
@pytest.mark.parametrize("d", [128, 90])
def test_rows_stand_alone(d, dtype):
    """Infinities, NaN and zeros stay in their rows; a row's result does not depend on the others."""
    rng = np.random.default_rng(4)
    n, h = 12, 6
    q, pos = rows(rng, (n, h, d), dtype), torch.from_numpy(positions(rng, n)).cuda()
    w = torch.ones(d, device="cuda")
    rope = iq.isoq_rope_init(d, d // 2 // 2 * 2, "pairs")
    clean = iq.isoq_qk_norm_rope(rope, q, None, pos, w)[0]
    bad = q.clone()
    bad[3, 2, 5], bad[7, 0, d - 1], bad[9, 5] = float("inf"), float("nan"), 0.0
    got = iq.isoq_qk_norm_rope(rope, bad, None, pos, w)[0]
    keep = torch.ones((n, h), dtype=torch.bool, device="cuda")
    keep[3, 2] = keep[7, 0] = keep[9, 5] = False
    assert torch.equal(got[keep], clean[keep])
    assert got[7, 0].isnan().all() and got[3, 2].isnan().any() and (got[9, 5] == 0).all()
    for t in (0, 5, n - 1):
        one = iq.isoq_qk_norm_rope(rope, q[t:t + 1], None, pos[t:t + 1], w)[0]
        assert torch.equal(one[0], clean[t])


def test_norm_of_small_and_large_rows():
    """The norm brings rows of any size to its weight; eps is what holds rows of next to nothing."""
    d = 128
    x = torch.tensor([1e-30, 1e-4, 1.0, 1e15], device="cuda")[:, None, None] * torch.ones(1, 1, d, device="cuda")
    rope = iq.isoq_rope_init(d, 0)
    got = iq.isoq_qk_norm_rope(rope, x, None, torch.zeros(4, dtype=torch.int32, device="cuda"), torch.ones(d, device="cuda"), eps=1e-6)[0]
    ref = (x.double() / (x.double() ** 2 + 1e-6).sqrt()).float()
    assert ((got - ref).abs() <= 20 * 2.0 ** -24 * ref.abs()).all()


def test_offsets_past_32_bits():
    """Tokens whose rows lie more than 2^32 bytes apart."""
    d, h = 64, 2
    far = 2 ** 31 + 4096
    base = torch.zeros(far + h * d, dtype=torch.float16, device="cuda")
    q = base.as_strided((2, h, d), (far, d, 1))
    x = rows(np.random.default_rng(0), (2, h, d), torch.float16)
    q.copy_(x)
    pos = torch.tensor([3, 70000], dtype=torch.int32, device="cuda")
    rope = iq.isoq_rope_init(d)
    assert torch.equal(iq.isoq_qk_norm_rope(rope, q, None, pos)[0], iq.isoq_qk_norm_rope(rope, x, None, pos)[0])


def test_streams_and_graphs():
    d = 128
    rng = np.random.default_rng(2)
    q, k = rows(rng, (17, 8, d), torch.float16), rows(rng, (17, 2, d), torch.float16)
    pos = torch.from_numpy(positions(rng, 17)).cuda()
    rope = iq.isoq_rope_init(d)
    ref = [x.clone() for x in iq.isoq_qk_norm_rope(rope, q, k, pos)]
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    got = iq.isoq_qk_norm_rope(rope, q, k, pos, stream=stream)
    stream.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, ref))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = iq.isoq_qk_norm_rope(rope, q, k, pos)
    for shift in range(3):
        pos.add_(1)
        ref = iq.isoq_qk_norm_rope(rope, q, k, pos)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, ref))


def test_no_tokens():
    rope = iq.isoq_rope_init(64)
    q = torch.zeros(0, 4, 64, device="cuda")
    got = iq.isoq_qk_norm_rope(rope, q, None, torch.zeros(0, dtype=torch.int32, device="cuda"))
    assert got[0].shape == q.shape
