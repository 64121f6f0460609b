"""Attention over values whose norms differ by many orders of magnitude: a row's
result is as exact as its own weights and norms allow, whatever norms stand at
positions that it does not attend to, or attends to with next to no weight, and
whatever norms came before.  Reference and tolerances of test_gpu_kv_attn.py,
which are relative to sum p ||v|| of each row.  Logits are steered: every key has
the same indices, the queries lie along it, so a logit is its position's key norm.
Needs an MI355X."""
import numpy as np
import pytest

import oracle

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

import paper_2603_28430_amd as iq  # noqa: E402
from test_gpu_kv_attn import check, device, reference, setup  # noqa: E402


def steered(variant, d, bits, dtype, q_lens, heads, group, seq_lens, logits, norms, seed=0, bs=16):
    """logits, norms: [positions] for every sequence and head (its first seq_lens[s])."""
    rng, pw = np.random.default_rng(seed), oracle.padded_width(variant, d)
    calls = []

    def keys(s, h, length):
        calls.append((s, h))
        if len(calls) <= len(seq_lens) * heads:
            return np.full((length, pw), (1 << bits) - 1, np.uint8), np.float32(logits[:length])
        return rng.integers(0, 1 << bits, (length, pw)).astype(np.uint8), np.float32(norms[:length])
    w = setup(variant, d, bits, dtype, q_lens, heads * group, heads, bs, seq_lens, keys=keys, seed=seed)
    _, rot, c = w["sides"][0]
    per = oracle.raw_params_per_set(variant, d)
    for h in range(heads):
        x = oracle.dequantize(variant, d, bits, np.asarray(rot).reshape(-1)[h * per:][:per], w["levels"],
                              np.full((1, pw), (1 << bits) - 1, np.uint8), np.ones(1))[0]
        w["q"][:, h * group:(h + 1) * group] = x / (x @ x)
    return w


def run(w):
    """The call, checked: lse of every row, and the outputs that fp16 holds (fp32: all)."""
    out, lse = iq.isoq_kv_attn(**device(w), scale=1.0)
    torch.cuda.synchronize()
    ref = reference(w, 1.0)
    for (t, hq), (_, l, _, bl) in ref.items():
        assert abs(float(lse[t, hq]) - l) <= bl, (t, hq, float(lse[t, hq]), l)
    held = {k: v for k, v in ref.items() if w["dtype"] == "f32" or np.abs(v[0]).max() < 60000}
    assert held
    check(out, lse, held)


# (by digits 4, 8 and 12 rows a workgroup and more; in fp16; width-generic)
KERNELS = [(128, 2, "f16", 3, 1), (128, 3, "f16", 2, 4), (128, 4, "f16", 3, 4), (64, 4, "f32", 3, 1), (96, 3, "f32", 2, 3),
           (80, 2, "f32", 12, 1), (256, 4, "f32", 3, 3), (192, 3, "f16", 5, 1), (512, 2, "f32", 3, 1), (128, 3, "f32", 9, 4),
           (128, 2, "f16", 40, 1), (128, 3, "f16", 20, 2), (128, 4, "f16", 40, 4), (64, 3, "f16", 33, 1), (80, 4, "f16", 70, 2),
           (96, 2, "f16", 9, 4), (70, 3, "f16", 3, 2), (70, 4, "f32", 5, 1)]


@pytest.mark.parametrize("ratio", [1e6, 1e9, 1e13])
@pytest.mark.parametrize("d,bits,dtype,n,group", KERNELS)
def test_a_later_tokens_value_is_large(d, bits, dtype, n, group, ratio):
    """The newest token's value is `ratio` times the others': the tokens before it do not attend to it."""
    rng = np.random.default_rng(n)
    length = 90
    logits, norms = rng.uniform(0.1, 2.0, length), rng.uniform(0.5, 2.0, length)
    norms[length - 1] = ratio
    w = steered("full", d, bits, dtype, [n, 1], 2, group, [length, 70], logits, norms, seed=d)
    run(w)


@pytest.mark.parametrize("d,bits,dtype,n,group", KERNELS)
def test_values_grow_from_token_to_token(d, bits, dtype, n, group):
    """A prompt whose values grow by up to 10^20: each row's sum is its newest position's."""
    length = max(n, 40)
    t = np.arange(length)
    norms = 10.0 ** (np.maximum(0, t - (length - n)) / n * 20.0)
    w = steered("fast", d, bits, dtype, [n], 2, group, [length], np.full(length, 0.7), norms, seed=d)
    run(w)


@pytest.mark.parametrize("where", [3, 70, 130])
@pytest.mark.parametrize("ratio", [1e6, 1e9, 1e13])
@pytest.mark.parametrize("d,bits,dtype,n,group", KERNELS)
def test_a_large_value_with_next_to_no_weight(d, bits, dtype, n, group, ratio, where):
    """e^-45 of the weight and `ratio` of the norm: 1e-6 of the sum at most, with
    the others before, in and after its tile."""
    rng = np.random.default_rng(n + where)
    length = 200 + n
    logits, norms = rng.uniform(45.0, 46.0, length), rng.uniform(0.5, 2.0, length)
    logits[where], norms[where] = 0.5, ratio
    run(steered("full", d, bits, dtype, [n, 1], 2, group, [length, 170], logits, norms, seed=d))


@pytest.mark.parametrize("tiles", [((1e18, 1.0), (1e-18, 1.0), (1.0, 64.0)), ((1e16, 1.0), (1e-17, 1.0), (2.0, 64.0)),
                                   ((1e-18, 30.0), (1e18, 0.1), (1.0, 110.0)), ((1.0, 60.0), (1e18, 0.5), (1e-18, 60.0)),
                                   ((1e-18, 1.0), (1e-12, 2.0), (1e-3, 40.0)), ((10.0, 2.0),) * 8 + ((1e-31, 2.0), (3.0, 2.0)),
                                   ((2.0, 1.0), (1e-31, 1.0)), ((1e-36, 2.0), (2.0, 2.0), (1e-36, 2.0), (1.0, 2.0))])
@pytest.mark.parametrize("d,bits,dtype,n,group", KERNELS)
def test_norms_from_tile_to_tile(d, bits, dtype, n, group, tiles):
    """Tiles of 64 and of 128 positions, each with a norm and a logit of its own,
    both ends of what the encoder takes (rows of 1e-18 to 1e18) and past them among
    them; where the sum is made of the last one it is held to that one's size."""
    rng = np.random.default_rng(n)
    for size in (64, 128):
        norms = np.concatenate([v * rng.uniform(0.5, 1.0, size) for v, _ in tiles])
        logits = np.concatenate([np.full(size, x) for _, x in tiles])
        run(steered("2d", d, bits, dtype, [n], 1, group, [len(norms)], logits, norms, seed=d))


@pytest.mark.parametrize("d,bits,dtype,n,group", KERNELS)
def test_norms_at_random(d, bits, dtype, n, group):
    """Norms over 30 orders of magnitude, position by position, with logits that
    bring the products of weight and norm to the same size."""
    rng = np.random.default_rng(n)
    length = 300
    e = rng.uniform(-15.0, 15.0, length)
    e[rng.integers(0, length, 20)] = -15.0
    logits = 40.0 - np.log(10.0) * e * rng.uniform(0.9, 1.0, length)
    norms = 10.0 ** e
    w = steered("full", d, bits, dtype, [n], 2, group, [length], logits, norms, seed=d)
    ref = reference(w, 1.0)
    sizes = [np.abs(o).max() for o, _, _, _ in ref.values()]
    if dtype == "f16":   # (outputs inside fp16's normal numbers)
        c = w["sides"][1][2]
        f = np.float32(1.0 / max(sizes))
        c.rho = c.rho * f
        for h in range(2):
            c.norms[0, h] = c.norms[0, h] * f
    run(w)


@pytest.mark.parametrize("step", [5, 6, 9, -5, -7])
@pytest.mark.parametrize("d,bits,dtype,n,group", KERNELS)
def test_norms_fall_as_the_logits_rise(d, bits, dtype, n, group, step):
    """From tile to tile norms by 2^-step and logits by step ln 2, so that the units of
    weights and of exponentials move against each other and their product stays."""
    rng = np.random.default_rng(n)
    tiles, size = 6, 64
    k = np.repeat(np.arange(tiles), size)
    norms = 2.0 ** (-step * (k - tiles // 2)) * rng.uniform(0.55, 0.95, len(k))
    logits = 40.0 + step * (k - tiles // 2) * np.log(2.0) + rng.uniform(0.0, 0.2, len(k))
    w = steered("full", d, bits, dtype, [n], 2, group, [len(k)], logits, norms, seed=d)
    run(w)
