"""Rotary positions of tokens behind a prefix: isoq_kv_plan counts a sequence's own positions
from 0, its prefix's length is added before isoq_qk_norm_rope, and isoq_kv_attn_prefix then gives
what isoq_kv_attn does of the whole sequence in a cache of its own; without it, it does not.

Tolerance: both results against the definition as test_gpu_kv_attn.py derives it for fp32 (the
rows of both caches are the same, so their records are), with the norms at their largest.
Needs an MI355X."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

import paper_2603_28430_amd as iq  # noqa: E402

D, BITS, BS, KV, GROUP = 64, 4, 16, 2, 2


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def planes(blocks):
    rec = iq.isoq_record_bytes("fast", D, BITS)
    return torch.zeros(blocks, KV, BS, rec, dtype=torch.uint8, device="cuda"), torch.zeros(blocks, KV, BS, device="cuda")


def plan(want, blocks, n_tokens):
    """A step's plan of sequences that begin, in a cache of that many blocks."""
    n = len(want)
    table = torch.full((n, 8), -1, dtype=torch.int32, device="cuda")
    got = iq.isoq_kv_plan(ints([0] * n), ints(want), table, BS, torch.arange(blocks, dtype=torch.int32, device="cuda"),
                          ints([blocks]), n_tokens)
    return got[:4], table


@pytest.mark.parametrize("prefix_lens,prefix_start", [([50], None), ([50, 33], [0, 2, 3])])
def test_positions_behind_a_prefix(prefix_lens, prefix_start):
    gen = torch.Generator(device="cuda").manual_seed(1)
    own = [20, 7, 40, 5]
    of = [0, 0, 0, 0] if prefix_start is None else [0, 0, 1, None]
    rows = lambda n, heads: torch.randn(n, heads, D, device="cuda", generator=gen)   # noqa: E731
    pk, pv = (iq.isoq_params_init("fast", D, BITS, seed=s) for s in (1, 2))
    rope, scale, total = iq.isoq_rope_init(D), D ** -0.5, sum(own)
    q, k, v = rows(total, KV * GROUP), rows(total, KV), rows(total, KV)
    pre = [(rows(n, KV), rows(n, KV)) for n in prefix_lens]
    step = np.split(np.arange(total), np.cumsum(own)[:-1])

    # every sequence as a whole, in a cache of its own
    whole = [(prefix_lens[p] if p is not None else 0) + n for p, n in zip(of, own)]
    (lens, q_start, slots, pos), table = plan(whole, 40, sum(whole))
    parts = [[x for p, s in zip(of, step) for x in (([pre[p][i]] if p is not None else []) + [(k, v)[i][s]])] for i in (0, 1)]
    kw, vw = (torch.cat(x) for x in parts)
    kw = iq.isoq_qk_norm_rope(rope, kw, None, pos)[0]
    cache = planes(40), planes(40)
    iq.isoq_kv_append(pk, kw, slots, *cache[0], pv, vw, *cache[1])
    real = torch.cat([pos[end - n:end] for end, n in zip(np.cumsum(whole), own)])
    qw = iq.isoq_qk_norm_rope(rope, q, None, real)[0]
    starts = ints(np.concatenate([[0], np.cumsum(own)]))
    ref, _ = iq.isoq_kv_attn(pk, qw, *cache[0], pv, *cache[1], table, lens, scale, starts, max(own))

    # prefixes in the cache once, and a step of the sequences behind them
    (lens_p, _, slots_p, pos_p), table_p = plan(prefix_lens, 10, sum(prefix_lens))
    cache = planes(40), planes(40)
    kp, vp = (torch.cat([x[i] for x in pre]) for i in (0, 1))
    kp = iq.isoq_qk_norm_rope(rope, kp, None, pos_p)[0]
    iq.isoq_kv_append(pk, kp, slots_p, *cache[0], pv, vp, *cache[1])
    n_tokens = total + 3     # (some padding)
    (lens, q_start, slots, positions), table = plan(own, 30, n_tokens)
    slots, table = torch.where(slots >= 0, slots + 10 * BS, slots), torch.where(table >= 0, table + 10, table)
    pad = lambda x: torch.cat([x, x[:3]])   # noqa: E731
    if prefix_start is None:
        behind = positions + lens_p
    else:
        offsets = ints([prefix_lens[p] if p is not None else 0 for p in of])
        seq = torch.searchsorted(q_start[1:].contiguous(), torch.arange(n_tokens, device="cuda"), right=True)
        behind = positions + offsets[seq.clamp(max=len(own) - 1)]
    assert behind[:total].tolist() == real.tolist()
    out = {}
    for name, at in (("behind", behind), ("own", positions)):
        qs, ks = iq.isoq_qk_norm_rope(rope, pad(q), pad(k), at)
        iq.isoq_kv_append(pk, ks, slots, *cache[0], pv, pad(v), *cache[1])
        out[name], _ = iq.isoq_kv_attn_prefix(pk, qs, *cache[0], pv, *cache[1], table, lens, table_p, lens_p,
                                              None if prefix_start is None else ints(prefix_start), scale, q_start, max(own))
    top = float(iq.isoq_codebook_lloyd(BITS, D).max()) * D ** 0.5     # ||c[idx]|| at most
    big = lambda *x: max(float(y.norm(dim=-1).max()) for y in x)   # noqa: E731
    t = scale * big(q) * big(k, *(x for x, _ in pre)) * top
    ds, vn = (4 + 8) * 2.0 ** -23 * t + 2.0 ** -22 * t, big(v, *(x for _, x in pre)) * top
    tol = 2 * (2 * ds + 2.0 ** -19 + 2.0 ** -20 + 2.0 ** -22 + 2.0 ** -22) * vn
    off = {name: float((x[:total] - ref).norm(dim=-1).max()) for name, x in out.items()}
    assert off["behind"] <= tol < 0.01 < off["own"], (off, tol)
