"""The operators around the paged quantized K/V cache that a serving step takes
besides append and causal attention, as calls whose speed and exactness are
tracked on one MI355X: the block tables and slots of a step's tokens (plan),
norms and rotary positions of queries and keys (rope), attention of a batch that
shares a prefix (prefix), and attention to an encoder's states (cross).

A cache slot of a key (or value) head holds rho and the b-bit indices of a
rotated row: x_hat = rho T^{-1} c[idx], T a block rotation of the head, c the
codebook.  Where `own` is false, run() computes an operator in its plain form,
elementary torch operations in 32 bits (angles in 64); where it is true it calls
the package.  prepare() makes a case's inputs on the GPU from the seed alone;
exact() is the definition in 64 bits, from the indices rather than the packed
records.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
F16, F32, F64, I32, I64 = torch.float16, torch.float32, torch.float64, torch.int32, torch.int64
EPS = 1e-6        # of the norms
BASE = 500000.0   # of the rotary frequencies

_CACHE = dict(variant="fast", d=128, bits=3, block_size=16, dtype="f16")


def _attn(name, op, **kw):
    return dict(_CACHE, **dict({"name": name} if name else {}, op=op, **kw))


def _plan(name, **kw):
    return dict({"name": name} if name else {}, op="plan", **kw)


def _rope(name, **kw):
    return dict({"name": name} if name else {}, op="rope", **kw)


def listed():
    return [
        # a decode step's bookkeeping: one token for each of 64 sequences
        _plan("plan_decode", kind="decode", seqs=64, ctx=4096, block_size=16),
        # a mixed step: single tokens, prompts that begin, drafts taken back, sequences that have ended
        _plan("plan_mixed", kind="mixed", seqs=513, ctx=3001, block_size=13),
        # long prompts that begin together
        _plan("plan_prefill", kind="prefill", seqs=8, ctx=32768, block_size=16),
        # a decode step's queries and keys
        _rope("rope_decode", tokens=32, heads=32, kv_heads=8, d=128, rot=128, halves=True, norm=True, scaled=False,
              packed=False, far=131072, dtype="f16"),
        # prompts, as they come out of one projection of queries, keys and values
        _rope("rope_prefill", tokens=32768, heads=32, kv_heads=8, d=128, rot=128, halves=True, norm=True, scaled=True,
              packed=True, far=32768, dtype="f16"),
        # fp32 rows of an odd width, adjacent pairs in a part of the head, very far positions
        _rope("rope_f32_d90", tokens=4133, heads=5, kv_heads=5, d=90, rot=44, halves=False, norm=False, scaled=True,
              packed=False, far=2 ** 30, dtype="f32"),
        # a few requests behind one short instruction: latency
        _attn("prefix_short", "prefix", seqs=4, prefixes=1, heads=8, group=4, prefix=700, ctx=60, q_len=1),
        # a serving batch behind one long instruction, 4 bits
        _attn("prefix_batch", "prefix", seqs=64, prefixes=1, heads=8, group=4, prefix=8192, ctx=512, q_len=1, bits=4,
              variant="full"),
        # drafts of three groups of requests, one of them behind nothing; fp32, odd sizes
        _attn("prefix_drafts_f32", "prefix", seqs=24, prefixes=3, heads=4, group=5, prefix=3001, ctx=300, q_len=5, d=96,
              bits=2, variant="2d", block_size=17, dtype="f32"),
        # many questions about one very long document
        _attn("prefix_longest", "prefix", seqs=32, prefixes=1, heads=8, group=8, prefix=131071, ctx=1000, q_len=1),
        # a step of a decoder that attends to its encoder's states, inputs of different lengths (an empty one among them)
        _attn("cross_decode", "cross", seqs=16, heads=16, group=1, ctx=1500, q_len=1),
        # whole targets against their inputs
        _attn("cross_targets", "cross", seqs=8, heads=16, group=1, ctx=1500, q_len=448, d=64, bits=4),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["plan", "rope", "prefix", "prefix", "cross"])
    if op == "plan":
        kind = rng.choice(["decode", "mixed", "prefill"])
        seqs = _log_int(rng, 1, 2000) if kind != "prefill" else rng.choice([1, 3, 8, 20])
        return _plan(None, kind=kind, seqs=seqs, ctx=_log_int(rng, 2, min(32768, 2 ** 18 // seqs if kind == "prefill" else 2 ** 21 // seqs)),
                     block_size=rng.choice([16, 32, 64, 13, 1]))
    if op == "rope":
        d = rng.choice([64, 80, 96, 128, 128, 192, 256, 90, 20, 512])
        heads, kv_heads = rng.choice([(32, 8), (8, 8), (16, 2), (5, 1), (64, 8), (12, 12)])
        return _rope(None, tokens=_log_int(rng, 1, 2 ** 27 // (d * (heads + kv_heads))), heads=heads, kv_heads=kv_heads, d=d,
                     rot=rng.choice([d, d, d // 4 * 2, d // 2 // 16 * 16 or d]), halves=rng.random() < 0.6,
                     norm=rng.random() < 0.6, scaled=rng.random() < 0.5, packed=rng.random() < 0.4,
                     far=_log_int(rng, 100, 2 ** 30), dtype=rng.choice(["f16", "f16", "f32"]))
    kw = dict(variant=rng.choice(["full", "fast", "2d"]), bits=rng.choice([2, 3, 4]),
              d=rng.choice([64, 80, 96, 128, 128, 160, 192, 256]), block_size=rng.choice([16, 16, 32, 64, 13]),
              dtype=rng.choice(["f16", "f16", "f32"]))
    d = kw["d"]
    heads, group = rng.choice([(8, 1), (16, 1), (8, 4), (4, 8), (16, 2), (8, 5), (2, 16), (1, 12)])
    q_len = rng.choice([1, 1, 1, 2, 5, 16]) if op == "prefix" else _log_int(rng, 1, 448)
    seqs = rng.choice([2, 3, 8, 16, 33, 64]) if op == "prefix" else rng.choice([1, 2, 4, 8, 13])
    rows = heads * group * q_len * seqs
    # (at most a third of the longest listed case's operations, where fp32 and wide rows take longer; and of memory for the plain form)
    top = min(2 ** 35 // (rows * d), 2 ** 28 // rows, 2 ** 28 // (heads * d))
    if op == "prefix":
        return _attn(None, op, heads=heads, group=group, seqs=seqs, q_len=q_len, prefixes=rng.choice([1, 1, 2, 5]),
                     prefix=_log_int(rng, 1, max(2, min(100000, top))), ctx=_log_int(rng, q_len, max(q_len, min(1500, top // 4, 2 ** 26 // (heads * seqs * d)))), **kw)
    return _attn(None, op, heads=heads, group=group, seqs=seqs, q_len=q_len,
                 ctx=_log_int(rng, 1, max(2, min(30000, top, 2 ** 27 // (heads * seqs * d)))), **kw)


# ---- inputs ------------------------------------------------------------------------

def generator(seed, stream):
    return torch.Generator(device=DEV).manual_seed(int(seed) * 64 + stream)


def device_ints(a, dtype=np.int32):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(a).astype(dtype))).to(DEV)


def step_lengths(case, seed):
    """(lengths before, lengths after) of a step's sequences."""
    r = np.random.default_rng([seed, 41])
    n, ctx = case["seqs"], case["ctx"]
    if case["kind"] == "prefill":
        return np.zeros(n, np.int64), np.concatenate([[ctx], r.integers(max(1, ctx // 2), ctx + 1, n - 1)])
    old = r.integers(1, ctx, n)
    new = old + 1
    if case["kind"] == "mixed":
        what = r.random(n)
        new = np.where(what < 0.1, r.integers(0, old + 1), new)                  # drafts taken back
        new = np.where(what < 0.05, 0, new)                                     # ended
        old = np.where(what > 0.95, 0, old)
        new = np.where(what > 0.95, r.integers(1, min(ctx, 700) + 1, n), new)     # begun
    return old, new


def plan_tokens(case):
    """The step's tokens at most, as its program knows them: buffers are as long."""
    return case["seqs"] * case["ctx"] if case["kind"] == "prefill" else \
        case["seqs"] + (case["seqs"] // 8 + 4) * min(case["ctx"], 700) if case["kind"] == "mixed" else case["seqs"]


def frequencies(case):
    """Angles (radians) a position of the rot / 2 pairs, in 64 bits: base^(-2 i / rot), and for contexts eight times as
    long as the first 8,192 positions pairs that turn less than once in those slowed by 8, more than 32 times not, blended between."""
    f = BASE ** (-2.0 * np.arange(case["rot"] // 2) / case["rot"])
    if case["scaled"]:
        keep = np.clip((f * 8192 / (2 * math.pi) - 1.0) / 31.0, 0.0, 1.0)
        f = f * (keep + (1.0 - keep) / 8.0)
    return f


def amplitude(case):
    return 1.1 if case["scaled"] else 1.0


def rows_of(case, seed):
    """Query and key rows [tokens, heads, d] (views of one projection's output where they are packed), positions, weights."""
    g = generator(seed, 5)
    t, hq, hk, d = case["tokens"], case["heads"], case["kv_heads"], case["d"]
    dt = F16 if case["dtype"] == "f16" else F32
    width = hq + 2 * hk if case["packed"] else hq + hk
    x = torch.randn((t, width, d), generator=g, device=DEV)
    x *= torch.exp(0.5 * torch.randn((t, width, 1), generator=g, device=DEV))
    x = x.to(dt)
    q, k = x[:, :hq], x[:, hq:hq + hk]
    if not case["packed"]:
        q, k = q.contiguous(), k.contiguous()
    pos = torch.randint(0, case["far"], (t,), generator=g, device=DEV, dtype=I32)
    w = 1.0 + 0.2 * torch.randn((2, d), generator=g, device=DEV)
    return q, k, pos, w[0].contiguous(), w[1].contiguous()


_codebooks = {}


def codebook(bits, d):
    """Lloyd-Max levels of N(0, 1/d), ascending and symmetric (numpy, 64 bits)."""
    if bits not in _codebooks:
        h = 1 << (bits - 1)
        c = (np.arange(h) + 0.5) * (3.0 / h)
        for _ in range(2000):
            t = np.concatenate([[0.0], 0.5 * (c[1:] + c[:-1]), [40.0]])
            pdf = np.exp(-0.5 * t * t) / math.sqrt(2 * math.pi)
            cdf = np.array([0.5 * (1 + math.erf(v / math.sqrt(2))) for v in t])
            c = (pdf[:-1] - pdf[1:]) / (cdf[1:] - cdf[:-1])
        _codebooks[bits] = np.concatenate([-c[::-1], c])
    return _codebooks[bits] / math.sqrt(d)


def record_bytes(case):
    return case["d"] * case["bits"] // 8   # (every width here is a multiple of 16)


def draws(case, seed):
    """Raw rotation draws [heads][...]: quaternions N(0, I_4) or planar angles."""
    rng = np.random.default_rng([seed, 11])
    if case["variant"] == "2d":
        return rng.uniform(0, 2 * math.pi, (case["heads"], case["d"] // 2))
    return rng.standard_normal((case["heads"], case["d"] // 4, 8 if case["variant"] == "full" else 4))


def matrices(case, seed):
    """The block rotations [heads, blocks, k, k] in 64 bits (k = 4; 2 for planar pairs)."""
    u = draws(case, seed)
    if case["variant"] == "2d":
        c, s = np.cos(u), np.sin(u)
        m = np.stack([np.stack([c, -s], -1), np.stack([s, c], -1)], -2)
    else:
        def product(q, sign):   # of a quaternion with the four units, from the left or the right
            a, b, c, d = np.moveaxis(q, -1, 0)
            e = sign * d, sign * c, sign * b
            return np.stack([np.stack(v, -1) for v in
                             ((a, -b, -c, -d), (b, a, -e[0], e[1]), (c, e[0], a, -e[2]), (d, -e[1], e[2], a))], -2)
        halves = u.reshape(u.shape[:-1] + (-1, 4))
        unit = (halves / np.linalg.norm(halves, axis=-1, keepdims=True)).reshape(u.shape)
        m = product(unit[..., :4], 1.0)
        if case["variant"] == "full":
            m = m @ product(unit[..., 4:] * np.array([1.0, -1.0, -1.0, -1.0]), -1.0)
    return torch.from_numpy(np.ascontiguousarray(m)).to(DEV)


def random_slots(case, blocks, seed, stream):
    """(indices [blocks, heads, block_size, d] uint8 as quantized rows have them, norms of the same slots)."""
    shape = (blocks, case["heads"], case["block_size"])
    count, base = math.prod(shape), 1 << 14
    g = generator(seed, stream)
    lev = codebook(case["bits"], 1)
    z = torch.randn((min(count, base), case["d"]), generator=g, device=DEV)
    idx = torch.bucketize(z, torch.tensor(0.5 * (lev[1:] + lev[:-1]), device=DEV, dtype=F32)).to(torch.uint8)
    if count > base:   # rows of the base, each rotated by a number of coordinates of its own
        pick = torch.randint(0, base * 8, (count,), generator=g, device=DEV, dtype=I32)
        idx = idx.repeat(1, 2).unfold(1, case["d"], 1)[:, :8].reshape(-1, case["d"])[pick]
    rho = math.sqrt(case["d"]) * torch.exp(0.3 * torch.randn(shape, generator=g, device=DEV))
    return idx.reshape(shape + (case["d"],)), rho


def pack(idx, bits):
    """Records [..., d bits / 8] of indices [..., d], least significant bit first."""
    v = idx.reshape(-1, idx.shape[-1] // 8, 8).to(I32)   # eight coordinates are `bits` bytes
    lo = sum(v[..., i] << (bits * i) for i in range(4))
    hi = sum(v[..., i + 4] << (bits * i) for i in range(4))
    w = lo.to(I64) | (hi.to(I64) << (4 * bits))
    out = torch.stack([(w >> (8 * i)) & 255 for i in range(bits)], -1)
    return out.to(torch.uint8).reshape(idx.shape[:-1] + (idx.shape[-1] * bits // 8,))


def piece(r):
    return 16 if r % 16 == 0 else 8 if r % 8 == 0 else r


def piece_major(rec):
    """[blocks, heads, block_size, R] records as the cache holds them: pieces of
    16 or 8 bytes (where that divides R) of consecutive positions adjacent."""
    nb, h, bs, r = rec.shape
    p = piece(r)
    return rec.reshape(nb, h, bs, r // p, p).transpose(2, 3).contiguous().reshape(nb, h, bs, r)


def layout(case, seed):
    """(blocks in the cache, block table of the sequences, of the prefixes), blocks placed at random, none shared."""
    bs = case["block_size"]
    n, m = case["seqs"], case.get("prefixes", 0)
    per, pre = -(-case["ctx"] // bs), -(-case.get("prefix", 0) // bs)
    blocks = n * per + m * pre + 7
    perm = np.random.default_rng([seed, 19]).permutation(blocks)
    return blocks, perm[:n * per].reshape(n, per), perm[n * per:n * per + m * pre].reshape(m, pre)


def lengths(case, seed):
    """(contexts, new tokens) of the sequences: an empty sequence among eight or more."""
    r = np.random.default_rng([seed, 17])
    n, ctx, q = case["seqs"], case["ctx"], case["q_len"]
    new = np.random.default_rng(q).integers(max(1, q // 2), q + 1, n)   # (as many rows for every seed)
    new[-1] = q
    lens = np.maximum(r.integers(max(1, ctx // 4), ctx + 1, n), np.minimum(new, ctx))
    if n >= 8:
        lens[1] = 0        # a slot of the batch without a sequence
    return lens, new


def shares(case, seed):
    """(first sequence of each prefix and their number, the prefixes' lengths): the third of several prefixes is empty."""
    r = np.random.default_rng([seed, 23])
    n, m = case["seqs"], case["prefixes"]
    first = np.sort(np.random.default_rng(n).integers(0, n + 1, m - 1))
    lens = r.integers(max(1, case["prefix"] // 2), case["prefix"] + 1, m)
    lens[0] = case["prefix"]
    if m >= 3:
        lens[2] = 0
    return np.concatenate([[0], first, [n]]), lens


def queries(case, total, seed):
    """Query rows [tokens, query heads, d]: Gaussian, a few channels larger than the rest."""
    g = generator(seed, 3)
    q = 1.5 * torch.randn((total, case["heads"] * case["group"], case["d"]), generator=g, device=DEV)
    q[..., torch.randint(0, case["d"], (3,), generator=g, device=DEV)] *= 2.0
    return q.to(F16 if case["dtype"] == "f16" else F32)


def prepare(case, seed):
    s = dict(case=case)
    if own:
        import paper_2603_28430_amd as iq
    if case["op"] == "plan":
        old, new = step_lengths(case, seed)
        bs = case["block_size"]
        per = -(-max(case["ctx"], int(new.max())) // bs)
        held = int((-(-old // bs)).sum())
        blocks = case["seqs"] * per + 5
        perm = np.random.default_rng([seed, 43]).permutation(blocks)
        table = np.full((case["seqs"], per), -1)
        table[np.arange(per) < -(-old // bs)[:, None]] = perm[:held]
        s.update(lens=device_ints(old), new=device_ints(new), table=device_ints(table),
                 free=device_ints(np.concatenate([perm[held:], np.full(held, -1)])), n_free=device_ints([blocks - held]))
        return s
    if case["op"] == "rope":
        s["q"], s["k"], s["pos"], s["wq"], s["wk"] = rows_of(case, seed)
        s["freq"] = torch.from_numpy(frequencies(case)).to(DEV)   # (for the plain form)
        if own:   # the rotation's handle, which a program builds once
            kw = dict(factor=8.0, original=8192, low=1.0, high=32.0) if case["scaled"] else {}
            s["rope"] = iq.isoq_rope_init(case["d"], case["rot"], "halves" if case["halves"] else "pairs",
                                          freqs=iq.isoq_rope_freqs(case["rot"], BASE, **kw), amplitude=amplitude(case))
        return s
    blocks, table, prefix_table = layout(case, seed)
    s["table"] = device_ints(table)
    for name, stream in (("k", 22), ("v", 24)):
        idx, rho = random_slots(case, blocks, seed, stream)
        s[name + "_idx"], s[name + "_rho"] = piece_major(pack(idx, case["bits"])), rho
        del idx
    lens, new = lengths(case, seed)
    s["lens"] = device_ints(lens)
    s["q"] = queries(case, int(new.sum()), seed)
    s["scale"] = 1.0 / math.sqrt(case["d"])
    s["start"] = device_ints(np.concatenate([[0], np.cumsum(new)])) if case["q_len"] > 1 else None
    if case["op"] == "prefix":
        first, plens = shares(case, seed)
        s["prefix_table"], s["prefix_lens"], s["prefix_start"] = device_ints(prefix_table), device_ints(plens), device_ints(first)
        ends = np.concatenate([[0], np.cumsum(new)])[first]
        s["prefix_tokens"] = int((ends[1:] - ends[:-1]).max())   # the most tokens that share one, which a program knows
    if own:   # the quantizers' handles, which a program builds once
        s["pk"], s["pv"] = [
            iq.isoq_params_init(case["variant"], case["d"], case["bits"], case["heads"], rot=draws(case, x).reshape(-1),
                                codebook=codebook(case["bits"], case["d"])) for x in (seed, seed + 1000003)]
    # the rotations and levels that the plain form works with
    s["lev"] = torch.from_numpy(codebook(case["bits"], case["d"])).to(DEV, F32)
    s["mk"], s["mv"] = matrices(case, seed).to(F32), matrices(case, seed + 1000003).to(F32)
    return s


# ---- one pass ------------------------------------------------------------------------

def run(s):
    case = s["case"]
    if not own:
        return {"plan": plain_plan, "rope": plain_rope, "prefix": plain_prefix, "cross": plain_cross}[case["op"]](s)
    import paper_2603_28430_amd as iq

    if case["op"] == "plan":
        step = iq.isoq_kv_plan(s["lens"], s["new"], s["table"], case["block_size"], s["free"], s["n_free"],
                               n_tokens=plan_tokens(case))
        return (*step, s["table"], s["free"])
    if case["op"] == "rope":
        w = dict(q_weight=s["wq"], k_weight=s["wk"], eps=EPS) if case["norm"] else {}
        return iq.isoq_qk_norm_rope(s["rope"], s["q"], s["k"], s["pos"], **w)
    if case["op"] == "prefix":
        return iq.isoq_kv_attn_prefix(s["pk"], s["q"], s["k_idx"], s["k_rho"], s["pv"], s["v_idx"], s["v_rho"], s["table"],
                                      s["lens"], s["prefix_table"], s["prefix_lens"], s["prefix_start"], scale=s["scale"],
                                      q_start=s["start"], max_q_len=case["q_len"], max_prefix_tokens=s["prefix_tokens"])
    return iq.isoq_kv_attn_cross(s["pk"], s["q"], s["k_idx"], s["k_rho"], s["pv"], s["v_idx"], s["v_rho"], s["table"],
                                 s["lens"], scale=s["scale"], q_start=s["start"], max_q_len=case["q_len"])


def plain_plan(s):
    """(lengths, first token of each sequence, slots, positions, free blocks left, block table, free list)."""
    case = s["case"]
    bs, tokens = case["block_size"], plan_tokens(case)
    table, free = s["table"], s["free"]
    n, width = table.shape
    old, want = s["lens"].clamp(0, width * bs).long(), s["new"].clamp(0, width * bs).long()
    have, need = (old + bs - 1) // bs, (want + bs - 1) // bs
    grow, drop = (need - have).clamp(min=0), (have - need).clamp(min=0)
    there = s["n_free"].long() + drop.sum()
    before = grow.cumsum(0)
    fine = (grow == 0) | (before <= there)        # its blocks are there
    j = torch.arange(width, device=DEV)
    # blocks of what ends go on top of the free list, those of what grows come from its top
    back = (j >= need[:, None]) & (j < have[:, None])
    at = s["n_free"].long() + (drop.cumsum(0) - drop)[:, None] + j - need[:, None]
    longer = torch.cat([free, free.new_zeros(1)])
    longer.scatter_(0, torch.where(back, at, len(free)).flatten(), table.flatten())
    free.copy_(longer[:-1])
    take = (j >= have[:, None]) & (j < need[:, None]) & fine[:, None]
    at = there - 1 - ((before - grow)[:, None] + j - have[:, None])
    table.copy_(torch.where(take, free[at.clamp(0, len(free) - 1)], table))
    lens = torch.where(fine, want, old)
    new = (want - old).clamp(min=0)
    start = torch.cat([new.new_zeros(1), new.cumsum(0)])
    t = torch.arange(tokens, device=DEV)
    q = torch.searchsorted(start[1:], t, right=True)
    there_t = q < n
    q = q.clamp(max=n - 1)
    pos = torch.where(there_t, old[q] + t - start[q], 0)
    blk = table[q, (pos // bs).clamp(max=width - 1)].long()
    slots = torch.where(there_t & fine[q] & (blk >= 0), blk * bs + pos % bs, -1)
    left = there - torch.where(fine, grow, 0).sum()
    return (lens.to(I32), start.to(I32), slots, pos.to(I32), left.to(I32).reshape(1), table, free)


def plain_rope(s):
    case = s["case"]
    half = case["rot"] // 2
    angle = torch.remainder(s["pos"].double()[:, None] * (s["freq"] / (2 * math.pi)), 1.0) * (2 * math.pi)
    cos, sin = (f(angle).to(F32)[:, None] * amplitude(case) for f in (torch.cos, torch.sin))
    out = []
    for x, w in ((s["q"], s["wq"]), (s["k"], s["wk"])):
        dt, x = x.dtype, x.float()
        if case["norm"]:
            x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w
        a, b = (x[..., :half], x[..., half:2 * half]) if case["halves"] else (x[..., :2 * half:2], x[..., 1:2 * half:2])
        a, b = a * cos - b * sin, a * sin + b * cos
        r = torch.cat([a, b], -1) if case["halves"] else torch.stack([a, b], -1).flatten(-2)
        out.append(torch.cat([r, x[..., 2 * half:]], -1).to(dt))
    return tuple(out)


def levels_of(s, cache, table):
    """c[idx] of every position behind a block table: [seqs, heads, positions, d]."""
    bits = s["case"]["bits"]
    nb, h, bs, r = cache.shape
    p = piece(r)
    c = cache.reshape(nb, h, r // p, bs, p)[table]                     # [seqs, blocks, heads, pieces, bs, p]
    rec = c.permute(0, 2, 1, 4, 3, 5).reshape(table.shape[0], h, -1, r)
    b = (rec.unsqueeze(-1) >> torch.arange(8, device=DEV, dtype=torch.uint8)) & 1
    b = b.reshape(rec.shape[:-1] + (-1, bits))
    return s["lev"][(b << torch.arange(bits, device=DEV, dtype=torch.uint8)).sum(-1, dtype=I32)]


def norms_of(rho, table):
    return rho[table].transpose(1, 2).reshape(table.shape[0], rho.shape[1], -1)


def block_product(m, x):
    """Block matrices m [heads, 1.., blocks, k, k] times rows x [..., d]."""
    x = x.reshape(x.shape[:-1] + (-1, m.shape[-1]))
    return (m * x.unsqueeze(-2)).sum(-1).flatten(-2)


def plain_part(s, row, limit, table):
    """Unnormalised attention of the tokens row [seqs, tokens] to the first limit [seqs, tokens] positions behind a
    table: the largest logit, the sum of exponentials [seqs, tokens, query heads], the sum of values (rotated) [.., d]."""
    case = s["case"]
    h, g, d = case["heads"], case["group"], case["d"]
    n, most = row.shape
    q = s["q"][row].float().reshape(n, -1, h, g, d).permute(0, 2, 1, 3, 4)      # [seqs, heads, tokens, group, d]
    q = block_product(s["mk"][:, None, None], q * s["scale"]).flatten(2, 3)
    logits = q @ levels_of(s, s["k_idx"], table).transpose(-1, -2) * norms_of(s["k_rho"], table).unsqueeze(-2)
    t = torch.arange(logits.shape[-1], device=DEV, dtype=I32)
    limit = limit.repeat_interleave(g, 1)[:, None, :, None]                     # [seqs, 1, rows, 1]
    logits = torch.where(t < limit, logits, float("-inf"))
    top = torch.where(limit > 0, logits.amax(-1, keepdim=True), float("-inf"))
    p = torch.exp(logits - torch.where(limit > 0, top, 0.0))
    o = (p * norms_of(s["v_rho"], table).unsqueeze(-2)) @ levels_of(s, s["v_idx"], table)
    total = p.sum(-1, keepdim=True)
    return [x.reshape(n, h, most, g, -1).permute(0, 2, 1, 3, 4).reshape(n, most, h * g, -1) for x in (top, total, o)]


def plain_rows(s, parts):
    """out and lse of tokens whose parts [(top, total, sum of values)] are given."""
    case = s["case"]
    top = torch.stack([p[0] for p in parts]).amax(0)
    some = top > float("-inf")
    total, o = 0.0, 0.0
    for m, l, x in parts:
        f = torch.where(some, torch.exp(m - torch.where(some, top, 0.0)), 0.0)
        total, o = total + f * l, o + f * x
    o = torch.where(some, o / torch.where(some, total, 1.0), 0.0)
    lse = torch.where(some, top + torch.log(torch.where(some, total, 1.0)), float("-inf"))[..., 0]
    h, g = case["heads"], case["group"]
    o = block_product(s["mv"].transpose(-1, -2)[:, None], o.reshape(-1, h, g, case["d"])).reshape(s["q"].shape)
    return o.to(s["q"].dtype), lse


def starts(s):
    return s["start"] if s["start"] is not None else torch.arange(s["case"]["seqs"] + 1, device=DEV, dtype=I32)


def rows_between(start, most, total):
    """Tokens [ranges, most] of consecutive ranges (clamped), and which of them there are."""
    i = torch.arange(most, device=DEV, dtype=I32)
    return (start[:-1, None] + i).clamp(max=total - 1), i < (start[1:] - start[:-1])[:, None], i


def plain_cross(s):
    row, valid, _ = rows_between(starts(s), s["case"]["q_len"], s["q"].shape[0])
    part = plain_part(s, row, torch.where(valid, s["lens"][:, None], 0), s["table"])
    return plain_rows(s, [[x[valid] for x in part]])


def plain_prefix(s):
    start, total = starts(s), s["q"].shape[0]
    row, valid, i = rows_between(start, s["case"]["q_len"], total)
    new = (start[1:] - start[:-1])[:, None]
    limit = torch.where(valid, s["lens"][:, None] - (new - 1 - i), 0)
    mine = [x[valid] for x in plain_part(s, row, limit, s["table"])]
    row, valid, _ = rows_between(start[s["prefix_start"]], s["prefix_tokens"], total)
    part = plain_part(s, row, torch.where(valid, s["prefix_lens"][:, None], 0), s["prefix_table"])
    return plain_rows(s, [[x[valid] for x in part], mine])


# ---- what a pass cannot do without, and the same in 64 bits -----------------------------

def work(case):
    if case["op"] == "plan":
        n, bs, kind = case["seqs"], case["block_size"], case["kind"]
        written = plan_tokens(case)                 # slots and positions, those of no token too
        new = 0.75 * n * case["ctx"] if kind == "prefill" else n * (1 + 0.05 * min(case["ctx"], 700) / 2) if kind == "mixed" else n
        return dict(bytes=12 * written + 16 * n + 8 * new / bs + 4 * n, flops=0)
    if case["op"] == "rope":
        es = 2 if case["dtype"] == "f16" else 4
        x = case["tokens"] * (case["heads"] + case["kv_heads"]) * case["d"]
        return dict(bytes=2 * es * x + 4 * case["tokens"], flops=6 * x)
    r, h, g, d = record_bytes(case), case["heads"], case["group"], case["d"]
    es = 2 if case["dtype"] == "f16" else 4
    new = int(lengths(case, 0)[1].sum())
    keys = 0.625 * (case["seqs"] - (case["seqs"] >= 8)) * case["ctx"]     # of the sequences themselves
    pairs = 0.625 * new * case["ctx"]
    if case["op"] == "prefix":
        first, plens = shares(case, 0)
        mean = np.where(plens > 0, 0.75 * case["prefix"], 0.0)
        mean[0] = case["prefix"]
        ends = np.concatenate([[0], np.cumsum(lengths(case, 0)[1])])[first]
        keys += float((mean * (ends[1:] > ends[:-1])).sum())
        pairs += float((mean * (ends[1:] - ends[:-1])).sum())
    return dict(bytes=keys * h * 2 * (r + 4) + new * h * g * (2 * d * es + 4) + keys / case["block_size"] * 4,
                flops=pairs * h * g * 4 * d)


def exact(case, seed):
    if case["op"] == "plan":
        return None     # (whole numbers)
    if case["op"] == "rope":
        return exact_rope(case, seed)
    h, g, bs, d = case["heads"], case["group"], case["block_size"], case["d"]
    blocks, table, prefix_table = layout(case, seed)
    caches = [random_slots(case, blocks, seed, 22), random_slots(case, blocks, seed, 24)]
    lens, new = lengths(case, seed)
    rot = [matrices(case, seed), matrices(case, seed + 1000003)]
    lev = torch.from_numpy(codebook(case["bits"], d)).to(DEV)
    q = queries(case, int(new.sum()), seed).double()
    out = torch.zeros(q.shape, device=DEV, dtype=F64)
    lse = torch.full(q.shape[:2], float("-inf"), device=DEV, dtype=F64)

    def cached(blocks_of, length, i):
        """The rows themselves of head i: the levels rotated back, times the norm."""
        t = np.arange(length)
        blk, pos = torch.from_numpy(blocks_of[t // bs].astype(np.int64)).to(DEV), torch.from_numpy(t % bs).to(DEV)
        rows = []
        for (idx, rho), m in zip(caches, rot):
            c = lev[idx[blk, i, pos].long()].reshape(length, d // m.shape[-1], m.shape[-1])
            x = sum(c[..., j, None] * m[i][:, j] for j in range(m.shape[-1])).reshape(length, d)
            rows.append(x * rho[blk, i, pos].double()[:, None])
        return rows

    first, plens = shares(case, seed) if case["op"] == "prefix" else (np.array([0, case["seqs"]]), np.array([0]))
    ends = np.concatenate([[0], np.cumsum(new)])
    for p in range(len(plens)):
        for i in range(h):
            shared = cached(prefix_table[p], int(plens[p]), i) if plens[p] > 0 else None
            for s in range(first[p], first[p + 1]):
                n, length = int(new[s]), int(lens[s])
                mine = cached(table[s], length, i)
                for j in range(0, n, 64):
                    m = min(n, j + 64) - j
                    at = slice(int(ends[s]) + j, int(ends[s]) + j + m)
                    x = q[at, i * g:(i + 1) * g].reshape(-1, d)
                    a = x @ mine[0].t().contiguous() / math.sqrt(d)
                    if case["op"] == "prefix":
                        last = length - n + j + torch.arange(m, device=DEV).repeat_interleave(g)
                        a = a.masked_fill(torch.arange(length, device=DEV) > last[:, None], float("-inf"))
                    keys, vals = [a], [mine[1]]
                    if shared is not None:
                        keys, vals = [x @ shared[0].t().contiguous() / math.sqrt(d), a], [shared[1], mine[1]]
                    a = torch.cat(keys, 1)
                    if a.shape[1] == 0:
                        continue
                    l = torch.logsumexp(a, -1)
                    w = torch.exp(a - torch.where(l > float("-inf"), l, 0.0)[:, None])
                    out[at, i * g:(i + 1) * g] = (w @ torch.cat(vals)).reshape(m, g, d)
                    lse[at, i * g:(i + 1) * g] = l.reshape(m, g)
    return out, lse


def exact_rope(case, seed):
    """Pairs as complex numbers, turned by amplitude e^{i angle}."""
    q, k, pos, wq, wk = rows_of(case, seed)
    turns = torch.remainder(pos.double()[:, None] * torch.from_numpy(frequencies(case) / (2 * math.pi)).to(DEV), 1.0)
    turn = torch.polar(torch.full_like(turns, amplitude(case)), turns * (2 * math.pi))[:, None]
    out = []
    for x, w in ((q, wq), (k, wk)):
        x = x.double()
        if case["norm"]:
            x = x / torch.sqrt(torch.linalg.vector_norm(x, dim=-1, keepdim=True) ** 2 / case["d"] + EPS) * w.double()
        y, half = x.clone(), case["rot"] // 2
        places = (slice(0, half), slice(half, 2 * half)) if case["halves"] else (slice(0, 2 * half, 2), slice(1, 2 * half, 2))
        z = torch.complex(x[..., places[0]].contiguous(), x[..., places[1]].contiguous()) * turn
        y[..., places[0]], y[..., places[1]] = z.real, z.imag
        out.append(y)
    return tuple(out)
