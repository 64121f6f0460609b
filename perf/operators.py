"""The operators on the paged quantized K/V cache, as calls whose speed and
exactness are tracked on one MI355X: attention over the cache (one new token a
sequence, or a chunk of new tokens), copies of cache blocks, and compaction of
sequences to the positions that are kept.

A cache slot of a key (or value) head holds rho and the b-bit indices of a
rotated row: x_hat = rho T^{-1} c[idx], T a block rotation of the head, c the
codebook.  Where `own` is false, run() computes an operator in its plain form,
elementary torch operations in 32 bits; where it is true it calls the package.
prepare() makes a case's inputs on the GPU from the seed alone; exact() is the
definition in 64 bits, from the indices rather than the packed records.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
F16, F32, F64 = torch.float16, torch.float32, torch.float64

_DEFAULTS = dict(variant="fast", d=128, bits=3, block_size=16)


def _case(name, op, **kw):
    c = dict(_DEFAULTS, op=op, **kw)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one user's decode step on a short context: latency
        _case("attn_one_short", "attn", dtype="f16", seqs=1, heads=8, group=4, ctx=700, q_len=1, ragged=False),
        # a serving batch of grouped-query heads, ragged contexts (an empty one among them), 4 bits
        _case("attn_gqa_ragged_b4", "attn", dtype="f16", seqs=16, heads=8, group=4, ctx=8192, q_len=1, ragged=True,
              bits=4, variant="full"),
        # the large cache of the logit benchmark, one query head per key head
        _case("attn_mha_long", "attn", dtype="f16", seqs=8, heads=32, group=1, ctx=32768, q_len=1, ragged=False),
        # one user's very long context, eight query heads per key head
        _case("attn_gqa8_longest", "attn", dtype="f16", seqs=1, heads=8, group=8, ctx=131071, q_len=1, ragged=False),
        # fp32 queries, a head width that is no power of two, odd group and block size
        _case("attn_f32_d96", "attn", dtype="f32", seqs=5, heads=4, group=5, ctx=3001, q_len=1, ragged=True, d=96,
              bits=2, variant="2d", block_size=17),
        # wide heads
        _case("attn_d256", "attn", dtype="f16", seqs=4, heads=8, group=2, ctx=8190, q_len=1, ragged=False, d=256),
        # drafted tokens checked against the cache: up to five new tokens a sequence
        _case("chunk_draft", "attn", dtype="f16", seqs=16, heads=8, group=4, ctx=4096, q_len=5, ragged=True),
        # chunks of prompts whose beginnings are in the cache already
        _case("chunk_prefill", "attn", dtype="f16", seqs=2, heads=8, group=4, ctx=8192, q_len=512, ragged=True),
        # a step's copy-on-write: the last block of each of 16 forked sequences
        _case("copy_fork", "copy", pairs=16, heads=8),
        # moving a large part of the cache to other blocks
        _case("copy_many", "copy", pairs=4096, heads=32),
        # eviction in one short sequence, one list for all heads
        _case("compact_short", "compact", seqs=1, heads=8, ctx=1000, keep=0.6, per_head=False),
        # eviction by head in a batch of long sequences
        _case("compact_long", "compact", seqs=8, heads=8, ctx=32768, keep=0.5, per_head=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attn", "attn", "attn", "chunk", "chunk", "copy", "compact"])
    kw = dict(variant=rng.choice(["full", "fast", "2d"]), bits=rng.choice([2, 3, 4]),
              d=rng.choice([64, 80, 96, 128, 128, 160, 192, 256]), block_size=rng.choice([16, 16, 32, 64, 13]))
    d = kw["d"]
    if op in ("attn", "chunk"):
        heads, group = rng.choice([(8, 1), (32, 1), (8, 4), (4, 8), (16, 2), (8, 5), (2, 16), (1, 12)])
        seqs = rng.choice([1, 2, 4, 8, 13])
        kw.update(heads=heads, group=group, seqs=seqs, ragged=rng.random() < 0.5,
                  dtype=rng.choice(["f16", "f16", "f32"]))
        if op == "attn":
            kw.update(q_len=1, ctx=_log_int(rng, 1, min(100000, 2 ** 29 // (heads * seqs * d))))
        else:
            q_len = _log_int(rng, 2, 300)
            top = min(2 ** 28 // (heads * seqs * d), 2 ** 28 // (heads * group * seqs * q_len))
            kw.update(q_len=q_len, ctx=_log_int(rng, 200, min(20000, top)))
        op = "attn"
    elif op == "copy":
        heads = rng.choice([1, 4, 8, 32])
        kw.update(heads=heads, pairs=_log_int(rng, 1, 2 ** 28 // (heads * d * kw["block_size"])))
    else:
        heads, seqs = rng.choice([1, 4, 8, 32]), rng.choice([1, 3, 8])
        kw.update(heads=heads, seqs=seqs, ctx=_log_int(rng, 2, min(60000, 2 ** 28 // (heads * seqs * d))),
                  keep=round(rng.uniform(0.05, 1.0), 2), per_head=rng.random() < 0.5)
    return _case(None, op, **kw)


# ---- inputs ------------------------------------------------------------------------

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
    return (case["d"] * case["bits"] + 7) // 8   # (every width here is a multiple of 16)


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
        unit = u / np.concatenate([np.repeat(np.linalg.norm(u[..., i:i + 4], axis=-1, keepdims=True), 4, -1)
                                   for i in range(0, u.shape[-1], 4)], -1)
        m = product(unit[..., :4], 1.0)
        if case["variant"] == "full":
            m = m @ product(unit[..., 4:] * np.array([1.0, -1.0, -1.0, -1.0]), -1.0)
    return torch.from_numpy(np.ascontiguousarray(m)).to(DEV)


def generator(seed, stream):
    return torch.Generator(device=DEV).manual_seed(int(seed) * 64 + stream)


def random_slots(case, blocks, seed, stream):
    """(indices [blocks, heads, block_size, d] uint8 as quantized rows have them, norms of the same slots)."""
    shape = (blocks, case["heads"], case["block_size"])
    count, base = math.prod(shape), 1 << 14
    g = generator(seed, stream)
    lev = codebook(case["bits"], 1)
    z = torch.randn((min(count, base), case["d"]), generator=g, device=DEV)
    idx = torch.bucketize(z, torch.tensor(0.5 * (lev[1:] + lev[:-1]), device=DEV, dtype=F32)).to(torch.uint8)
    if count > base:   # rows of the base, each rotated by a number of coordinates of its own
        pick = torch.randint(0, base, (count,), generator=g, device=DEV, dtype=torch.int32)
        idx = idx.repeat(1, 2).unfold(1, case["d"], 1)[:, :8].reshape(-1, case["d"])[
            pick * 8 + torch.randint(0, 8, (count,), generator=g, device=DEV, dtype=torch.int32)]
    rho = math.sqrt(case["d"]) * torch.exp(0.3 * torch.randn(shape, generator=g, device=DEV))
    return idx.reshape(shape + (case["d"],)), rho


def pack(idx, bits):
    """Records [..., d bits / 8] of indices [..., d], least significant bit first."""
    lead, d = idx.shape[:-1], idx.shape[-1]
    v = idx.reshape(-1, d // 8, 8).to(torch.int32)   # eight coordinates are `bits` bytes
    w = sum(v[..., i] << (bits * i) for i in range(8)) if bits < 4 else None
    if bits == 4:
        return (idx.reshape(lead + (d // 2, 2))[..., 0] | (idx.reshape(lead + (d // 2, 2))[..., 1] << 4)).contiguous()
    out = torch.stack([(w >> (8 * i)) & 255 for i in range(bits)], -1)
    return out.to(torch.uint8).reshape(lead + (d * bits // 8,))


def piece(r):
    return 16 if r % 16 == 0 else 8 if r % 8 == 0 else r


def piece_major(rec):
    """[blocks, heads, block_size, R] records as the cache holds them: pieces of
    16 or 8 bytes (where that divides R) of consecutive positions adjacent."""
    nb, h, bs, r = rec.shape
    p = piece(r)
    return rec.reshape(nb, h, bs, r // p, p).transpose(2, 3).contiguous().reshape(nb, h, bs, r)


def layout(case, seed):
    """(blocks in the cache, block table [seqs, blocks a sequence]), blocks placed at random, none shared."""
    per = -(-case["ctx"] // case["block_size"])
    blocks = case["seqs"] * per + 7
    perm = np.random.default_rng([seed, 19]).permutation(blocks)[:case["seqs"] * per]
    return blocks, perm.reshape(case["seqs"], per).astype(np.int32)


def lengths(case, seed):
    """(contexts, new tokens among them) of the sequences."""
    r = np.random.default_rng([seed, 17])
    n, ctx, q = case["seqs"], case["ctx"], case.get("q_len", 1)
    if not case.get("ragged"):
        return np.full(n, ctx), np.full(n, q)
    lens = r.integers(max(1, ctx // 4), ctx + 1, n)
    new = np.random.default_rng(q).integers(max(1, q // 2), q + 1, n)   # (as many rows for every seed)
    new[-1] = q
    if n >= 8:
        lens[1] = 0        # a slot of the batch without a sequence
    return lens, new


def kept(case, seed):
    """(positions that stay [seqs, heads or 1, most] ascending, how many of each sequence)."""
    n, ctx = case["seqs"], case["ctx"]
    most = max(1, int(case["keep"] * ctx))
    h = case["heads"] if case["per_head"] else 1
    order = torch.rand((n, h, ctx), generator=generator(seed, 31), device=DEV).topk(most, -1).indices
    count = np.random.default_rng([seed, 33]).integers(max(1, most // 2), most + 1, n)
    count[0] = most
    # a shorter list: the first `count` positions of the ascending ones
    return order.sort(-1).values.to(torch.int32).contiguous(), torch.from_numpy(count.astype(np.int32)).to(DEV)


def block_pairs(case, seed):
    perm = np.random.default_rng([seed, 35]).permutation(2 * case["pairs"] + 9)[:2 * case["pairs"]]
    return torch.from_numpy(perm.reshape(-1, 2).astype(np.int32)).to(DEV)


def queries(case, total, seed):
    """Query rows [tokens, query heads, d]: Gaussian, a few channels larger than the rest."""
    g = generator(seed, 3)
    q = 1.5 * torch.randn((total, case["heads"] * case["group"], case["d"]), generator=g, device=DEV)
    q[..., torch.randint(0, case["d"], (3,), generator=g, device=DEV)] *= 2.0
    return q.to(F16 if case["dtype"] == "f16" else F32)


def handles(case, seed):
    import paper_2603_28430_amd as iq

    return [iq.isoq_params_init(case["variant"], case["d"], case["bits"], case["heads"], rot=draws(case, s).reshape(-1),
                                codebook=codebook(case["bits"], case["d"])) for s in (seed, seed + 1000003)]


def prepare(case, seed):
    s = dict(case=case)
    if case["op"] == "copy":
        blocks = 2 * case["pairs"] + 9
        s["pairs"] = block_pairs(case, seed)
    else:
        blocks, table = layout(case, seed)
        s["table"] = torch.from_numpy(table).to(DEV)
    for name, stream in (("k", 22), ("v", 24)):
        idx, rho = random_slots(case, blocks, seed, stream)
        s[name + "_idx"], s[name + "_rho"] = piece_major(pack(idx, case["bits"])), rho
        del idx
    if own:   # the quantizers' handles, which a program builds once
        s["pk"], s["pv"] = handles(case, seed)
    if case["op"] == "compact":
        s["keep"], s["n_keep"] = kept(case, seed)
    if case["op"] == "attn":
        lens, new = lengths(case, seed)
        s["lens"] = torch.from_numpy(lens.astype(np.int32)).to(DEV)
        s["q"] = queries(case, int(new.sum()), seed)
        s["scale"] = 1.0 / math.sqrt(case["d"])
        s["start"] = None
        if case["q_len"] > 1:
            s["start"] = torch.from_numpy(np.concatenate([[0], np.cumsum(new)]).astype(np.int32)).to(DEV)
        # the rotations and levels that the plain form works with
        s["lev"] = torch.from_numpy(codebook(case["bits"], case["d"])).to(DEV, F32)
        s["mk"], s["mv"] = matrices(case, seed).to(F32), matrices(case, seed + 1000003).to(F32)
    return s


# ---- one pass ------------------------------------------------------------------------

def run(s):
    op = s["case"]["op"]
    if own:
        import paper_2603_28430_amd as iq

        if op == "attn":
            return iq.isoq_kv_attn(s["pk"], s["q"], s["k_idx"], s["k_rho"], s["pv"], s["v_idx"], s["v_rho"], s["table"],
                                   s["lens"], scale=s["scale"], q_start=s["start"], max_q_len=s["case"]["q_len"])
        if op == "copy":
            iq.isoq_kv_copy_blocks(s["pk"], s["pairs"], s["k_idx"], s["k_rho"], s["v_idx"], s["v_rho"])
        else:
            iq.isoq_kv_compact(s["pk"], s["keep"], s["n_keep"], s["table"], s["k_idx"], s["k_rho"], s["v_idx"],
                               s["v_rho"])
        return s["k_idx"], s["k_rho"], s["v_idx"], s["v_rho"]
    if op == "attn":
        return plain_attn(s)
    return plain_copy(s) if op == "copy" else plain_compact(s)


def paged(cache, table):
    """[seqs, heads, positions, R] records of a piece-major cache through a block table."""
    nb, h, bs, r = cache.shape
    p = piece(r)
    c = cache.reshape(nb, h, r // p, bs, p)[table]                     # [seqs, blocks, heads, pieces, bs, p]
    return c.permute(0, 2, 1, 4, 3, 5).reshape(table.shape[0], h, -1, r)


def levels_of(s, cache):
    """c[idx] of every position of every sequence: [seqs, heads, positions, d]."""
    bits = s["case"]["bits"]
    rec = paged(cache, s["table"])
    b = (rec.unsqueeze(-1) >> torch.arange(8, device=DEV, dtype=torch.uint8)) & 1
    b = b.reshape(rec.shape[:-1] + (-1, bits))
    idx = (b << torch.arange(bits, device=DEV, dtype=torch.uint8)).sum(-1, dtype=torch.int32)
    return s["lev"][idx]


def norms_of(s, rho):
    return rho[s["table"]].transpose(1, 2).reshape(s["table"].shape[0], rho.shape[1], -1)


def block_product(m, x):
    """Block matrices m [heads, 1.., blocks, k, k] times rows x [..., d]."""
    k = m.shape[-1]
    x = x.reshape(x.shape[:-1] + (-1, k))
    return (m * x.unsqueeze(-2)).sum(-1).flatten(-2)


def plain_attn(s):
    case = s["case"]
    n, h, g, d = case["seqs"], case["heads"], case["group"], case["d"]
    total = s["q"].shape[0]
    start = s["start"] if s["start"] is not None else torch.arange(n + 1, device=DEV, dtype=torch.int32)
    new = start[1:] - start[:-1]
    i = torch.arange(case["q_len"], device=DEV, dtype=torch.int32)
    row = (start[:-1, None] + i).clamp(max=total - 1)                   # [seqs, q_len] token of each place
    limit = torch.where(i < new[:, None], s["lens"][:, None] - (new[:, None] - 1 - i), 0)
    q = s["q"][row].float().reshape(n, -1, h, g, d).permute(0, 2, 1, 3, 4)   # [seqs, heads, q_len, group, d]
    q = block_product(s["mk"][:, None, None], q * s["scale"]).flatten(2, 3)
    logits = q @ levels_of(s, s["k_idx"]).transpose(-1, -2) * norms_of(s, s["k_rho"]).unsqueeze(-2)
    t = torch.arange(logits.shape[-1], device=DEV, dtype=torch.int32)
    limit = limit.repeat_interleave(g, 1)[:, None, :, None]              # [seqs, 1, rows, 1]
    logits = torch.where(t < limit, logits, float("-inf"))
    top = logits.amax(-1, keepdim=True)
    top = torch.where(limit > 0, top, 0.0)
    p = torch.exp(logits - top)
    total_p = p.sum(-1, keepdim=True)
    o = (p * norms_of(s, s["v_rho"]).unsqueeze(-2)) @ levels_of(s, s["v_idx"])
    o = torch.where(limit > 0, o / total_p, 0.0)
    lse = torch.where(limit > 0, top + torch.log(total_p), float("-inf"))
    o = block_product(s["mv"].transpose(-1, -2)[:, None], o)
    valid = i < new[:, None]
    o = o.reshape(n, h, -1, g, d).permute(0, 2, 1, 3, 4).reshape(n, -1, h * g, d)[valid]
    lse = lse.reshape(n, h, -1, g).permute(0, 2, 1, 3).reshape(n, -1, h * g)[valid]
    return o.to(s["q"].dtype), lse


def plain_copy(s):
    src, dst = s["pairs"].long().unbind(1)
    s["k_idx"][dst] = s["k_idx"][src]
    s["k_rho"][dst] = s["k_rho"][src]
    s["v_idx"][dst] = s["v_idx"][src]
    s["v_rho"][dst] = s["v_rho"][src]
    return s["k_idx"], s["k_rho"], s["v_idx"], s["v_rho"]


def plain_compact(s):
    keep, bs = s["keep"].long(), s["case"]["block_size"]
    h = s["case"]["heads"]
    keep = keep.expand(-1, h, -1)
    n, _, most = keep.shape
    to = torch.arange(most, device=DEV).expand(n, h, most)
    ok = to < s["n_keep"][:, None, None]
    seq = torch.arange(n, device=DEV)[:, None, None].expand(n, h, most)[ok]
    head = torch.arange(h, device=DEV)[:, None].expand(n, h, most)[ok]
    keep, to = keep[ok], to[ok]
    table = s["table"].long()
    a, b = (table[seq, keep // bs], head, keep % bs), (table[seq, to // bs], head, to % bs)
    return (move_records(s["k_idx"], a, b), move_norms(s["k_rho"], a, b), move_records(s["v_idx"], a, b),
            move_norms(s["v_rho"], a, b))


def move_records(cache, a, b):
    nb, h, bs, r = cache.shape
    c = cache.view(nb, h, r // piece(r), bs, piece(r)).transpose(2, 3)   # [block, head, position, pieces, bytes]
    c[b] = c[a]
    return cache


def move_norms(rho, a, b):
    rho[b] = rho[a]
    return rho


# ---- what a pass cannot do without, and the same in 64 bits -----------------------------

def work(case):
    r, h, bs = record_bytes(case), case["heads"], case["block_size"]
    if case["op"] == "copy":
        moved = case["pairs"] * h * bs * 2 * (r + 4)
        return dict(bytes=2 * moved + 8 * case["pairs"], flops=0)
    if case["op"] == "compact":
        # kept positions (three quarters of the longest list in the mean, the first sequence all of it)
        most = max(1, int(case["keep"] * case["ctx"]))
        n = (1 + 0.75 * (case["seqs"] - 1)) * most
        return dict(bytes=n * h * 4 * (r + 4) + 4 * n * (h if case["per_head"] else 1), flops=0)
    frac, new = (0.625, 0.75 * case["q_len"]) if case["ragged"] else (1.0, case["q_len"])
    seqs = case["seqs"] - (1 if case["ragged"] and case["seqs"] >= 8 else 0)
    keys = frac * seqs * case["ctx"]
    rows = max(1.0, new) * case["seqs"] * h * case["group"]
    es = 2 if case["dtype"] == "f16" else 4
    return dict(bytes=keys * h * 2 * (r + 4) + rows * (2 * case["d"] * es + 4) + keys / bs * 4,
                flops=keys * h * case["group"] * max(1.0, new) * 4 * case["d"])


def exact(case, seed):
    h, bs, d = case["heads"], case["block_size"], case["d"]
    blocks = 2 * case["pairs"] + 9 if case["op"] == "copy" else layout(case, seed)[0]
    (ki, kr), (vi, vr) = random_slots(case, blocks, seed, 22), random_slots(case, blocks, seed, 24)
    if case["op"] == "copy":
        out = []
        for src, dst in [block_pairs(case, seed).long().unbind(1)]:
            for idx, rho in ((ki, kr), (vi, vr)):
                rho = rho.double()
                rho.index_copy_(0, dst, rho.index_select(0, src))
                out += [None, rho]
        return tuple(out)
    table = torch.from_numpy(layout(case, seed)[1].astype(np.int64)).to(DEV)
    if case["op"] == "compact":
        keep, n_keep = kept(case, seed)
        out = []
        for rho in (kr, vr):
            new = rho.double()
            for s in range(case["seqs"]):
                n = int(n_keep[s])
                flat = rho[table[s]].double().transpose(0, 1).reshape(h, -1)   # [heads, positions]
                flat[:, :n] = flat.gather(1, keep[s, :, :n].long().expand(h, n)).clone()
                new[table[s]] = flat.reshape(h, -1, bs).transpose(0, 1)
            out += [None, new]
        return tuple(out)
    lens, new = lengths(case, seed)
    lev = torch.from_numpy(codebook(case["bits"], d)).to(DEV)
    rot = [matrices(case, seed), matrices(case, seed + 1000003)]
    q = queries(case, int(new.sum()), seed).double()
    out = torch.zeros(q.shape, device=DEV, dtype=F64)
    lse = torch.full(q.shape[:2], float("-inf"), device=DEV, dtype=F64)
    g, at = case["group"], 0
    for s in range(case["seqs"]):
        n, length = int(new[s]), int(lens[s])
        if length > 0:
            t = torch.arange(length, device=DEV)
            blk, pos = table[s][t // bs], t % bs
            mask = t[None] <= length - n + torch.arange(n, device=DEV)[:, None]    # [new, positions]
            some = mask.any(1)
            for i in range(h):
                rows = []
                for idx, rho, m in ((ki, kr, rot[0][i]), (vi, vr, rot[1][i])):
                    # the row itself: the levels rotated back, times the norm
                    c = lev[idx[blk, i, pos].long()].reshape(length, -1, m.shape[-1])
                    x = sum(c[..., j, None] * m[:, j] for j in range(m.shape[-1])).reshape(length, d)
                    rows.append(x * rho[blk, i, pos].double()[:, None])
                for j in range(0, n, 64):
                    part = q[at + j:at + min(n, j + 64), i * g:(i + 1) * g]
                    a = part.reshape(-1, d) @ rows[0].t().contiguous() / math.sqrt(d)
                    a = a.reshape(part.shape[0], g, length).masked_fill(~mask[j:j + 64, None], float("-inf"))
                    l = torch.logsumexp(a, -1)
                    p = torch.exp(a - torch.where(some[j:j + 64, None], l, 0.0)[..., None])
                    out[at + j:at + j + part.shape[0], i * g:(i + 1) * g] = (p.reshape(-1, length) @ rows[1]).reshape(part.shape)
                    lse[at + j:at + j + part.shape[0], i * g:(i + 1) * g] = l
        at += n
    return out, lse
