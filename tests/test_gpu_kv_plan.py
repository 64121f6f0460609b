"""Block tables and slots of a step's tokens (isoq_kv_plan) against the same
walk in Python integers: every output equal, every other byte as it was.  Needs
an MI355X."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

import paper_2603_28430_amd as iq  # noqa: E402


def walk(lens, new, table, bs, free, n_free, n_tokens):
    """The definition (include/isoquant.h), sequence by sequence; table and free are changed."""
    n, width = table.shape
    cap = width * bs
    old = [min(max(int(x), 0), cap) for x in lens]
    want = [min(max(int(x), 0), cap) for x in new]
    blocks = lambda x: -(-x // bs)   # noqa: E731
    top = min(max(int(n_free), 0), len(free))
    for s in range(n):
        for j in range(blocks(want[s]), blocks(old[s])):
            if top < len(free):
                free[top] = table[s, j]
                top += 1
    there = top
    taken = granted = 0
    out, q_start, tokens = [], [0], []
    for s in range(n):
        grow = max(0, blocks(want[s]) - blocks(old[s]))
        fine = grow == 0 or taken + grow <= there
        if fine:
            for i in range(grow):
                table[s, blocks(old[s]) + i] = free[there - 1 - taken - i]
            granted += grow
        taken += grow
        out.append(want[s] if fine else old[s])
        q_start.append(q_start[-1] + max(0, want[s] - old[s]))
        for p in range(old[s], want[s]):
            blk = table[s, p // bs] if fine else -1
            tokens.append((blk * bs + p % bs if blk >= 0 else -1, p))
    tokens = (tokens + [(-1, 0)] * n_tokens)[:n_tokens]
    return out, q_start, [t[0] for t in tokens], [t[1] for t in tokens], [there - granted]


def state(rng, old, width, bs, spare, max_free=None):
    """A table whose first blocks of each row are owned (canaries behind), and a free list of `spare` others."""
    have = -(-np.clip(old, 0, width * bs) // bs)
    perm = rng.permutation(int(have.sum()) + spare)
    table = np.full((len(old), width), -77)
    table[np.arange(width) < have[:, None]] = perm[:have.sum()]
    max_free = spare + int(have.sum()) if max_free is None else max_free
    free = np.full(max_free, -99)
    free[:min(spare, max_free)] = perm[have.sum():][:max_free]
    return table, free


def dev(x, dtype=np.int32):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(x).astype(dtype))).cuda()


def check(old, new, table, bs, free, n_free, n_tokens, **kw):
    """One call against the walk; returns the state after it."""
    args = dict(lens=dev(old), new_lens=dev(new), block_table=dev(table), block_size=bs, free_blocks=dev(free),
                n_free=dev([n_free]), n_tokens=n_tokens)
    got = iq.isoq_kv_plan(**args, **kw)
    table, free = table.copy(), free.copy()
    ref = walk(old, new, table, bs, free, n_free, n_tokens)
    for name, g, r in zip(("seq_lens", "q_start", "slot_mapping", "positions", "n_free"), got, ref):
        assert g.cpu().tolist() == list(r), name
    assert (args["block_table"].cpu().numpy() == table).all()
    assert (args["free_blocks"].cpu().numpy() == free).all()
    return ref, table, free


def mixed(rng, n, ctx, most=40):
    old = rng.integers(0, ctx, n)
    new = old + 1
    kind = rng.random(n)
    new = np.where(kind < 0.2, rng.integers(0, old + 1), new)
    new = np.where(kind < 0.1, 0, new)
    new = np.where(kind > 0.8, old + rng.integers(0, most, n), new)
    return old, np.minimum(new, ctx)


@pytest.mark.parametrize("n", [1, 2, 63, 64, 65, 1023, 1024, 1025, 2050, 7001])
@pytest.mark.parametrize("bs", [1, 13, 16])
def test_mixed_steps(n, bs):
    rng = np.random.default_rng(n * 31 + bs)
    ctx = 300 if n < 2000 else 60
    old, new = mixed(rng, n, ctx)
    table, free = state(rng, old, -(-ctx // bs), bs, n * (40 // bs + 2))
    total = int(np.maximum(new - old, 0).sum())
    check(old, new, table, bs, free, n * (40 // bs + 2), total + 3)


@pytest.mark.parametrize("lens", [[5000], [0, 4097, 1], [3, 20000, 9000, 1, 16], [4096] * 3])
def test_prompts(lens):
    """Long prompts: blocks by the hundred a sequence, tokens past what one workgroup writes, short sequences among them."""
    rng = np.random.default_rng(len(lens))
    old = np.array([0 if i % 2 == 0 else min(x, 7) for i, x in enumerate(lens)])
    table, free = state(rng, old, 1300, 16, 4000)
    total = int((np.array(lens) - old).sum())
    check(old, lens, table, 16, free, 4000, total)
    check(old, lens, table, 16, free, 4000, max(1, total - 5))   # fewer places than tokens
    check(lens, old, *state(rng, np.array(lens), 1300, 16, 3)[:1], 16, state(rng, np.array(lens), 1300, 16, 3)[1], 3, 4)


@pytest.mark.parametrize("spare", [0, 1, 2, 3, 5, 8, 20])
def test_too_few_blocks(spare):
    """Sequences are refused from the first on whose blocks are not there; those that need none are not."""
    rng = np.random.default_rng(spare)
    old = np.array([4, 8, 3, 16, 0, 9, 7, 12, 4])
    new = np.array([5, 13, 4, 17, 9, 2, 8, 13, 4])
    table, free = state(rng, old, 6, 4, spare, max_free=40)
    ref, _, _ = check(old, new, table, 4, free, spare, 30)
    assert ref[4][0] >= 0


def test_what_is_released_is_taken_in_the_same_step():
    rng = np.random.default_rng(3)
    old, new = np.array([48, 0, 16, 1]), np.array([0, 20, 3, 17])
    table, free = state(rng, old, 3, 16, 0)
    ref, after, _ = check(old, new, table, 16, free, 0, 40)
    assert ref[0] == [0, 20, 3, 17] and ref[4] == [0]
    assert set(after[1][:2]) | {after[3][1]} == set(table[0])


@pytest.mark.parametrize("bs", [4, 7])
def test_lengths_that_do_not_fit_the_table_and_short_lists(bs):
    rng = np.random.default_rng(bs)
    old = np.array([-5, 3, 10, 99, 2 ** 31 - 1, -2 ** 31, 0, 12])
    new = np.array([4, -3, 2 ** 31 - 1, 5, 2, 6, -1, 13])
    for max_free in (0, 1, 3, 6, 30):
        table, free = state(rng, old, 3, bs, 4, max_free=max_free)
        for n_free in (-3, 0, 2, 4, 100):   # (counts are cut to the list)
            check(old, new, table, bs, free, n_free, 50)


def test_no_sequences_no_tokens_no_table():
    none = np.zeros(0, np.int64)
    ref, _, _ = check(none, none, np.zeros((0, 4), np.int64), 16, np.arange(3), 3, 5)
    assert ref[1] == [0] and ref[2] == [-1] * 5 and ref[4] == [3]
    check(np.array([3, 5]), np.array([3, 4]), np.arange(4).reshape(2, 2), 4, np.zeros(4, np.int64), 0, 0)
    check(np.array([3, 5]), np.array([9, 4]), np.zeros((2, 0), np.int64), 4, np.zeros(0, np.int64), 0, 3)


def test_blocks_that_are_not_there_give_no_slot():
    table = np.array([[5, -1, -1], [-1, -1, -1]])
    check(np.array([3, 2]), np.array([6, 4]), table, 4, np.array([8, 9]), 2, 8)


@pytest.mark.parametrize("n_tokens", [6, 5000])
def test_graph_of_steps_in_place(n_tokens):
    """lens and n_free updated in place by a captured step, replayed, the new lengths given between the replays."""
    rng = np.random.default_rng(1)
    n, bs, width = 9, 4, 9
    old = rng.integers(0, 20, n)
    table, free = state(rng, old, width, bs, 30, max_free=n * width + 30)
    lens, new, tab, fr, n_free = dev(old), dev(old), dev(table), dev(free), dev([30])
    out = dict(slot_mapping=torch.empty(n_tokens, dtype=torch.int64, device="cuda"),
               positions=torch.empty(n_tokens, dtype=torch.int32, device="cuda"),
               q_start=torch.empty(n + 1, dtype=torch.int32, device="cuda"))

    def step():
        return iq.isoq_kv_plan(lens, new, tab, bs, fr, n_free, seq_lens=lens, n_free_out=n_free, **out)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()   # (nothing grows)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    assert got[0] is lens and got[4] is n_free
    spare = 30
    for k in range(6):
        want = np.clip(old + rng.integers(-3, 4, n), 0, width * bs)
        new.copy_(dev(want))
        graph.replay()
        torch.cuda.synchronize()
        ref = walk(old, want, table, bs, free, spare, n_tokens)
        for g, r in zip(got, ref):
            assert g.cpu().tolist() == list(r)
        assert (tab.cpu().numpy() == table).all() and (fr.cpu().numpy() == free).all()
        old, spare = np.array(ref[0]), ref[4][0]


def test_on_a_stream_of_its_own():
    rng = np.random.default_rng(5)
    old, new = mixed(rng, 100, 200)
    table, free = state(rng, old, 50, 4, 600)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    torch.cuda.synchronize()
    args = dev(old), dev(new), dev(table), 4, dev(free), dev([600])
    torch.cuda.synchronize()
    got = iq.isoq_kv_plan(*args, n_tokens=700, stream=stream)
    stream.synchronize()
    ref = walk(old, new, table, 4, free, 600, 700)
    for g, r in zip(got, ref):
        assert g.cpu().tolist() == list(r)
