"""What isoq_kv_attn_prefix launches, on the CPU (tests/hip_stub.py): every call that
the header allows has a kernel for each of its launches, in the workspace that it
asked for, over sizes on both sides of every choice of kernels, splits and forms."""
from hip_stub import run

# fp16 rows of several tokens behind prefixes that are attended to in a launch of their own: 32 rows a key head and
# more, own positions in one split and in several.  (variant, d, bits, tokens of each sequence, key heads, query heads
# of each, own positions, their bound max_len, prefixes' lengths, sequences of each or None); test_gpu_kv_attn_prefix_many.py
# runs them.
MANY = [
    ("full", 128, 3, [40, 1, 33], 2, 4, [128, 40, 33], 128, [150], None),
    ("full", 128, 3, [8, 8], 2, 4, [0, 0], 1, [150], None),
    ("fast", 64, 2, [32, 5, 0, 17], 2, 1, [64, 1, 30, 17], 64, [130], None),
    ("2d", 80, 4, [11, 24, 16], 1, 3, [100, 24, 1], 100, [257], None),
    ("fast", 96, 3, [150, 20], 2, 4, [128, 20], 128, [70], None),
    ("8d", 128, 4, [20, 33, 1], 2, 2, [128, 33, 60], 128, [200], None),
    ("2d", 64, 4, [64, 40, 3, 9], 2, 2, [64, 128, 3, 100], 128, [200, 0, 77], [2, 1, 1]),
    ("full", 96, 2, [9, 8, 12, 1, 7], 2, 4, [100, 8, 1, 70, 0], 100, [300, 33], [3, 1]),
    ("full", 80, 3, [33, 90], 1, 1, [300, 90], 300, [90], None),
    ("fast", 128, 2, [16] * 64, 8, 2, [400, 16, 0, 60] * 16, 400, [100], None),
    ("2d", 128, 3, [1] * 40, 1, 32, [100, 1, 0, 57] * 10, 100, [300], None),
    ("fast", 128, 4, [1] * 33, 1, 40, [300] + [12] * 32, 300, [300, 100], [20, 13]),
]
WIDE = 100000   # positions of the prefixes' table

CALLS = """
P = 1 << 20   # (an address that nothing reads)
handles = {}


def handle(variant, d, bits):
    key = variant, d, bits
    if key not in handles:
        handles[key] = iq.isoq_params_init(variant, d, bits)
    return handles[key].handle


def prefix(variant, d, bits, dtype, seqs, q_len, kv, group, own, pre, prefixes=1, bs=16, n_blocks=1000, most=None, n=None):
    h, n = handle(variant, d, bits), n or seqs * q_len
    sizes = [n, q_len, seqs, kv * group, kv]
    blocks, pre_blocks = -(-own // bs), -(-pre // bs)
    most = n if most is None else most
    need = lib.isoq_kv_attn_prefix_workspace(h, h, dtype, *sizes, bs, blocks, own, prefixes, most, pre_blocks, pre)
    st = lib.isoq_kv_attn_prefix(h, h, dtype, P, None if q_len == 1 else P, *sizes, P, P, P, P, n_blocks, bs, P, blocks, P,
                                 own, P, pre_blocks, P, pre, None if prefixes <= 1 else P, prefixes, most, 1.0, P, P, P,
                                 need, None)
    return st, launches()


"""


def test_many_rows_behind_a_prefix(tmp_path):
    """fp16 rows of several tokens, 32 a key head and more, whose own positions take one split."""
    run(tmp_path, CALLS + """
for seqs, q_len, kv, group, own, pre in [(8, 64, 8, 4, 64, 2048), (1, 128, 8, 4, 128, 32768), (16, 100, 8, 4, 100, 4096),
                                         (8, 256, 8, 4, 256, 4096), (64, 512, 8, 4, 512, 4096), (64, 5, 8, 8, 1000, 8192),
                                         (64, 16, 8, 4, 512, 8192), (64, 1, 1, 32, 512, 8192), (64, 16, 8, 4, 1500, 2000),
                                         (33, 16, 16, 2, 500, 20000), (2, 16, 8, 4, 128, 30000), (4, 8, 8, 4, 100, 30000)]:
    st, held = prefix("full", 128, 3, iq.ISOQ_F16, seqs, q_len, kv, group, own, pre)
    assert st == 0 and len(held) == 3, (seqs, q_len, kv, group, own, pre, st, len(held))
""")


def test_sizes_of_the_device_tests(tmp_path):
    """The prefixes' launch, that of the own positions, the join of both."""
    run(tmp_path, CALLS + f"""
for variant, d, bits, q_lens, kv, group, own, max_len, prefixes, counts in {MANY!r}:
    n = sum(q_lens) + (0 if max(q_lens) == 1 else 2)
    most = None if counts is None else max(sum(q_lens[sum(counts[:p]):sum(counts[:p + 1])]) for p in range(len(counts)))
    st, held = prefix(variant, d, bits, iq.ISOQ_F16, len(q_lens), max(q_lens), kv, group, max_len, {WIDE}, len(prefixes),
                      most=most, n=n)
    assert st == 0 and len(held) == 3, (variant, d, bits, q_lens, st, len(held))
""")


def test_sizes_of_the_serving_steps(tmp_path):
    """Those of test_gpu_step_run_shared.py: 7 sequences with at most 60 to 128 new tokens, 128 own positions, two prefixes."""
    run(tmp_path, CALLS + f"""
for variant, d, bits, bs, kv, group in (("full", 128, 3, 16, 2, 4), ("fast", 64, 4, 8, 1, 2), ("2d", 80, 2, 16, 2, 1), ("8d", 96, 3, 16, 1, 3)):
    for q_len, n in ((128, 234), (60, 140)):
        st, held = prefix(variant, d, bits, iq.ISOQ_F16, 7, q_len, kv, group, 128, {WIDE}, 2, bs, n=n)
        assert st == 0 and len(held) == 3, (variant, d, q_len, st, len(held))
""")


def test_every_size_has_its_kernels(tmp_path):
    run(tmp_path, CALLS + """
rng = random.Random(1)
some = lambda lo, hi: int(lo * (hi / lo) ** rng.random())
for k in range(6000):
    case = (rng.choice(["full", "fast", "2d", "8d"]), rng.choice([64, 80, 96, 128, 160, 192, 256, 512, 100, 7]), rng.choice([2, 3, 4]),
            rng.choice([iq.ISOQ_F16, iq.ISOQ_F16, iq.ISOQ_F32]), some(1, 600), rng.choice([1, 1, some(1, 700)]), some(1, 33), some(1, 70),
            rng.choice([0, 1, 128, 129, some(1, 9000)]), some(1, 140000), rng.choice([1, 1, 3, some(1, 300)]), rng.choice([1, 16, 17, 64]),
            rng.choice([1000, 1000, 1000, 0]))
    if case[4] * case[5] * case[6] * case[7] > 2 ** 23:
        continue
    st, held = prefix(*case, most=rng.choice([None, some(1, 300), 2 ** 40]))
    assert st == 0 and 1 <= len(held) <= 3, (case, st, len(held))
""")


def test_without_a_prefix_its_bounds_do_not_count(tmp_path):
    """No prefix, or none with positions: isoq_kv_attn's launches and workspace, for more tokens than a prefix may have."""
    run(tmp_path, CALLS + """
for variant, d, dtype in (("full", 128, iq.ISOQ_F16), ("fast", 100, iq.ISOQ_F32)):
    h, sizes = handle(variant, d, 3), (600 * 512, 512, 600, 32, 8)
    need = lib.isoq_kv_attn_workspace(h, h, dtype, *sizes, 16, 64, 1024)
    assert lib.isoq_kv_attn(h, h, dtype, P, P, *sizes, P, P, P, P, 1000, 16, P, 64, P, 1024, 1.0, P, P, P, need, None) == 0
    plain = [bytes(x) for x in launches()]
    for prefixes, blocks, length in ((0, 4, 64), (1, 0, 64), (1, 4, 0), (0, 0, 0), (1, 4, 64)):
        more = prefixes, sizes[0], blocks, length
        size = lib.isoq_kv_attn_prefix_workspace(h, h, dtype, *sizes, 16, 64, 1024, *more)
        st = lib.isoq_kv_attn_prefix(h, h, dtype, P, P, *sizes, P, P, P, P, 1000, 16, P, 64, P, 1024, P, blocks, P, length, P,
                                     prefixes, sizes[0], 1.0, P, P, P, need, None)
        held = [bytes(x) for x in launches()]
        if prefixes and blocks and length:   # (more rows than one prefix may have)
            assert st == 2 and not held and size == 0
        else:
            assert st == 0 and held == plain and size == need, (prefixes, blocks, length, st)
""")
