"""What isoq_qk_norm_rope launches, on the CPU (tests/hip_stub.py): calls up to the
header's limits in launches that the device takes (fewer than 2^32 threads each), with a wave
for every row, or every token's rows."""
from hip_stub import run

CALLS = """
P = 1 << 20   # (an address that nothing reads)
ropes = {}


def waves(d, rot, layout, dtype, n_tokens, q_heads, kv_heads):
    key = d, rot, layout
    if key not in ropes:
        ropes[key] = iq.isoq_rope_init(*key)
    st = lib.isoq_qk_norm_rope(ropes[key].handle, dtype, P, q_heads * d, q_heads, P, kv_heads * d, kv_heads, P, n_tokens,
                               None, None, 1e-6, P, P, None)
    held = launches()
    return st, sum(x.grid[0] * x.block[0] // 64 for x in held), len(held)


"""


def test_largest_calls(tmp_path):
    run(tmp_path, CALLS + """
for shape, rows in (((128, 128, "halves"), False), ((64, 24, "pairs"), False), ((3, 2, "pairs"), True), ((1, 0, "pairs"), True)):
    for dtype in (iq.ISOQ_F16, iq.ISOQ_F32):
        for n, hq, hk in ((2 ** 26 - 4, 1, 0), (2 ** 26 - 3, 1, 0), (2 ** 26 + 1, 1, 0), (2 ** 20, 60, 4), (2 ** 20 + 1, 60, 4),
                          (2 ** 31 - 1, 1, 0), (2 ** 30 - 1, 1, 1), (50000000, 32, 8), (16383, 65535, 65535), (1, 65535, 65535), (7, 0, 3)):
            st, w, k = waves(*shape, dtype, n, hq, hk)
            if n * (hq + hk) > 2 ** 31 - 1:
                assert st == 2 and k == 0
                continue
            least = n * (hq + hk) if rows else n
            assert st == 0 and least <= w, (shape, n, hq, hk, st, w)
            if rows:   # (no more than whole workgroups in each launch)
                assert w < least + 4 * k
""")
