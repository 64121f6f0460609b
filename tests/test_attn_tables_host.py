"""A handle does not pay for attention's tables before its first attention: the
host part of isoq_params_init at a tuned width (one search for the units of the
logits' digits: about 1.6 times a width without them at 2 bits) against a width
that has no tables.  With the searches for attention's tables it is 3.9 times.
Minima over many calls.  Runs on the CPU (without a GPU the call ends in an error
when the host part is done)."""
import time

import oracle
import paper_2603_28430_amd as iq


def host_us(d, levels):
    t = time.perf_counter()
    try:
        iq.isoq_params_init("full", d, 2, 1, codebook=levels)
    except iq.IsoqError:
        pass
    return time.perf_counter() - t


def test_init_leaves_out_attention_tables():
    best = {}
    for _ in range(400):
        for d in (120, 128):
            best[d] = min(best.get(d, 1.0), host_us(d, oracle.codebook(2, d)))
    assert best[128] <= 2.5 * best[120], best
