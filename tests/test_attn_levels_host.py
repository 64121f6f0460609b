"""The codebook's forms for attention, summed as the kernels sum them.

Digits (build_value_digits): integers of the largest magnitude 32,639 (two
digits) or 8,355,711 (three) in units of at most twice the largest level over
that, so a level is off by half a unit, 1 / 32,639 or 1 / 8,355,711 of the
largest one at most (and by 2^-24 of itself: the unit is a float).
fp16 (build_half_levels): off by half a step, 2^-11 of a level, at most; the unit
is chosen among 4,096 for a small error of all levels, of which the reported one
is the largest.  With what that leaves in e4m3, whose half step is 2^-4 of it (and
2^-10 of the unit 2^-19 where it is small): 2^-15 of the level and 2^-29 of the
largest.  In e4m3 alone: 2^-4 of a level, and 2^-10 of the largest.  A level's mirror
image is its negative in all of them.
Runs on the CPU."""
import os
import shutil
import subprocess

import numpy as np
import pytest

import oracle

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2603_28430_amd", "csrc")


def test_attn_levels(tmp_path):
    cxx = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "llvm", "bin", "clang++")
    if not os.path.exists(cxx) and (cxx := shutil.which("clang++")) is None:
        pytest.skip("no clang++")
    exe = tmp_path / "attn_levels_check"
    subprocess.run([cxx, "-O2", "-std=c++17", f"-I{CSRC}", os.path.join(HERE, "native", "attn_levels_check.cpp"),
                    os.path.join(CSRC, "isoq_host_params.cpp"), "-o", str(exe)], check=True, capture_output=True,
                   text=True)
    books = [(b, oracle.codebook(b, d), True) for b in (2, 3, 4) for d in (64, 80, 96, 128, 160, 192, 256, 512)]
    rng = np.random.default_rng(0)
    for b in (2, 3, 4):
        for _ in range(6):
            pos = np.sort(rng.uniform(0.02, 1.0, 1 << (b - 1)))
            books.append((b, np.concatenate([-pos[::-1], pos]) * 10.0 ** rng.uniform(-3, 3), False))
    books += [(b, c * scale, lloyd) for b, c, lloyd in books[::5] for scale in (2.0 ** -80, 2.0 ** 80)]
    books += [(b, c * 1e-60, False) for b, c, _ in books[:24:8]]   # (zero as floats)
    text = "".join("%d %s\n" % (b, " ".join("%.9g" % np.float32(v) for v in c)) for b, c, _ in books)
    out = subprocess.run([str(exe)], input=text, capture_output=True, text=True, check=True, timeout=60).stdout
    lines = [np.array(line.split(), float) for line in out.strip().splitlines()]
    assert len(lines) == 5 * len(books)
    for i, (b, c, lloyd) in enumerate(books):
        ref = np.float32(c).astype(float)
        top = ref[-1]
        two, three, half, rest, byte = lines[5 * i:5 * i + 5]
        off, half = half[0], half[1:]
        for vals, units in ((two, 32639), (three, 8355711)):
            assert np.all(np.abs(vals - ref) <= top / units + 2.0 ** -24 * np.abs(ref)), (b, units)
        left = np.abs(half - ref)
        scale = 2.0 ** -23 * np.abs(ref)   # (the unit is a float, and so are the levels)
        assert np.all(left <= off * np.abs(ref) + scale) and off <= 2.0 ** -11, (b, off)
        assert np.all(np.abs(rest - ref) <= 2.0 ** -4 * left + 2.0 ** -29 * top + scale), b
        assert np.all(np.abs(byte - ref) <= 2.0 ** -4 * np.abs(ref) + 2.0 ** -10 * top + scale), b
        if lloyd:
            # of the levels' root mean square under equal weights: what the kernel's comment states
            rms = np.sqrt(np.mean(left ** 2) / np.mean(ref ** 2))
            assert rms <= {2: 4e-7, 3: 1.6e-5, 4: 1e-4}[b], (b, rms)
            assert b > 2 or off <= 2.0 ** -20
        for v in (two, three, half, rest, byte):
            assert np.array_equal(v, -v[::-1])
