"""CPU checks of isoq_kv_plan, the rotary handle and isoq_qk_norm_rope: bad
arguments are refused before anything is launched, in the binding and in the
library, and the frequencies are those of the definition."""
import ctypes
import math

import numpy as np
import pytest
import torch

import paper_2603_28430_amd as iq
from paper_2603_28430_amd import isoquant as binding
from test_binding_checks import _raises

STEP = ("isoq_kv_plan", "isoq_qk_norm_rope")


class _NoLaunch:
    def __init__(self, real):
        self._real = real

    def __getattr__(self, name):
        if name in STEP:
            raise AssertionError("the library was reached with a bad argument")
        return getattr(self._real, name)


@pytest.fixture
def cpu_as_device(monkeypatch):
    monkeypatch.setattr(binding, "_is_gpu", lambda t: t.device.type == "cpu")
    monkeypatch.setattr(binding, "_on_current", lambda ref, ts, stream: binding._placed(ref, ts))
    monkeypatch.setattr(binding, "_stream_ptr", lambda stream: 0)
    monkeypatch.setattr(binding, "lib", _NoLaunch(binding.lib))


def plan_args():
    i = lambda *shape: torch.zeros(shape, dtype=torch.int32)   # noqa: E731
    return dict(lens=i(3), new_lens=i(3), block_table=i(3, 4), block_size=16, free_blocks=i(7), n_free=i(1), n_tokens=5)


def test_plan_tensor_checks(cpu_as_device):
    ok = plan_args()
    with pytest.raises(AssertionError, match="library was reached"):
        iq.isoq_kv_plan(**ok)
    for name in ("lens", "new_lens", "block_table", "free_blocks", "n_free"):
        t = ok[name]
        for bad in (t.long(), t.to("meta"), t[None] if t.dim() == 1 else t[0], torch.zeros((8, 2), dtype=torch.int32)[:, 0]):
            _raises(lambda: iq.isoq_kv_plan(**dict(ok, **{name: bad})))
    outs = dict(seq_lens=torch.zeros(3, dtype=torch.int32), q_start=torch.zeros(4, dtype=torch.int32),
                slot_mapping=torch.zeros(5, dtype=torch.int64), positions=torch.zeros(5, dtype=torch.int32),
                n_free_out=torch.zeros(1, dtype=torch.int32))
    for name, t in outs.items():
        for bad in (t.float(), t[:-1], t.to("meta"), t[None]):
            _raises(lambda: iq.isoq_kv_plan(**ok, **{name: bad}))
    _raises(lambda: iq.isoq_kv_plan(**{k: v for k, v in ok.items() if k != "n_tokens"}))


def test_plan_library_checks():
    buf = (ctypes.c_int64 * 64)()
    a = ctypes.addressof(buf)
    names = ("lens", "new_lens", "n_seqs", "table", "max_blocks", "block_size", "free", "max_free", "n_free", "seq_lens",
             "q_start", "slots", "positions", "n_tokens", "n_free_out", "stream")
    ok = dict(lens=a, new_lens=a + 32, n_seqs=1, table=a + 64, max_blocks=1, block_size=4, free=a + 96, max_free=1,
              n_free=a + 128, seq_lens=a + 160, q_start=a + 192, slots=a + 256, positions=a + 288, n_tokens=1,
              n_free_out=a + 320, stream=None)

    def status(**bad):
        return binding.lib.isoq_kv_plan(*[dict(ok, **bad)[n] for n in names])

    for bad in (dict(n_seqs=-1), dict(max_blocks=-1), dict(block_size=0), dict(max_free=-1), dict(n_tokens=-1),
                dict(seq_lens=ok["new_lens"])):
        assert status(**bad) == 1, bad
    for bad in (dict(n_seqs=65536), dict(max_blocks=2 ** 29), dict(block_size=2 ** 30, max_blocks=2), dict(max_free=2 ** 31),
                dict(n_tokens=2 ** 31), dict(block_size=2 ** 31 - 1, max_blocks=1)):
        assert status(**bad) == 2, bad
    for name in ("lens", "new_lens", "table", "free", "n_free", "seq_lens", "q_start", "slots", "positions", "n_free_out"):
        assert status(**{name: None}) == 3, name
        assert status(**{name: ok[name] + 2}) == 4, name
    assert status(slots=ok["slots"] + 4) == 4


def test_frequencies():
    for rot, base in ((2, 10000.0), (64, 10000.0), (128, 500000.0), (44, 1e6)):
        f = base ** (-2.0 * np.arange(rot // 2) / rot)
        assert np.allclose(iq.isoq_rope_freqs(rot, base), f, rtol=1e-15)
        assert np.allclose(iq.isoq_rope_freqs(rot, base, factor=8.0), f / 8, rtol=1e-15)   # every pair slowed
        keep = np.clip((f * 8192 / (2 * math.pi) - 1) / 31, 0, 1)
        got = iq.isoq_rope_freqs(rot, base, factor=8.0, original=8192, low=1.0, high=32.0)
        assert np.allclose(got, f * (keep + (1 - keep) / 8), rtol=1e-14)
    step = iq.isoq_rope_freqs(128, 1e4, factor=4.0, original=1000, low=2.0, high=2.0)   # no blending
    turns = 1e4 ** (-np.arange(64) / 64) * 1000 / (2 * math.pi)
    assert np.allclose(step, 1e4 ** (-np.arange(64) / 64) * np.where(turns > 2, 1, 0.25), rtol=1e-14)


def test_frequency_checks():
    for kw in (dict(rot_dim=0), dict(rot_dim=-2), dict(rot_dim=3), dict(rot_dim=8, base=0.0), dict(rot_dim=8, base=-2.0),
               dict(rot_dim=8, base=math.nan), dict(rot_dim=8, base=math.inf), dict(rot_dim=8, factor=0.0),
               dict(rot_dim=8, factor=math.nan), dict(rot_dim=8, factor=math.inf), dict(rot_dim=8, original=-1.0),
               dict(rot_dim=8, original=math.inf), dict(rot_dim=8, low=-1.0), dict(rot_dim=8, low=3.0, high=2.0),
               dict(rot_dim=8, high=math.inf), dict(rot_dim=8, low=math.nan)):
        with pytest.raises(iq.IsoqError, match="ISOQ_E_INVALID"):
            iq.isoq_rope_freqs(**kw)
    assert binding.lib.isoq_rope_freqs(8, 1e4, 1.0, 0.0, 1.0, 2.0, None) == 3


def test_rope_init_checks():
    for kw, status in ((dict(d=0), "INVALID"), (dict(d=64, rot_dim=66), "INVALID"), (dict(d=64, rot_dim=-2), "INVALID"),
                       (dict(d=64, rot_dim=31), "INVALID"), (dict(d=64, layout=2), "INVALID"),
                       (dict(d=64, amplitude=math.inf), "INVALID"), (dict(d=64, amplitude=math.nan), "INVALID"),
                       (dict(d=1026, rot_dim=64), "UNSUPPORTED"),
                       (dict(d=64, rot_dim=4, freqs=[1.0, math.inf]), "INVALID"), (dict(d=64, rot_dim=4, freqs=[math.nan, 1.0]), "INVALID")):
        with pytest.raises(iq.IsoqError, match="ISOQ_E_" + status):
            iq.isoq_rope_init(**kw)
    with pytest.raises(ValueError):
        iq.isoq_rope_init(64, 8, freqs=[1.0, 2.0])
    with pytest.raises(KeyError):
        iq.isoq_rope_init(64, layout="thirds")
    h = ctypes.c_void_p(5)
    assert binding.lib.isoq_rope_init(ctypes.byref(h), 64, 8, 0, None, 1.0) == 3 and not h
    assert binding.lib.isoq_rope_init(None, 64, 8, 0, None, 1.0) == 3
    assert binding.lib.isoq_rope_destroy(None) == 0


def rope(d=64):
    r = iq.Rope.__new__(iq.Rope)
    r.handle, r.d, r.rot_dim, r.layout = ctypes.c_void_p(None), d, d, 1
    return r


def test_norm_rope_tensor_checks(cpu_as_device):
    q, k = torch.zeros(5, 4, 64), torch.zeros(5, 2, 64)
    ok = dict(rope=rope(), q=q, k=k, positions=torch.zeros(5, dtype=torch.int32))
    w = torch.zeros(64)
    for more in ({}, dict(q_weight=w, k_weight=w), dict(k=None), dict(q_out=q, k_out=k)):
        with pytest.raises(AssertionError, match="library was reached"):
            iq.isoq_qk_norm_rope(**dict(ok, **more))
    bad = [dict(q=q[0]), dict(q=q[..., :32]), dict(q=q.bfloat16()), dict(q=q.half()), dict(q=q[:3]), dict(k=k[:, 0]),
           dict(k=k.half()), dict(k=k[:4]), dict(q=q.to("meta")), dict(k=k.to("meta")),
           dict(q=torch.zeros(4, 5, 64).transpose(0, 1)), dict(q=torch.zeros(5, 64, 4).transpose(1, 2)),
           dict(q=torch.zeros(1, 4, 64).expand(5, 4, 64)), dict(k=torch.zeros(5, 2, 128)[..., ::2]),
           dict(positions=ok["positions"].long()), dict(positions=ok["positions"][:4]), dict(positions=ok["positions"].to("meta")),
           dict(positions=torch.zeros(10, dtype=torch.int32)[::2]),
           dict(q_weight=w.half()), dict(q_weight=w[:32]), dict(k_weight=w.to("meta")), dict(k_weight=torch.zeros(128)[::2]),
           dict(q_out=q.half()), dict(q_out=k), dict(k_out=q), dict(q_out=torch.zeros(4, 5, 64).transpose(0, 1)),
           dict(k_out=k.to("meta")), dict(k=None, k_out=k), dict(k=None, k_weight=w)]
    for more in bad:
        _raises(lambda: iq.isoq_qk_norm_rope(**dict(ok, **more)))


def test_norm_rope_library_checks():
    assert binding.lib.isoq_qk_norm_rope(None, 0, None, 0, 0, None, 0, 0, None, 0, None, None, 1e-6, None, None, None) == 3
