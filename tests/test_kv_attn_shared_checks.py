"""CPU checks of the arguments of isoq_kv_attn_prefix and isoq_kv_attn_cross in the
binding and of null handles in the library: a bad argument is refused before
anything is launched."""
import pytest
import torch

import paper_2603_28430_amd as iq
from paper_2603_28430_amd import isoquant as binding
from test_binding_checks import _raises
from test_kv_attn_checks import good

CALLS = ("isoq_kv_attn", "isoq_kv_attn_cross", "isoq_kv_attn_prefix")


class _NoLaunch:
    def __init__(self, real):
        self._real = real

    def __getattr__(self, name):
        if name in CALLS:
            raise AssertionError(f"the library was reached: {name}")
        return getattr(self._real, name)


@pytest.fixture
def cpu_as_device(monkeypatch):
    monkeypatch.setattr(binding, "_is_gpu", lambda t: t.device.type == "cpu")
    monkeypatch.setattr(binding, "_on_current", lambda ref, ts, stream: binding._placed(ref, ts))
    monkeypatch.setattr(binding, "_stream_ptr", lambda stream: 0)
    monkeypatch.setattr(binding, "lib", _NoLaunch(binding.lib))


def prefixed():
    return dict(good(), prefix_table=torch.zeros((2, 3), dtype=torch.int32), prefix_lens=torch.zeros(2, dtype=torch.int32),
                prefix_start=torch.tensor([0, 1, 3], dtype=torch.int32))


def reaches(fn, name):
    with pytest.raises(AssertionError, match=f"reached: {name}$"):
        fn()


def test_good_calls_reach_the_library(cpu_as_device):
    ok = prefixed()
    reaches(lambda: iq.isoq_kv_attn_prefix(**ok), "isoq_kv_attn_prefix")
    one = dict(ok, prefix_table=ok["prefix_table"][:1], prefix_lens=ok["prefix_lens"][:1])
    one.pop("prefix_start")
    reaches(lambda: iq.isoq_kv_attn_prefix(**one), "isoq_kv_attn_prefix")
    reaches(lambda: iq.isoq_kv_attn_cross(**good()), "isoq_kv_attn_cross")
    reaches(lambda: iq.isoq_kv_attn(**good()), "isoq_kv_attn")


def test_prefix_tensor_checks(cpu_as_device):
    ok = prefixed()
    table, lens, start = ok["prefix_table"], ok["prefix_lens"], ok["prefix_start"]
    bad = [("prefix_table", table.to("meta")), ("prefix_table", table.long()), ("prefix_table", table[0]),
           ("prefix_table", table[:1]), ("prefix_table", torch.zeros((3, 2), dtype=torch.int32).t()),
           ("prefix_lens", lens.to("meta")), ("prefix_lens", lens.long()), ("prefix_lens", lens[:1]), ("prefix_lens", lens[None]),
           ("prefix_lens", torch.zeros(4, dtype=torch.int32)[::2]),
           ("prefix_start", start.to("meta")), ("prefix_start", start.long()), ("prefix_start", start[:2]),
           ("prefix_start", start[None]), ("prefix_start", None), ("prefix_start", torch.zeros(6, dtype=torch.int32)[::2]),
           ("q", ok["q"][0]), ("q", ok["q"].bfloat16()), ("k_idx", ok["k_idx"][0]), ("workspace", torch.zeros(4)),
           ("workspace", torch.zeros(4, dtype=torch.uint8, device="meta"))]
    for name, t in bad:
        _raises(lambda: iq.isoq_kv_attn_prefix(**dict(ok, **{name: t})))


def test_cross_tensor_checks(cpu_as_device):
    ok = good()
    for name, t in (("q", ok["q"][..., :64]), ("q", ok["q"][:2]), ("block_table", ok["block_table"].long()),
                    ("seq_lens", ok["seq_lens"][:2]), ("k_idx", ok["k_idx"][:1]), ("v_rho", ok["v_rho"].double()),
                    ("max_q_len", 2), ("q_start", torch.zeros(3, dtype=torch.int32))):
        _raises(lambda: iq.isoq_kv_attn_cross(**dict(ok, **{name: t})))


def test_null_handles():
    lib = binding.lib
    assert lib.isoq_kv_attn_cross(*[None if t is binding.ctypes.c_void_p else 0 for t in lib.isoq_kv_attn_cross.argtypes]) == 3
    assert lib.isoq_kv_attn_prefix(*[None if t is binding.ctypes.c_void_p else 0 for t in lib.isoq_kv_attn_prefix.argtypes]) == 3
    assert lib.isoq_kv_attn_prefix_workspace(*[None if t is binding.ctypes.c_void_p else 1
                                               for t in lib.isoq_kv_attn_prefix_workspace.argtypes]) == 0
