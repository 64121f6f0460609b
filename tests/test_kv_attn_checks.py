"""CPU checks of the arguments of isoq_kv_attn in the binding and of null
handles in the library: a bad argument is refused before anything is launched
(the stand-ins are those of test_binding_checks.py)."""
import pytest
import torch

import paper_2603_28430_amd as iq
from paper_2603_28430_amd import isoquant as binding
from test_binding_checks import _params, _raises


class _NoLaunch:
    def __init__(self, real):
        self._real = real

    def __getattr__(self, name):
        if name == "isoq_kv_attn":
            raise AssertionError("the library was reached with a bad argument")
        return getattr(self._real, name)


@pytest.fixture
def cpu_as_device(monkeypatch):
    monkeypatch.setattr(binding, "_is_gpu", lambda t: t.device.type == "cpu")
    monkeypatch.setattr(binding, "lib", _NoLaunch(binding.lib))


def good():
    p = _params()
    cache = torch.zeros((2, 2, 16, p.record_bytes), dtype=torch.uint8)
    rho = torch.zeros((2, 2, 16))
    return dict(pk=p, pv=p, q=torch.zeros((3, 4, 128), dtype=torch.float16), k_idx=cache, k_rho=rho,
                v_idx=cache.clone(), v_rho=rho.clone(), block_table=torch.zeros((3, 2), dtype=torch.int32),
                seq_lens=torch.zeros(3, dtype=torch.int32))


def test_attn_tensor_checks(cpu_as_device):
    ok = good()
    q, cache, rho, table, lens = ok["q"], ok["k_idx"], ok["k_rho"], ok["block_table"], ok["seq_lens"]
    bad = [("q", q.to("meta")), ("q", q[..., :64]), ("q", q.to(torch.bfloat16)), ("q", q[:2]), ("q", q[0]),
           ("q", torch.zeros((4, 3, 128), dtype=torch.float16).transpose(0, 1)),
           ("block_table", table.to("meta")), ("block_table", table.long()), ("block_table", table[:2]),
           ("block_table", torch.zeros((2, 3), dtype=torch.int32).t()),
           ("seq_lens", lens.to("meta")), ("seq_lens", lens.long()), ("seq_lens", lens[:2]), ("seq_lens", lens[None])]
    for k in ("k", "v"):
        bad += [(k + "_idx", cache.to("meta")), (k + "_idx", cache[..., :40]), (k + "_idx", cache[:1]),
                (k + "_idx", cache.to(torch.int8)), (k + "_idx", cache[:, :, ::2]),
                (k + "_rho", rho.to("meta")), (k + "_rho", rho[:, :, :8]), (k + "_rho", rho.double()),
                (k + "_rho", torch.zeros((2, 16, 2)).transpose(1, 2))]
    for name, t in bad:
        _raises(lambda: iq.isoq_kv_attn(**dict(ok, **{name: t})))


def test_attn_token_checks(cpu_as_device):
    ok = good()
    start = torch.tensor([0, 1, 2, 3], dtype=torch.int32)
    for more in (dict(max_q_len=2), dict(q_start=start[:3]), dict(q_start=start.long()), dict(q_start=start[None]),
                 dict(q_start=start.to("meta")), dict(q_start=torch.zeros(8, dtype=torch.int32)[::2])):
        _raises(lambda: iq.isoq_kv_attn(**ok, **more))


def test_attn_output_checks(cpu_as_device):
    ok = good()
    out, lse = torch.zeros_like(ok["q"]), torch.zeros((3, 4))
    ws = torch.zeros(64, dtype=torch.uint8)
    for more in (dict(out=out.float()), dict(out=out[:2]), dict(out=out.to("meta")), dict(lse=lse.half()),
                 dict(lse=lse[:, :3]), dict(lse=lse.to("meta")), dict(lse=torch.zeros((4, 3)).t()),
                 dict(workspace=ws.float()), dict(workspace=ws.to("meta")), dict(workspace=ws[::2])):
        _raises(lambda: iq.isoq_kv_attn(**ok, **more))


def test_attn_null_handles():
    assert binding.lib.isoq_kv_attn(None, None, 1, None, None, 1, 1, 1, 1, 1, None, None, None, None, 1, 16, None, 1,
                                    None, 16, 1.0, None, None, None, 0, None) == 3
    assert binding.lib.isoq_kv_attn_workspace(None, None, 1, 1, 1, 1, 1, 1, 16, 1, 16) == 0


class _NoPages(_NoLaunch):
    def __getattr__(self, name):
        if name in ("isoq_kv_copy_blocks", "isoq_kv_compact"):
            raise AssertionError("the library was reached with a bad argument")
        return getattr(self._real, name)


def test_page_call_checks(monkeypatch):
    monkeypatch.setattr(binding, "_is_gpu", lambda t: t.device.type == "cpu")
    monkeypatch.setattr(binding, "lib", _NoPages(binding.lib))
    ok = good()
    sk = iq.Sketch(0, ok["pk"], 64)
    planes = {k: ok[k] for k in ("k_idx", "k_rho", "v_idx", "v_rho")}
    signs, gamma = torch.zeros((2, 2, 16, 8), dtype=torch.uint8), torch.zeros((2, 2, 16))
    pairs = torch.zeros((3, 2), dtype=torch.int32)
    keep, n_keep = torch.zeros((3, 1, 5), dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    table = ok["block_table"]
    cache, rho = planes["k_idx"], planes["k_rho"]
    bad = [dict(v_idx=None), dict(v_rho=None), dict(sketch=sk), dict(sketch=sk, k_signs=signs), dict(k_signs=signs),
           dict(sketch=sk, k_signs=signs[..., :4], k_gamma=gamma), dict(sketch=sk, k_signs=signs.int(), k_gamma=gamma),
           dict(sketch=sk, k_signs=signs, k_gamma=gamma.half()), dict(sketch=sk, k_signs=signs, k_gamma=gamma[:1])]
    for k in ("k", "v"):
        bad += [{k + "_idx": x} for x in (cache.to("meta"), cache[..., :40], cache[:1], cache.to(torch.int8), cache[:, :, ::2])]
        bad += [{k + "_rho": x} for x in (rho.to("meta"), rho[:, :, :8], rho.double(), torch.zeros((2, 16, 2)).transpose(1, 2))]
    for kw in bad:
        _raises(lambda: iq.isoq_kv_copy_blocks(ok["pk"], pairs, **dict(planes, **kw)))
        _raises(lambda: iq.isoq_kv_compact(ok["pk"], keep, n_keep, table, **dict(planes, **kw)))
    for x in (pairs.long(), pairs[:, :1], pairs.to("meta"), pairs.t().contiguous().t(), pairs[0]):
        _raises(lambda: iq.isoq_kv_copy_blocks(ok["pk"], x, **planes))
    three = torch.zeros((3, 3, 5), dtype=torch.int32)
    for args in ((keep.long(), n_keep, table), (keep[0], n_keep, table), (three, n_keep, table), (keep[:2], n_keep, table),
                 (keep[:, :, ::2], n_keep, table), (keep.to("meta"), n_keep, table), (keep, n_keep.long(), table),
                 (keep, n_keep[:2], table), (keep, n_keep.to("meta"), table), (keep, n_keep, table.long()),
                 (keep, n_keep, table[:2]), (keep, n_keep, table.to("meta"))):
        _raises(lambda: iq.isoq_kv_compact(ok["pk"], *args, **planes))


def test_page_calls_null_handles():
    assert binding.lib.isoq_kv_copy_blocks(None, None, None, 1, 1, None, None, None, None, None, None, 1, 16, None) == 3
    assert binding.lib.isoq_kv_compact(None, None, None, 1, 1, None, 1, None, 1, 1, None, None, None, None, None, None, 1,
                                       16, None) == 3


def test_tensors_off_the_current_device(monkeypatch):
    """Tensors, or a stream, on another device than the current one are refused (the stand-ins' device is -1)."""
    monkeypatch.setattr(binding, "_is_gpu", lambda t: t.device.type == "cpu")
    monkeypatch.setattr(binding, "lib", _NoPages(_NoLaunch(binding.lib)))
    ok = good()
    planes = {k: ok[k] for k in ("k_idx", "k_rho", "v_idx", "v_rho")}
    calls = [lambda **kw: iq.isoq_kv_attn(**ok, **kw),
             lambda **kw: iq.isoq_kv_copy_blocks(ok["pk"], torch.zeros((3, 2), dtype=torch.int32), **planes, **kw),
             lambda **kw: iq.isoq_kv_compact(ok["pk"], torch.zeros((3, 1, 5), dtype=torch.int32),
                                             torch.zeros(3, dtype=torch.int32), ok["block_table"], **planes, **kw)]

    class Stream:
        device, cuda_stream = torch.device("cuda:1"), 0
    for call in calls:
        monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0)
        with pytest.raises(ValueError, match="not the current device"):
            call()
        monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: -1)
        with pytest.raises(ValueError, match="stream on cuda:1"):
            call(stream=Stream())
