"""CPU checks of the forms of isoq_kv_attn in the binding: a prefix together with attention
to all positions, which no kernel has, is refused and not taken as causal."""
import pytest

import paper_2603_28430_amd as iq
from paper_2603_28430_amd import isoquant as binding
from test_kv_attn_checks import good
from test_kv_attn_shared_checks import cpu_as_device, prefixed, reaches  # noqa: F401


def test_all_positions_behind_a_prefix(cpu_as_device):   # noqa: F811
    ok = prefixed()
    prefix = binding._Prefix(ok["prefix_table"], ok["prefix_lens"], ok["prefix_start"], None, None, ok["q"].shape[0],
                             ok["k_idx"].shape[2])
    reaches(lambda: iq.isoq_kv_attn(**good(), prefix=prefix), "isoq_kv_attn_prefix")
    reaches(lambda: iq.isoq_kv_attn(**good(), causal=False), "isoq_kv_attn_cross")
    with pytest.raises(ValueError, match="causal"):
        iq.isoq_kv_attn(**good(), causal=False, prefix=prefix)
