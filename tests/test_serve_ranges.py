"""Numbers that do not fit the library's 32-bit arguments are refused, not taken modulo 2^32."""
import pytest
import torch

import paper_2606_10531_amd as lc


def _args(B=1):
    data, scales = lc.kv_cache(2, 16, 2, 64, device="cpu")
    return dict(q=torch.zeros((3, 4, 64), dtype=torch.bfloat16), data=data, table=torch.zeros((B, 0), dtype=torch.int32),
                kv_lens=torch.zeros(1, dtype=torch.int32).expand(B), q_starts=torch.zeros(1, dtype=torch.int32).expand(B + 1), scales=scales)


@pytest.mark.parametrize("name", ["window", "max_q"])
@pytest.mark.parametrize("value", [2**31, 2**32 + 5, 2**63, -2**31 - 1, -2**32 + 1])
def test_attention(name, value):
    with pytest.raises(ValueError, match=name):
        lc.attn_paged(**_args(), **{name: value})


def test_attention_sequences():
    with pytest.raises(ValueError, match="sequences"):
        lc.attn_paged(**_args(2**32 + 1))


@pytest.mark.parametrize("f", [lambda **k: lc.attn_workspace_bytes(**{**dict(T=4, B=2, Hq=4, Hkv=2, D=64, max_q=4), **k})])
@pytest.mark.parametrize("name", ["B", "Hq", "Hkv", "D", "max_q"])
def test_workspace_size(f, name):
    assert f() > 0
    with pytest.raises(ValueError, match=name):
        f(**{name: 2**32 + 4})


@pytest.mark.parametrize("group", [2**32 + 64, 2**31, -2**32 + 64])
def test_group(group):
    """(n = 0 is a multiple of any.)"""
    with pytest.raises(ValueError, match="group"):
        lc.linear_fwd_int4(torch.zeros((8, 0), dtype=torch.uint8), torch.zeros((8, 0), dtype=torch.bfloat16),
                           torch.zeros((2, 0), dtype=torch.bfloat16), group)
