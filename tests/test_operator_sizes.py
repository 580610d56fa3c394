"""Sizes past 32 bits through the binding: refused as sizes, not taken for what is left of them."""
import pytest

from paper_2310_14997_amd import binding as bd

FAR = 1 << 32


def refused(call, *args):
    with pytest.raises(bd.SpcfgError) as err:
        call(*args)
    assert err.value.code == -2


def test_sizes_past_32_bits():
    import torch
    for sizes in ((FAR + 4, 8, 8), (4, FAR + 8, 8), (4, 8, FAR + 8)):
        refused(bd.make_dense_config, *sizes)
    for sizes in ((FAR + 5, 7), (5, FAR + 7), (5, -FAR + 7)):
        refused(bd.spcfg_distill_workspace_bytes, *sizes)
    m = lambda *s, **k: torch.empty(*s, device="meta", **k)  # (no memory behind them: only their sizes are looked at)
    i32, out = torch.int32, m(1)
    refused(bd.spcfg_distill_forward, m(1, FAR + 10), m(1, 3), m(1, 3, dtype=i32), 1.0, out, out, None)
    refused(bd.spcfg_distill_backward, m(FAR + 1, 10), m(FAR + 1, 3), m(FAR + 1, 3, dtype=i32), 1.0, out, None, out)
    refused(bd.spcfg_distill_forward, m(1, 10), m(1, FAR + 3), m(1, FAR + 3, dtype=i32), 1.0, out, out, None)
    refused(bd.spcfg_preference_forward, m(FAR + 4), None, m(2, dtype=i32), m(2, dtype=i32), 0.1, 0.0, out, out)
    refused(bd.spcfg_preference_forward, m(4), None, m(FAR + 2, dtype=i32), m(FAR + 2, dtype=i32), 0.1, 0.0, out, out)
