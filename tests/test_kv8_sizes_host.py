"""Sizes of the 8-bit cache's layer workspace beyond 32 bits (host)."""
import pytest

from paper_2308_16369_amd import sarathi as S


@pytest.mark.parametrize("T", [(1 << 24), (1 << 26), (1 << 31) - 1])
@pytest.mark.parametrize("dtype", [S.BF16, S.F32])
def test_layer_workspace_in_64_bits(T, dtype):
    """rows x heads passes 2^31: every region still has room for its rows, and the total for all of them."""
    nh, nkv, hd, H, F = 256, 8, 128, 256, 512
    kv_cfg = S.make_kv8_cfg(nh, nkv, hd, n_layers=1, dtype=dtype, rope_dim=128)
    model = S.make_cfg(H, nh, hd, F, n_layers=1, dtype=dtype)
    es = 2 if dtype == S.BF16 else 4
    L = S.sarathi_kv8_workspace_layout(model, kv_cfg, T, 1, 128)
    assert L.total == S.sarathi_kv8_workspace_bytes(model, kv_cfg, T, 1, 128)
    assert L.qkv - L.a >= T * H * es
    assert L.o - L.qkv >= T * (nh + 2 * nkv) * hd * es
    assert L.hres - L.o >= T * nh * hd * es
    assert L.m - L.hres >= T * H * 4
    assert L.ping[0] - L.m >= T * F * es and L.ping[1] - L.ping[0] >= T * H * es
    assert L.total - L.ping[1] >= T * H * es + S.sarathi_kv8_plan_bytes(kv_cfg, T, 1, 128)
