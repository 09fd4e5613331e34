"""The binding of the 8-bit model step: what it refuses before the library is called (host)."""
import pytest

from paper_2308_16369_amd import sarathi as S


@pytest.mark.parametrize("have", [0, 1])
def test_model_step_refuses_too_few_layers_of_weights(monkeypatch, have):
    """The library reads n_layers entries of the weights' array: a shorter list never reaches it."""
    def none():
        raise AssertionError("the library was called")

    w = [S.make_kv8_weights({"norm1_g": 0x100000}) for _ in range(have)]
    batch, keep = S.make_mixed_batch([(0, 0, 4)], [], [])
    cfg = S.make_cfg(128, 8, 64, 256, n_layers=2)
    monkeypatch.setattr(S, "lib", none)
    with pytest.raises(S.SarathiError) as e:
        S.sarathi_kv8_model_step(cfg, w, None, batch, 0x100000, 0x200000, 0x300000, 1 << 20)
    assert e.value.code == S.EINVAL and "layers" in str(e.value)
