"""The bindings of the model steps: what they refuse before the library is called (host)."""
import pytest

from paper_2308_16369_amd import sarathi as S


@pytest.mark.parametrize("have", [0, 1])
@pytest.mark.parametrize("step", [S.sarathi_model_step, S.sarathi_mixed_model_step], ids=["hybrid", "mixed"])
def test_model_steps_refuse_too_few_layers_of_weights(monkeypatch, step, have):
    """The library reads n_layers entries of the weights' array: a shorter list never reaches it."""
    def none():
        raise AssertionError("the library was called")

    class KV:
        handle = None

    w = [S.make_weights({"norm1_g": 0x100000}) for _ in range(have)]
    batch, keep = S.make_mixed_batch([(0, 0, 4)], [], [])
    monkeypatch.setattr(S, "lib", none)
    with pytest.raises(S.SarathiError) as e:
        step(S.make_cfg(128, 2, 64, 256, n_layers=2), w, KV, batch, 0x100000, 0x200000, 0x300000, 1 << 20)
    assert e.value.code == S.EINVAL and "layers" in str(e.value)
