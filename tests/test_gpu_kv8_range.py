"""8-bit KV cache, attention at the ends of its range: value scales far apart and beside zero blocks."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from kv8_harness import Batch, Cache, Spec, check_attention  # noqa: E402
from test_gpu_kv8 import attend, gen  # noqa: E402

KINDS = [("bf16", "int8"), ("bf16", "e4m3"), ("f32", "int8"), ("f32", "e4m3")]


@pytest.mark.parametrize("big,small", [(20, None), (60, None), (20, -60), (60, -74)], ids=str)
@pytest.mark.parametrize("first", [0, 1], ids=["big_first", "small_first"])
@pytest.mark.parametrize("block,run", [(16, 1), (32, 4)])
@pytest.mark.parametrize("dtype,fmt", KINDS)
def test_keys_count_whatever_their_value_scale(dtype, fmt, block, run, first, big, small):
    """Every key has the same score.  Runs of blocks with scales 2^big times the usual ones beside runs of zeros (scale
    0) or of scales 2^small times them, in both orders, within one step and from step to step: the small ones' keys
    count in the softmax all the same."""
    spec = Spec(heads=4, kv_heads=2, dim=64, dtype=dtype, fmt=fmt, block=block)
    cache = Cache(spec)
    cache.fill(gen(3))
    codes, scales = cache.views()
    codes[:, :, 0] = 0
    for b in range(scales.shape[-1]):
        if (b // run) % 2 == first:
            scales[:, :, 1, :, b] *= 2.0 ** big
        elif small is not None:
            scales[:, :, 1, :, b] *= 2.0 ** small
        else:
            codes[:, :, 1, :, b * block:(b + 1) * block] = 0
            scales[:, :, 1, :, b] = 0
    b = Batch(chunks=[(1, 37, 70)], decodes=[(0, 299), (2, 47), (3, 160)])
    q = torch.randn((b.T, 4 * 64), device="cuda", generator=gen(4)).to(spec.tdt)
    check_attention(spec, b, cache.values(), q, attend(cache, b, q), scales=cache.host()[1])
