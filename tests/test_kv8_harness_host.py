"""The 8-bit cache's test helpers on the host: what they enqueue is in order."""
import pytest

torch = pytest.importorskip("torch")

import kv8_harness as H  # noqa: E402


@pytest.mark.parametrize("other", [False, True])
def test_plan_memory_is_filled_before_another_stream_writes_it(monkeypatch, other):
    """A plan's workspace is filled on the current stream; a plan made on another stream waits for the fill (work
    items of a fill that lands after the upload are addresses far outside the cache)."""
    calls, full = [], torch.full

    class Stream:
        cuda_stream = 5

    def filled(size, value, **kw):
        calls.append("fill")
        return full(size, value, dtype=kw["dtype"])

    class Plan:
        pass

    def create(kv, batch, ws, size, stream):
        calls.append(("create", stream))
        return Plan()

    monkeypatch.setattr(H.torch, "full", filled)
    monkeypatch.setattr(H.torch.cuda, "current_stream", lambda: Stream)
    monkeypatch.setattr(H.torch.cuda, "synchronize", lambda: calls.append("wait"))
    monkeypatch.setattr(H.S, "sarathi_kv8_plan_create", create)
    cache = object.__new__(H.Cache)
    cache.spec = H.Spec()
    cache.c, cache.kv = cache.spec.cfg(), None
    cache.plan(H.Batch(chunks=[(0, 0, 3)]), 9 if other else None)
    assert calls == (["fill", "wait", ("create", 9)] if other else ["fill", ("create", 5)])
