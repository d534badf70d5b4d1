"""Without a GPU: what the decoding calls allocate, they allocate with the given stream
current, before they refuse host tensors; without one, with none made current."""
import contextlib

import pytest

torch = pytest.importorskip("torch")


def test_allocations_are_made_on_the_given_stream(monkeypatch):
    import paper_2111_13824_amd as fq
    from paper_2111_13824_amd import binding as B
    z = lambda *shape, dtype=torch.int8: torch.zeros(*shape, dtype=dtype)  # noqa: E731
    i32 = torch.int32
    r, ones = z(4, 8, dtype=torch.int16), torch.ones(8)
    kp, vp, w = z(5, 2, 16, 32), z(5, 2, 32, 16), z(5, 2, 16, dtype=torch.int64)
    table, n = z(3, 4, dtype=i32), z(3, dtype=i32)
    long = z(1, 1000, dtype=i32)
    calls = {"rmsnorm_int8": (2, lambda t: fq.rmsnorm_int8(r, ones, 1.0, 1.0, stream=t)),
             "rmsnorm_rows_int8": (3, lambda t: fq.rmsnorm_rows_int8(r, ones, 1.0, stream=t)),
             "kv_cache_append_int8": (0, lambda t: fq.kv_cache_append_int8(z(3, 2, 1, 32), z(3, 2, 1, 32), kp, vp,
                                                                          table, n, stream=t)),
             "lis_attention_paged": (2, lambda t: fq.lis_attention_paged(z(1, 4, 1, 32), kp, vp, long, z(1, dtype=i32),
                                                                        0.01, stream=t)),
             "kv_cache_evict": (2, lambda t: fq.kv_cache_evict(kp, vp, w, table, n, 20, stream=t))}
    assert set(calls) == set(B.DECODE_SIGNATURES)
    current, made, empty = [None], [], torch.empty

    @contextlib.contextmanager
    def on(stream):
        current[0] = stream
        yield
        current[0] = None

    class Stream:
        cuda_stream = 0

    def counted(*a, **kw):
        made.append(current[0])
        return empty(*a, **kw)

    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch, "empty", counted)
    for name, (count, call) in calls.items():
        for stream in (Stream(), None):
            del made[:]
            with pytest.raises(ValueError, match="device tensor"):
                call(stream)
            assert all(s is stream for s in made), name
            assert stream is None or len(made) == count, name
