"""Outputs and workspaces that the caller leaves to the binding come from the
memory of the stream that the call runs on."""
import contextlib

import pytest

torch = pytest.importorskip("torch")


def calls(fq, put):
    """(name, number of tensors the binding makes, call(stream)) of every entry point,
    with nothing given that it can make."""
    i8, i32, u8, f32 = torch.int8, torch.int32, torch.uint8, torch.float32
    z = lambda *shape, dtype=i8: put(torch.zeros(*shape, dtype=dtype))  # noqa: E731
    x, w, mul, q = z(4, 8), z(3, 8), z(3, dtype=f32), z(2, 5, 32)
    logits, alpha, ones = z(2, 5, 5, dtype=i32), z(8, dtype=u8), z(8, dtype=f32)
    s, zp = put(torch.ones(1, dtype=torch.float64)), z(1, dtype=i32)
    return [
        ("ptf_layernorm_int8", 1, lambda t: fq.ptf_layernorm_int8(x, 0, alpha, 3, ones, ones, 1.0, 0, stream=t)),
        ("lis_softmax_log4", 1, lambda t: fq.lis_softmax_log4(logits, 0.01, stream=t)),
        ("lis_attn_v_shift", 1, lambda t: fq.lis_attn_v_shift(z(2, 5, 3, dtype=u8), q, 5, stream=t)),
        ("lis_attn_v_shift_wide", 1,
         lambda t: fq.lis_attn_v_shift_wide(z(2, 5, 5, dtype=u8), q, 5, stream=t)),
        ("lis_attention_head", 1, lambda t: fq.lis_attention_head(logits, q, 0.01, stream=t)),
        ("lis_attention_qk", 1, lambda t: fq.lis_attention_qk(q, q, q, 0.01, stream=t)),
        ("ptf_calibrate", 4, lambda t: fq.ptf_calibrate(z(4, 8, dtype=f32), stream=t)),
        ("ptf_calibrate_noalloc", 3, lambda t: fq.ptf_calibrate_noalloc(z(4, 8, dtype=f32), stream=t)),
        ("ptf_quantize_int8", 1, lambda t: fq.ptf_quantize_int8(z(4, 8, dtype=f32), s, zp, alpha, stream=t)),
        ("requant_dyadic_int8", 1, lambda t: fq.requant_dyadic_int8(logits, 1.0, 1.0, 0, stream=t)),
        ("linear_fold_int8", 2, lambda t: fq.linear_fold_int8(w, mul, 1.0, stream=t)),
        ("linear_int8", 1, lambda t: fq.linear_int8(x, w, None, mul, stream=t)),
        ("linear_int32", 1, lambda t: fq.linear_int32(x, w, stream=t)),
        ("rope_table_int16", 1, lambda t: fq.rope_table_int16(z(1, 5, dtype=i32), s, z(1, dtype=u8), stream=t)),
        ("rope_qkv_int8", 3, lambda t: fq.rope_qkv_int8(z(2, 5, 32), None, 2, 1, 1.0, 1.0, 1.0, stream=t)),
        ("requant_heads_int8", 1, lambda t: fq.requant_heads_int8(z(2, 3, 5, 8, dtype=i32), 1.0, 1.0, 0, stream=t)),
    ]


def test_allocations_are_made_on_the_given_stream(monkeypatch):
    """Without a GPU: what each entry point allocates, it allocates with the given
    stream current, before it refuses the host tensors; without one, with none made
    current."""
    import paper_2111_13824_amd as fq
    from paper_2111_13824_amd import binding as B
    assert {n for n, _, _ in calls(fq, lambda t: t)} == set(B.SIGNATURES) - {"fq_activation_table"}
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
    for name, n, call in calls(fq, lambda t: t):
        for stream in (Stream(), None):
            del made[:]
            with pytest.raises(ValueError, match="device tensor"):
                call(stream)
            assert all(s is stream for s in made), name
            assert stream is None or len(made) == n, name


@pytest.mark.gpu
def test_outputs_come_from_the_memory_of_their_stream():
    import paper_2111_13824_amd as fq
    side = torch.cuda.Stream()
    made = calls(fq, lambda t: t.to("cuda:0"))
    torch.cuda.synchronize()
    for name, _, call in made:
        print("CASE stream", name, flush=True)
        out = call(side)
        torch.cuda.synchronize()
        for t in out if isinstance(out, tuple) else (out,):
            pool, = [s["stream"] for s in torch.cuda.memory_snapshot()
                     if s["address"] <= t.data_ptr() < s["address"] + s["total_size"]]
            assert pool == side.cuda_stream, name
