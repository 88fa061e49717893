"""What the binding of the key/value cache passes on and refuses, without a GPU:
the library is replaced by a recorder, so no kernel is launched."""

import pytest
import torch

from paper_2606_26587_amd import sharq as S


class Recorder:
    """Stands in for the library: every call succeeds and its arguments are kept."""
    sharq_status_str = S.lib.sharq_status_str

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append((name, args))
            return 0
        return call


@pytest.fixture
def lib(monkeypatch):
    r = Recorder()
    monkeypatch.setattr(S, "lib", r)
    monkeypatch.setattr(S, "_here", lambda *a: None)
    monkeypatch.setattr(S, "_current", lambda: 0)
    return r


def i32(*v):
    return torch.tensor(v, dtype=torch.int32)


def rows(n, width):
    return torch.zeros(n, width, dtype=torch.bfloat16)


@pytest.mark.parametrize("columns", [slice(0, 4), slice(60, 64)])
def test_tokens_past_a_sliced_page_table_are_refused(lib, columns):
    """A table that is a slice of a wider one has a row stride above its width: the entries behind a row's own are the
    parent's, and behind its last row there may be none.  max_len is bounded by the width, not by the stride."""
    cache = S.alloc_kv_cache(8, 16, 2, 64, "bf16", "cpu")
    table = torch.zeros(2, 64, dtype=torch.int32)[:, columns]
    q, kv = rows(2, 256), rows(2, 128)
    for max_len, fits in ((1, True), (64, True), (65, False), (1024, False), (1025, False)):
        b = S.KVBatch(i32(0, 1, 2), i32(1, 1), table, 2, 1, max_len)
        for f, args in ((S.sharq_kv_append, (q, kv, kv, cache, b)), (S.sharq_kv_read, (cache, b)),
                        (S.sharq_attention, (q, cache, b))):
            lib.calls.clear()
            if fits:
                f(*args)
                assert lib.calls
                continue
            with pytest.raises(S.SharqError) as e:
                f(*args)
            assert e.value.status == S.EINVAL and not lib.calls


def test_empty_batches_need_no_page_table(lib):
    """Nothing is looked up for no sequence or no row, whatever max_len says."""
    cache = S.alloc_kv_cache(8, 16, 2, 64, "bf16", "cpu")
    none = torch.zeros(0, 0, dtype=torch.int32)
    S.sharq_attention(rows(0, 256), cache, S.KVBatch(i32(0), i32(), none, 0, 1, 64))
    S.sharq_attention(rows(3, 256), cache, S.KVBatch(i32(0), i32(), none, 3, 1, 64))
    S.sharq_kv_read(cache, S.KVBatch(i32(0, 0), i32(5), torch.zeros(1, 0, dtype=torch.int32), 0, 1, 64))


@pytest.fixture
def on_stream(monkeypatch):
    """The stream that torch.cuda.stream made current, and those that were at every allocation."""
    now, seen = [None], []

    class Context:
        def __init__(self, stream):
            self.stream = stream

        def __enter__(self):
            self.before, now[0] = now[0], self.stream

        def __exit__(self, *exc):
            now[0] = self.before

    def allocates(real):
        def f(*a, **kw):
            seen.append(now[0])
            return real(*a, **kw)
        return f

    monkeypatch.setattr(torch.cuda, "stream", Context)
    monkeypatch.setattr(torch, "empty", allocates(torch.empty))
    monkeypatch.setattr(torch, "empty_like", allocates(torch.empty_like))
    return seen


def entry_points():
    """Every entry point that allocates a buffer of its call, without that buffer given."""
    cache = S.alloc_kv_cache(8, 16, 2, 64, "bf16", "cpu")
    batch = S.KVBatch(i32(0, 1, 2), i32(1, 1), torch.zeros(2, 4, dtype=torch.int32), 2, 1, 64)
    q, kv, x = rows(2, 256), rows(2, 128), rows(2, 128)
    w, act = S.alloc_weight(64, 128, device="cpu"), S.alloc_act(2, 128, device="cpu")
    return {"kv_append": (S.sharq_kv_append, (q, kv, kv, cache, batch)),
            "kv_read": (S.sharq_kv_read, (cache, batch)),
            "kv_read_v": (S.sharq_kv_read, (cache, batch, kv)),
            "attention": (S.sharq_attention, (q, cache, batch)),
            "quantize_weight": (S.sharq_quantize_weight, (rows(64, 128),)),
            "prepare": (S.sharq_prepare, (x, None)),
            "prepare_residual": (S.sharq_prepare_residual, (x, x, None)),
            "prepare_silu_mul": (S.sharq_prepare_silu_mul, (x, x)),
            "linear": (S.sharq_linear, (act, w)),
            "prepare_linear": (S.sharq_prepare_linear, (x, None, w)),
            "linear_grouped": (S.sharq_linear_grouped, (act, None, i32(0, 2), 2, w))}


@pytest.mark.parametrize("name", ["kv_append", "kv_read", "kv_read_v", "attention", "quantize_weight", "prepare",
                                  "prepare_residual", "prepare_silu_mul", "linear", "prepare_linear", "linear_grouped"])
def test_buffers_of_a_call_are_allocated_on_its_stream(lib, on_stream, monkeypatch, name):
    """The allocator orders a block's next use behind its last one on the stream it was allocated on, and on no other:
    what a call on another stream writes must come from that stream."""
    for entry in ("sharq_act_buffer_bytes_mode", "sharq_attention_workspace_bytes"):
        monkeypatch.setattr(lib, entry, lambda *a: 64, raising=False)
    f, args = entry_points()[name]
    side = type("Stream", (), {"cuda_stream": 7})()
    on_stream.clear()
    f(*args, stream=side)
    assert on_stream and all(s is side for s in on_stream)
    assert lib.calls[-1][1][-1] == 7                        # and the library is told the same stream
    on_stream.clear()
    f(*args, stream=None)
    assert on_stream and all(s is None for s in on_stream)


def test_a_scale_in_a_tensor_is_read_at_every_call(lib):
    """A 0-d tensor's value may change between calls; the structure of a call is kept by its values, not by the object
    that held them."""
    cache = S.alloc_kv_cache(8, 16, 2, 64, "bf16", "cpu")
    batch = S.KVBatch(i32(0, 1, 2), i32(1, 1), torch.zeros(2, 4, dtype=torch.int32), 2, 1, 64)
    scale, window, sinks = torch.tensor(0.5), torch.tensor(7), torch.tensor(1)

    def passed():
        lib.calls.clear()
        S.sharq_attention(rows(2, 256), cache, batch, scale=scale, window=window, sinks=sinks)
        t = lib.calls[-1][1][6]._obj
        return t.scale, t.window, t.sinks

    assert passed() == (0.5, 7, 1)
    scale.fill_(0.25)
    window.fill_(100)
    sinks.fill_(4)
    assert passed() == (0.25, 100, 4)
    assert passed() == (0.25, 100, 4)
    with pytest.raises(TypeError):
        S.sharq_attention(rows(2, 256), cache, batch, window=1.5)
