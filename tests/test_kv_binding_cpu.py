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
