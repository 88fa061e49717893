"""Tables from request lengths, beam search's choice and the reordering behind it without a GPU: the refusals of the C ABI
and of the binding, the work split, and the references that the GPU tests compare with."""

import ctypes
import os
import subprocess

import numpy as np
import pytest
import torch

import serve_ref as R
from test_kv_cpu import BAD_CACHES, EALIGN, EINVAL, EUNSUPPORTED, FAKE, LIB, OK, ROOT, Cache, cache

I32 = torch.int32


class Pool(ctypes.Structure):
    _fields_ = [("pages", ctypes.c_int64), ("free_pages", ctypes.c_void_p), ("count", ctypes.c_void_p),
                ("count_out", ctypes.c_void_p)]


class Requests(ctypes.Structure):
    _fields_ = [("seqs", ctypes.c_int64), ("rows", ctypes.c_int64), ("max_len", ctypes.c_int64),
                ("ld_table", ctypes.c_int64), ("page_size", ctypes.c_int32)] + [
        (n, ctypes.c_void_p) for n in ("keep", "add", "held", "held_out", "row_offsets", "lens", "page_table", "own_table",
                                       "row_seq", "positions", "slots", "missing")]


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(LIB):
        pytest.skip("libsharq.so not built")
    lib = ctypes.CDLL(LIB)
    i64, vp, p, i32 = ctypes.c_int64, ctypes.c_void_p, ctypes.POINTER, ctypes.c_int32
    lib.sharq_kv_assign_workspace_bytes.restype = lib.sharq_beam_workspace_bytes.restype = ctypes.c_size_t
    lib.sharq_kv_assign_workspace_bytes.argtypes = [p(Requests)]
    lib.sharq_kv_assign.argtypes = [p(Pool), p(Requests), vp, ctypes.c_size_t, vp]
    lib.sharq_beam_workspace_bytes.argtypes = [i64, i64, i64]
    lib.sharq_beam_select.argtypes = [vp, ctypes.c_int, i64, i64, i64, i64, vp, vp, i32, vp, vp, vp, vp, vp,
                                      ctypes.c_size_t, vp]
    lib.sharq_beam_reorder.argtypes = [i64, i64, vp, vp, i32, vp, i64, vp, i64, i64, vp, vp, vp, i64, vp, i64, i64, vp]
    lib.sharq_kv_copy.argtypes = [p(Cache), vp, i64, vp]
    return lib


def assign(L, pool=(), ws=FAKE, size=1 << 30, **kw):
    p = dict(pages=8, free_pages=FAKE, count=FAKE, count_out=FAKE)
    r = dict(seqs=4, rows=8, max_len=64, ld_table=4, page_size=16, keep=FAKE, add=FAKE, held=FAKE, held_out=FAKE,
             row_offsets=FAKE, lens=FAKE, page_table=FAKE)
    p.update(pool), r.update(kw)
    return L.sharq_kv_assign(ctypes.byref(Pool(**p)), ctypes.byref(Requests(**r)), ws, size, None)


BAD_REQUESTS = [
    (dict(seqs=-1), EINVAL), (dict(rows=-1), EINVAL), (dict(rows=1 << 31), EINVAL), (dict(max_len=-1), EINVAL),
    (dict(ld_table=3), EINVAL), (dict(page_size=0), EINVAL), (dict(page_size=24), EINVAL),
    (dict(page_size=8), EUNSUPPORTED), (dict(page_size=2048), EUNSUPPORTED), (dict(seqs=1 << 17), EUNSUPPORTED),
    (dict(max_len=1 << 31, ld_table=1 << 30), EUNSUPPORTED),
    (dict(seqs=1 << 16, max_len=1 << 20, ld_table=1 << 16), EUNSUPPORTED),
]


def test_bad_requests(L):
    for kw, status in BAD_REQUESTS:
        assert assign(L, **kw) == status, kw
        r = dict(seqs=4, rows=8, max_len=64, ld_table=4, page_size=16)
        r.update(kw)
        assert L.sharq_kv_assign_workspace_bytes(ctypes.byref(Requests(**r))) == 0
    for name in ("keep", "add", "held", "held_out", "row_offsets", "lens", "page_table"):
        assert assign(L, **{name: None}) == EINVAL, name
        assert assign(L, **{name: FAKE + 2}) == EALIGN, name
    for name in ("own_table", "row_seq", "positions", "slots", "missing"):
        assert assign(L, **{name: FAKE + 1}) == EALIGN, name
    for kw, status in [(dict(pages=-1), EINVAL), (dict(free_pages=None), EINVAL), (dict(count=None), EINVAL),
                       (dict(count_out=None), EINVAL), (dict(count=FAKE + 2), EALIGN), (dict(pages=1 << 28), EUNSUPPORTED)]:
        assert assign(L, pool=kw) == status, kw
    assert assign(L, ws=None) == EINVAL and assign(L, size=35) == EINVAL and assign(L, ws=FAKE + 1) == EALIGN
    assert L.sharq_kv_assign(None, ctypes.byref(Requests(page_size=16, row_offsets=FAKE)), FAKE, 100, None) == EINVAL
    assert L.sharq_kv_assign(ctypes.byref(Pool()), None, FAKE, 100, None) == EINVAL
    assert L.sharq_kv_assign_workspace_bytes(None) == 0
    assert L.sharq_kv_assign_workspace_bytes(ctypes.byref(Requests(seqs=4, max_len=64, ld_table=4, page_size=16))) == 36


def select(L, x=FAKE, dt=0, ld=100, groups=2, beams=3, vocab=100, scores=FAKE, done=None, eos=-1, out=FAKE, parents=FAKE,
           tokens=FAKE, done_out=None, ws=FAKE, size=1 << 30):
    return L.sharq_beam_select(x, dt, ld, groups, beams, vocab, scores, done, eos, out, parents, tokens, done_out, ws, size,
                               None)


def test_bad_choices(L):
    need = L.sharq_beam_workspace_bytes(2, 3, 100)
    for kw, status in [(dict(x=None), EINVAL), (dict(scores=None), EINVAL), (dict(out=None), EINVAL),
                       (dict(parents=None), EINVAL), (dict(tokens=None), EINVAL), (dict(ws=None), EINVAL),
                       (dict(size=need - 1), EINVAL), (dict(ld=99), EINVAL), (dict(dt=3), EINVAL), (dict(groups=-1), EINVAL),
                       (dict(beams=0), EINVAL), (dict(vocab=0), EINVAL), (dict(eos=100), EINVAL), (dict(eos=-2), EINVAL),
                       (dict(done=FAKE), EINVAL), (dict(done_out=FAKE), EINVAL), (dict(done=FAKE, eos=5), EINVAL),
                       (dict(done=FAKE, done_out=FAKE), EINVAL), (dict(beams=33), EUNSUPPORTED),
                       (dict(groups=1 << 20), EUNSUPPORTED), (dict(vocab=1 << 30, ld=1 << 30), EUNSUPPORTED),
                       (dict(x=FAKE + 1), EALIGN), (dict(x=FAKE + 2, dt=2), EALIGN), (dict(scores=FAKE + 2), EALIGN),
                       (dict(tokens=FAKE + 1), EALIGN), (dict(ws=FAKE + 4), EALIGN)]:
        assert select(L, **kw) == status, kw
    assert select(L, groups=0, x=None, scores=None, out=None, parents=None, tokens=None, ws=None, size=0) == OK
    for bad in ((-1, 3, 100), (2, 0, 100), (2, 33, 100), (2, 3, 0), (2, 3, 1 << 30)):
        assert L.sharq_beam_workspace_bytes(*bad) == 0


def reorder(L, groups=2, beams=3, parents=FAKE, lens=FAKE, page=16, table=FAKE, ldt=8, out=FAKE + 4096, ldto=8, cols=8,
            copies=FAKE, tokens=FAKE, ids=FAKE, ldi=50, ids_out=FAKE + 4096, ldio=50, id_cols=50):
    return L.sharq_beam_reorder(groups, beams, parents, lens, page, table, ldt, out, ldto, cols, copies, tokens, ids, ldi,
                                ids_out, ldio, id_cols, None)


def test_bad_reorders(L):
    for kw, status in [(dict(groups=-1), EINVAL), (dict(beams=0), EINVAL), (dict(beams=33), EUNSUPPORTED),
                       (dict(groups=1 << 20), EUNSUPPORTED), (dict(parents=None), EINVAL), (dict(lens=None), EINVAL),
                       (dict(page=0), EINVAL), (dict(page=48), EINVAL), (dict(page=8), EUNSUPPORTED),
                       (dict(table=None), EINVAL), (dict(out=None), EINVAL), (dict(copies=None), EINVAL),
                       (dict(table=None, out=None), EINVAL), (dict(ldt=7), EINVAL), (dict(ldto=7), EINVAL),
                       (dict(cols=-1), EINVAL), (dict(tokens=None), EINVAL), (dict(ids=None), EINVAL),
                       (dict(ids_out=None), EINVAL), (dict(ldi=49), EINVAL), (dict(ldio=49), EINVAL),
                       (dict(id_cols=-1), EINVAL), (dict(out=FAKE, ldto=9), EINVAL), (dict(ids_out=FAKE, ldio=60), EINVAL),
                       (dict(parents=FAKE + 2), EALIGN), (dict(copies=FAKE + 1), EALIGN), (dict(tokens=FAKE + 2), EALIGN),
                       (dict(groups=1 << 15, cols=1 << 29, ldt=1 << 29, ldto=1 << 29), EUNSUPPORTED)]:
        assert reorder(L, **kw) == status, kw
    assert reorder(L, groups=0, parents=None, lens=None) == OK
    assert reorder(L, table=None, out=None, copies=None, ids=None, ids_out=None, tokens=None) == OK


def test_bad_copies(L):
    copy = lambda c=cache(), x=FAKE, n=3: L.sharq_kv_copy(ctypes.byref(c), x, n, None)  # noqa: E731
    for bad, status in BAD_CACHES:
        assert copy(cache(**bad)) == status, bad
    assert copy(x=None) == EINVAL and copy(n=-1) == EINVAL and copy(x=FAKE + 2) == EALIGN
    assert copy(n=1 << 40) == EUNSUPPORTED
    assert copy(x=None, n=0) == OK and copy(cache(pages=0, k=None, v=None)) == OK


def test_beam_split(tmp_path):
    """Every column of a row is in one turn, the lists fit the join's threads and LDS, and the workspace holds them."""
    (tmp_path / "s.cpp").write_text(
        '#include "sharq_serve.hpp"\nusing namespace sharq;\nextern "C" {\n'
        "int chunks(int64_t r, int64_t b, int64_t v) { return beam_split(r, b, v).chunks; }\n"
        "int tiles(int64_t r, int64_t b, int64_t v) { return beam_split(r, b, v).tiles; }\n"
        "int64_t lds(int64_t b, int64_t c) { return beam_lds(b, c); }\n"
        "int64_t bytes(int64_t r, int64_t b, int64_t v) { return beam_workspace(r, b, v); }\n"
        "int64_t parts(int p, int D, int f) { return copy_parts(p, D, f); }\n"
        "int tile() { return kBeamTile; }\n}\n")
    so = str(tmp_path / "s.so")
    subprocess.run(["g++", "-std=c++17", "-shared", "-fPIC", "-I", os.path.join(ROOT, "paper_2606_26587_amd", "csrc"),
                    str(tmp_path / "s.cpp"), "-o", so], check=True)
    lib = ctypes.CDLL(so)
    lib.lds.restype = lib.bytes.restype = lib.parts.restype = ctypes.c_int64
    for f in (lib.chunks, lib.tiles, lib.bytes):
        f.argtypes = [ctypes.c_int64] * 3
    lib.lds.argtypes = [ctypes.c_int64] * 2
    rng = np.random.default_rng(0)
    for _ in range(3000):
        beams = int(rng.integers(1, 33))
        rows = beams * int(rng.choice([1, 2, 5, 40, 1000]))
        vocab = int(np.exp(rng.uniform(0, np.log(400000))))
        c, t = lib.chunks(rows, beams, vocab), lib.tiles(rows, beams, vocab)
        assert c >= 1 and t >= 1 and (c - 1) * t * lib.tile() < vocab <= c * t * lib.tile()
        assert c * beams <= 256 and lib.lds(beams, c) <= 56 << 10   # and 5 KB: 64 KB a workgroup
        assert lib.bytes(rows, beams, vocab) >= rows * c * (beams * 8 + 4 * 16)
    for page in (16, 64, 1024):
        for D in (64, 128):
            for f, w in ((0, 2 * D), (1, D // 2), (2, D)):
                n = lib.parts(page, D, f)
                assert n * 1024 >= 2 * page * w // 16 > (n - 1) * 1024


def test_binding_refuses_wrong_tensors(monkeypatch):
    from paper_2606_26587_amd import sharq as S
    monkeypatch.setattr(S, "_device", lambda: -1)

    def refused(f, *a, **kw):
        with pytest.raises(S.SharqError) as e:
            f(*a, **kw)
        assert e.value.status == EINVAL

    z = lambda *s, d=I32: torch.zeros(s, dtype=d)  # noqa: E731
    pool = S.KVPool(z(8), z(1))
    assert pool.pages == 8
    refused(S.KVPool, z(8, d=torch.int64), z(1))
    refused(S.KVPool, z(8), z(2))
    refused(S.KVPool, z(16)[::2], z(1))
    args = dict(keep=z(3), add=z(3), held=z(3), row_offsets=z(4), lens=z(3), page_table=z(3, 4), rows=5, max_len=64,
                page_size=16)
    r = S.KVRequests(**args)
    b = r.batch(2)
    assert b.rows == 5 and b.lens is r.lens and b.max_len == 64
    for bad in (dict(add=z(2)), dict(held=z(3, d=torch.int64)), dict(row_offsets=z(3)), dict(lens=z(6)[::2]),
                dict(page_table=z(3, 3)), dict(page_table=z(2, 4)), dict(page_table=z(4, 3).T), dict(held_out=z(4)),
                dict(own_table=z(3, 5)), dict(row_seq=z(4)), dict(positions=z(6)), dict(slots=z(5, d=torch.int64)),
                dict(missing=z(2)), dict(rows=-1), dict(max_len=-1), dict(page_size=0)):
        refused(S.KVRequests, **{**args, **bad})
    assert S.kv_assign_workspace_bytes(r) == 28
    refused(S.sharq_kv_assign, pool, r)                      # not on a GPU
    x, s = z(6, 50, d=torch.float32), z(2, 3, d=torch.float32)
    refused(S.sharq_beam_select, x, s)
    refused(S.sharq_beam_reorder, z(2, 3), z(6), z(6, 4), 16)
    c = S.alloc_kv_cache(4, 16, 2, 128, "fp8", "cpu")
    refused(S.sharq_kv_copy, c, z(3, 3))
    # the checks behind that of the device
    class OnDevice(torch.Tensor):
        def get_device(self):
            return 0
    monkeypatch.setattr(S, "_device", lambda: 0)
    g = lambda t: t.as_subclass(OnDevice)  # noqa: E731
    ok = dict(logits=g(x), scores=g(s))
    for bad in (dict(scores=g(z(3, 3, d=torch.float32))), dict(scores=s), dict(scores=g(z(2, 3))), dict(logits=g(z(50, 6, d=torch.float32).T)),
                dict(logits=g(x[:, 0])), dict(done=g(z(2, 3))), dict(parents=g(z(6))), dict(tokens=z(2, 3)),
                dict(scores_out=g(z(2, 4, d=torch.float32))), dict(workspace=z(99, d=torch.uint8))):
        refused(S.sharq_beam_select, **{**ok, **bad})
    ok = dict(parents=g(z(2, 3)), lens=g(z(6)), page_table=g(z(6, 4)), page_size=16)
    for bad in (dict(lens=g(z(5))), dict(page_table=g(z(5, 4))), dict(page_table=g(z(6, 4, d=torch.int64))),
                dict(table_out=g(z(6, 5))), dict(copies=g(z(6, 2))), dict(ids=g(z(5, 9)), tokens=g(z(2, 3))),
                dict(ids=g(z(6, 9)), tokens=g(z(3, 2))), dict(ids_out=g(z(6, 9))), dict(parents=g(z(6))),
                dict(page_table=None, copies=g(z(6, 3))), dict(page_table=None, table_out=g(z(6, 4)))):
        refused(S.sharq_beam_reorder, **{**ok, **bad})


# ---------------------------------------------------------------------------
# The references
# ---------------------------------------------------------------------------

def test_reference_assignment():
    table = np.full((3, 4), -9)
    table[0, :2], table[1, :3] = (5, 6), (7, -1, 8)
    free = [1, 2, 3, 0, 0, 0, 0, 0, 0, 0]
    out = R.assign(free, 3, [20, 0, 0], [13, 0, 20], [2, 3, 0], table, 100, 64, 16)
    assert out["row_offsets"] == [0, 13, 13, 33] and out["lens"] == [33, 0, 20] and out["held"] == [3, 0, 2]
    assert free[:5] == [1, 2, 3, 7, 8] and out["count"] == 2 and out["missing"] == 0
    assert list(table[0]) == [5, 6, 8, -9] and list(table[2]) == [7, 3, -9, -9]
    assert out["positions"][:13] == list(range(20, 33)) and out["slots"][:2] == [6 * 16 + 4, 6 * 16 + 5]
    assert out["slots"][12] == 8 * 16 and out["row_seq"][13:33] == [2] * 20 and out["slots"][99] is None


def test_reference_choice():
    x = np.log(np.array([[0.5, 0.25, 0.25], [0.9, 0.05, 0.05]]))
    c = R.candidates(x, np.log([0.5, 0.4]), None, -1)
    assert [(b, v) for _, b, v in c] == [(1, 0), (0, 0), (0, 1), (0, 2), (1, 1), (1, 2)]
    assert np.allclose(np.exp([s for s, _, _ in c]), [0.36, 0.25, 0.125, 0.125, 0.02, 0.02])
    c = R.candidates(x, np.log([0.5, 0.4]), [0, 1], 2)
    assert [(b, v) for _, b, v in c] == [(1, 2), (0, 0), (0, 1), (0, 2)]
    assert R.candidates(np.array([[-np.inf, -np.inf], [0, np.nan]]), [0.0, 0.0], None, -1) == []


def test_reference_reordering_keeps_pages_apart():
    rng = np.random.default_rng(1)
    for _ in range(200):
        beams, length = int(rng.integers(1, 9)), int(rng.integers(0, 70))
        table = rng.permutation(beams * 5).reshape(beams, 5)
        parents = rng.integers(0, beams, beams)
        new, copies, ids = R.reorder(parents, length, 16, table, rng.integers(0, 9, (beams, 80)), list(range(beams)))
        new = np.array(new)
        whole, part = divmod(length, 16)
        assert np.array_equal(new[:, :whole], table[parents][:, :whole])
        assert np.array_equal(new[:, whole + 1:], table[:, whole + 1:])
        if part:
            assert sorted(new[:, whole]) == sorted(table[:, whole])
            holds = {int(p): int(p) for p in table[:, whole]}       # page -> whose tokens it holds
            for s, d, n in copies:
                if n > 0:
                    assert n == part
                    holds[int(d)] = int(s)
            assert [holds[int(p)] for p in new[:, whole]] == [int(table[q, whole]) for q in parents]
        else:
            assert copies == [(-1, -1, -1)] * beams
