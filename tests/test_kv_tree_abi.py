"""What the calls for trees and eviction refuse, before anything is asked of the GPU: on the CPU, with a handle that has sizes and no memory."""

import ctypes as C

import pytest
import torch

from test_kv_abi import siso  # noqa: F401


class Handle(C.Structure):
    """The fields that arguments are checked against, as kv_internal.h has them, and room for the rest."""

    _fields_ = [("layers", C.c_int), ("kv_heads", C.c_int), ("dim", C.c_int), ("dp", C.c_int), ("page_tokens", C.c_int), ("dtype", C.c_int), ("pages", C.c_long),
                ("rest", C.c_char * 4096)]


@pytest.fixture
def at(siso):  # noqa: F811
    h = Handle(2, 2, 64, 64, 16, siso.BF16, 10)
    return C.addressof(h), h


def batch(siso, n=1, rows=3, first=64, length=64, pages=64, width=4, max_new=0, max_length=0):  # noqa: F811
    return C.byref(siso._KvBatchStruct(n, rows, first, length, pages, width, max_new, max_length))


A = 4096  # an address, never read


def test_trees(siso, at):  # noqa: F811
    lib, h = siso._lib, at[0]
    ok = batch(siso)
    assert lib.siso_kv_tree(None, ok, A, A, A) == siso.EINVAL
    for args in ((None, A, A, A), (ok, None, A, A), (ok, A, None, A), (ok, A, A + 8, A), (batch(siso, rows=257), A, A, A), (batch(siso, rows=600, max_new=257), A, A, A),
                 (batch(siso, first=None), A, A, A), (batch(siso, n=-1), A, A, A)):
        assert lib.siso_kv_tree(h, *args) == siso.EINVAL
        assert lib.siso_kv_last_error(h).startswith(b"siso_kv_tree")
    assert lib.siso_kv_tree(h, batch(siso, n=0, rows=0, first=None), None, None, None) == siso.OK


def test_attention_of_trees(siso, at):  # noqa: F811
    lib, h = siso._lib, at[0]
    ok = batch(siso)

    def call(layer=0, b=ok, mask=A, q=A, heads=4, scale=1.0, window=0, out=A, lse=A, handle=h):
        return lib.siso_kv_attend_tree(handle, layer, b, mask, q, 256, 64, heads, scale, window, out, lse)

    for wrong in (dict(handle=None), dict(layer=2), dict(layer=-1), dict(b=None), dict(mask=None), dict(mask=A + 4), dict(q=None), dict(q=A + 1), dict(heads=3), dict(heads=0),
                  dict(heads=2 * 129), dict(scale=float("nan")), dict(scale=float("inf")), dict(window=-1), dict(out=None), dict(out=A + 8), dict(lse=A + 2),
                  dict(b=batch(siso, rows=257)), dict(b=batch(siso, length=None)), dict(b=batch(siso, width=1 << 31))):
        assert call(**wrong) == siso.EINVAL, wrong
        if "handle" not in wrong:
            assert lib.siso_kv_last_error(h).startswith(b"siso_kv_attend_tree"), wrong


def test_verification_of_trees(siso, at):  # noqa: F811
    lib, h = siso._lib, at[0]
    ok = batch(siso)

    def call(b=ok, parent=A, tokens=A, vocab=10, type=siso.F32, target=A, u=A, accepted=A, rows=A, out=A, handle=h):
        return lib.siso_kv_verify_tree(handle, b, parent, tokens, vocab, type, target, 10, u, accepted, rows, out)

    for wrong in (dict(handle=None), dict(b=None), dict(parent=None), dict(tokens=None), dict(vocab=0), dict(vocab=(1 << 24) + 1), dict(type=siso.FP8), dict(target=None),
                  dict(target=A + 2), dict(type=siso.BF16, target=A + 1), dict(accepted=None), dict(rows=None), dict(out=None), dict(b=batch(siso, rows=257))):
        assert call(**wrong) == siso.EINVAL, wrong


def test_keeping(siso, at):  # noqa: F811
    lib, h = siso._lib, at[0]
    ok = batch(siso)
    for args in ((None, 0, ok, A), (h, 2, ok, A), (h, -2, ok, A), (h, 0, None, A), (h, 0, ok, None), (h, -1, batch(siso, pages=None), A)):
        assert lib.siso_kv_keep(*args) == siso.EINVAL


def test_weighing(siso, at):  # noqa: F811
    lib, h = siso._lib, at[0]
    ok = batch(siso)

    def call(layer=0, b=ok, q=A, heads=4, scale=1.0, window=0, lse=A, decay=1.0, mass=A, born=A, handle=h):
        return lib.siso_kv_weigh(handle, layer, b, q, 256, 64, heads, scale, window, lse, None, None, decay, mass, born)

    for wrong in (dict(handle=None), dict(layer=2), dict(layer=-1), dict(b=None), dict(q=None), dict(q=A + 1), dict(heads=5), dict(heads=2 * 129), dict(scale=float("nan")),
                  dict(window=-1), dict(lse=None), dict(lse=A + 2), dict(decay=-0.1), dict(decay=1.5), dict(decay=float("nan")), dict(mass=None), dict(mass=A + 1),
                  dict(born=A + 2), dict(b=batch(siso, rows=(1 << 24) + 1)), dict(b=batch(siso, length=None))):
        assert call(**wrong) == siso.EINVAL, wrong


def test_evicting(siso, at):  # noqa: F811
    lib, h = siso._lib, at[0]
    ok = batch(siso)

    def call(layer=0, b=ok, keep=10, recent=2, early=1, mass=A, born=A, to=None, width=0, handle=h):
        return lib.siso_kv_evict(handle, layer, b, keep, recent, early, mass, born, to, width)

    for wrong in (dict(handle=None), dict(layer=2), dict(layer=-2), dict(b=None), dict(keep=0), dict(keep=(1 << 23) + 1), dict(recent=-1), dict(early=-1), dict(recent=11),
                  dict(recent=6, early=5), dict(recent=1, early=1 << 62), dict(mass=None), dict(mass=A + 2), dict(born=A + 1), dict(to=A, width=-1), dict(to=A, width=1 << 30),
                  dict(b=batch(siso, pages=None))):
        assert call(**wrong) == siso.EINVAL, wrong


def test_tensors_that_do_not_fit(siso):  # noqa: F811
    """The binding's own checks, with tensors on the CPU and no handle."""
    kv = siso.PagedKV.__new__(siso.PagedKV)
    kv.kv_heads, kv.head_dim, kv.pages, kv.page_tokens, kv.layers = 2, 64, 5, 16, 2
    kv.device, kv._index, kv._h, kv._stream, kv._raw_stream = torch.device("cpu"), -1, None, None, 0
    kv._elsewhere = lambda: False
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    b = siso.KvBatch(i32(2), i32(1), i32(1, 2), 3, 0, 0)
    tree = siso.KvTree(i32(3), i32(3, 8), i32(3))
    with pytest.raises(ValueError, match="parent"):
        kv.tree(b, i32(4))
    with pytest.raises(ValueError, match="mask"):
        kv.attend(b, torch.zeros(3, 4, 64, dtype=torch.bfloat16), tree=siso.KvTree(i32(3), i32(3, 4), i32(3)))
    for tokens, target, u, what in ((i32(2), torch.zeros(3, 9), None, "tokens"), (i32(3), torch.zeros(2, 9), None, "target"), (i32(3), torch.zeros(3, 9).double(), None, "target"),
                                    (i32(3), torch.zeros(3, 18)[:, ::2], None, "target"), (i32(3), torch.zeros(3, 9), torch.zeros(4), "u")):
        with pytest.raises(ValueError, match=what):
            kv.verify_tree(b, tree, tokens, target, u)
    with pytest.raises(ValueError, match="rows"):
        kv.keep(b, i32(4))
    for layer in (-1, 2):
        with pytest.raises(ValueError, match="layer"):
            kv.keep(b, i32(3), layer=layer)
    with pytest.raises(ValueError, match="mass"):
        kv.weights(torch.zeros(2, 5, 2, 15))
    with pytest.raises(ValueError, match="born"):
        kv.weights(None, i32(2, 5, 2, 16))
    w = kv.weights()
    q, lse = torch.zeros(3, 4, 64, dtype=torch.bfloat16), torch.zeros(3, 4)
    for change, what in ((dict(lse=torch.zeros(3, 2)), "lse"), (dict(fresh=i32(2)), "fresh"), (dict(newest=i32(1).float()), "newest"),
                         (dict(weights=siso.KvWeights(torch.zeros(2, 5, 2, 16, dtype=torch.float64), None)), "mass")):
        with pytest.raises(ValueError, match=what):
            kv.weigh(b, **{**dict(q=q, lse=lse, weights=w), **change})
    with pytest.raises(ValueError, match="to"):
        kv.evict(b, w, 10, to=i32(2, 3))
    with pytest.raises(siso.SisoError):  # (all of it fits: there is no handle)
        kv.evict(b, w, 10, to=i32(1, 3))


def test_stored_answers_as_a_tree(siso):  # noqa: F811
    """near_hit's trees: what answers have in common is shared, token by token, at most so many rows."""
    from paper_2508_18736_amd import near_hit

    assert near_hit._branches([[1, 2, 3, 4], [1, 2, 5, 6], [7, 2]], 0, 6, 4) == ([1, 7, 2, 2, 3, 5], [0, 0, 1, 2, 3, 3], [1, 1, 2, 2, 3, 3])
    assert near_hit._branches([[1, 2, 3], [9, 2, 4, 5]], 1, 9, 2) == ([2, 3, 4], [0, 1, 1], [1, 2, 2])
    assert near_hit._branches([[1], []], 1, 4, 2) == ([], [], [])
    assert near_hit._branches([[1, 2]], 0, 0, 2) == ([], [], [])


@pytest.mark.parametrize("wrong", [dict(keep=-1), dict(keep=4, recent=5), dict(keep=4, recent=3, early=2), dict(keep=4, recent=-1), dict(keep=4, early=-1), dict(most=256)])
def test_bounds_that_near_hit_refuses(siso, wrong):  # noqa: F811
    from paper_2508_18736_amd import near_hit

    target = near_hit.Target(layers=1, heads=2, vocab=50, device="cpu")
    with pytest.raises(ValueError):
        near_hit.serve(target, [[1, 2]], [[[3, 4], [5]]], 3, **wrong)
