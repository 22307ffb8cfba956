"""Refusals of the gradient-list calls that need no GPU: arguments are looked at before the device is."""
import ctypes as C

import pytest


@pytest.fixture(scope="module")
def B():
    import __graft_entry__ as ge
    ge.build()
    from paper_2505_00347_b200 import binding
    return binding


def create(B, sizes, n=None, geom=256):
    h = C.c_void_p(1)
    arr = (C.c_int64 * max(1, len(sizes)))(*sizes)
    return B.lib().solo_grads_create(arr, len(sizes) if n is None else n, geom, None, C.byref(h)), h


def test_sizes_are_checked(B):
    for sizes, n in (([], None), ([1], -1), ([-1], None), ([5, -3], None), ([(1 << 48) + 1], None), ([1 << 48] * 40, None)):
        rc, h = create(B, sizes, n)
        assert rc == B.SOLO_EINVAL and not h.value, (sizes, n)
    assert create(B, [4], geom=None)[0] == B.SOLO_EINVAL and create(B, [4], geom=260)[0] == B.SOLO_EALIGN
    assert B.lib().solo_grads_create(None, 1, 256, None, C.byref(C.c_void_p())) == B.SOLO_EINVAL
    assert B.lib().solo_grads_create((C.c_int64 * 1)(4), 1, 256, None, None) == B.SOLO_EINVAL
    assert B.lib().solo_grads_destroy(None) == B.SOLO_OK
    assert B.lib().solo_grads_workspace(None, C.byref(C.c_size_t())) == B.SOLO_EINVAL


def test_lists_without_sizes_data_or_type_are_refused(B):
    L = B.lib()
    for bad in (B.GradList(None, 16, 0), B.GradList(None, None, 0)):
        p = C.byref(bad)
        assert L.solo_grad_norm(p, 2, 1.0, 16, None, 16, None) == B.SOLO_EINVAL
        assert L.solo_grad_clip(p, p, 16, 1, 2, 1.0, 1.0, None) == B.SOLO_EINVAL
        assert L.solo_grad_clip_norm(p, p, 2, 1.0, 1.0, 16, None, 16, None) == B.SOLO_EINVAL
        assert L.solo_grad_accumulate(p, p, 1.0, 0, -1, None, None, None, None) == B.SOLO_EINVAL
    assert L.solo_grad_norm(None, 2, 1.0, 16, None, 16, None) == B.SOLO_EINVAL


def test_python_checks_come_before_the_library(B):
    import torch
    with pytest.raises(ValueError):
        B.GradSet([])
    with pytest.raises(ValueError):
        B.GradSet([torch.zeros(4)])                       # not on a GPU
    with pytest.raises(ValueError):
        B.GradSet([torch.zeros(4, dtype=torch.float64)])
    for p in (0, 3, -1, "2"):
        with pytest.raises(ValueError):
            B._norm_type(p)
    assert (B._norm_type(2.0), B._norm_type(1), B._norm_type(float("inf"))) == (2, 1, 0)


def test_rows_are_checked(B):
    L, n = B.lib(), C.c_size_t()
    for tokens, width in ((-1, 8), (1, 0), (1, (1 << 24) + 1), ((1 << 40) + 1, 8)):
        assert L.solo_grad_rows_workspace(tokens, width, C.byref(n)) == B.SOLO_EINVAL
    assert L.solo_grad_rows_workspace(5, 8, None) == B.SOLO_EINVAL
    assert L.solo_grad_rows_workspace(0, 8, C.byref(n)) == B.SOLO_OK
    sizes = []
    for tokens in (1, 64, 2000, 65536, 65537, 1 << 40):
        assert L.solo_grad_rows_workspace(tokens, 768, C.byref(n)) == B.SOLO_OK
        sizes.append(n.value)
    assert sizes == sorted(sizes) and sizes[-1] == sizes[-3]              # one chunk's workspace serves all

    good = dict(acc=256, num_rows=5, width=8, tokens=256, token_bytes=8, grad_dtype=0, grad=256, grad_stride=8, num_tokens=3)
    call = lambda ws=256, scale=1.0, **kw: L.solo_grad_accumulate_rows(C.byref(B.GradRows(*{**good, **kw}.values())), scale, ws, None)  # noqa: E731
    for kw in (dict(acc=None), dict(num_rows=0), dict(num_rows=1 << 31), dict(width=0), dict(width=(1 << 24) + 1), dict(tokens=None),
               dict(token_bytes=2), dict(grad_dtype=3), dict(grad_dtype=-1), dict(grad=None), dict(grad_stride=-8), dict(num_tokens=-1),
               dict(num_tokens=(1 << 40) + 1), dict(ws=None, num_tokens=100000), dict(scale=float("nan")), dict(scale=float("inf"))):
        assert call(**kw) == B.SOLO_EINVAL, kw
    for kw in (dict(acc=258), dict(tokens=260), dict(grad=258), dict(ws=264), dict(token_bytes=4, tokens=258)):
        assert call(**kw) == B.SOLO_EALIGN, kw
    assert call(num_tokens=0, tokens=None, grad=None, ws=None) == B.SOLO_OK
    assert L.solo_grad_accumulate_rows(None, 1.0, 256, None) == B.SOLO_EINVAL
