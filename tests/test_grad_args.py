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


def test_rows_that_would_be_read_and_written_at_once_are_refused(B):
    """The accumulator and the workspace against each other, the tokens and the gradient's rows (of numbers, not of memory)."""
    n, width, rows = 2000, 8, 50                                # not the one-launch form: with a workspace
    size = C.c_size_t()
    assert B.lib().solo_grad_rows_workspace(n, width, C.byref(size)) == B.SOLO_OK and size.value
    at = dict(acc=1 << 20, tokens=2 << 20, grad=3 << 20, ws=4 << 20)
    bytes_of = dict(acc=rows * width * 4, tokens=n * 8, grad=((n - 1) * width + width) * 4, ws=size.value)

    def call(stride=width, n=n, **kw):
        p = {**at, **kw}
        return B.lib().solo_grad_accumulate_rows(C.byref(B.GradRows(p["acc"], rows, width, p["tokens"], 8, 0, p["grad"], stride, n)), 1.0, p["ws"], None)

    for a, b in (("acc", "tokens"), ("acc", "grad"), ("acc", "ws"), ("ws", "tokens"), ("ws", "grad")):
        for x, y in ((a, b), (b, a)):                           # x begins where y does, ends in it, or begins in its last bytes
            for place in (at[y], at[y] - bytes_of[x] // 16 * 16 + 16, at[y] + (bytes_of[y] - 1) // 16 * 16):
                assert call(**{x: place}) == B.SOLO_EINVAL, (x, y, place - at[y])
    gap = 64 * width                                            # acc within a gap, but for its first or its last bytes
    assert call(stride=gap, acc=at["grad"] + 5 * gap + width * 4 - 16) == B.SOLO_EINVAL
    assert call(stride=gap, acc=at["grad"] + 6 * gap * 4 - bytes_of["acc"] + 16) == B.SOLO_EINVAL
    assert call(stride=0, acc=at["grad"] + width * 4 - 16) == B.SOLO_EINVAL
    for stride, n_ in ((1 << 60, 3000), ((1 << 60) + 1, 2000), ((1 << 63) - 1, 2), ((1 << 62), 1 << 40)):
        assert call(stride=stride, n=n_) == B.SOLO_EINVAL, (stride, n_)


def test_few_rows_that_would_be_read_and_written_at_once_are_refused(B):
    rows = lambda acc, tokens, grad, n=3: B.lib().solo_grad_accumulate_rows(  # noqa: E731
        C.byref(B.GradRows(acc, 5, 8, tokens, 8, 1, grad, 8, n)), 1.0, None, None)
    for acc, tokens, grad in ((1024, 1024, 4096), (1024, 4096, 1024), (1024, 1024 + 152, 4096), (1024, 1024 - 16, 4096), (1024, 4096, 1024 + 158)):
        assert rows(acc, tokens, grad) == B.SOLO_EINVAL, (acc, tokens, grad)


def test_spans_that_share_memory(B):
    spans = [(10, 20), (20, 25), (40, 41), (60, 100)]
    taken = {x for a, b in spans for x in range(a, b)}
    for low in range(0, 110):
        for length in (1, 2, 4, 15, 40, 120):
            assert B._reaches_into(low, low + length, spans) == (not taken.isdisjoint(range(low, low + length))), (low, length)
    assert not B._reaches_into(0, 1 << 60, [])


def test_pointers_off_their_alignment_are_refused(B):
    """A list whose sizes are never looked at: pointers are refused before."""
    L = B.lib()
    p = lambda data=64: C.byref(B.GradList(64, data, 0))  # noqa: E731
    for off in (1, 2, 3):
        for per in (None, 64):
            assert L.solo_grad_norm(p(), 2, 1.0, 64 + off, per, 64, None) == B.SOLO_EALIGN
            assert L.solo_grad_clip_norm(p(), p(), 2, 1.0, 1.0, 64 + off, per, 64, None) == B.SOLO_EALIGN
            assert L.solo_grad_accumulate(p(), p(), 1.0, 0, 2, 64 + off, per, 64, None) == B.SOLO_EALIGN
        assert L.solo_grad_norm(p(), 2, 1.0, 64, 64 + off, 64, None) == B.SOLO_EALIGN
        assert L.solo_grad_clip_norm(p(), p(), 2, 1.0, 1.0, 64, 64 + off, 64, None) == B.SOLO_EALIGN
        assert L.solo_grad_accumulate(p(), p(), 1.0, 1, 1, 64, 64 + off, 64, None) == B.SOLO_EALIGN
        assert L.solo_grad_clip(p(), p(), 64 + off, 1, 2, 1.0, 1.0, None) == B.SOLO_EALIGN
    for data in (65, 66, 68, 71):
        assert L.solo_grad_norm(p(data), 2, 1.0, 64, None, 64, None) == B.SOLO_EALIGN
        assert L.solo_grad_clip(p(data), p(data), 64, 1, 2, 1.0, 1.0, None) == B.SOLO_EALIGN
        assert L.solo_grad_clip_norm(p(data), p(data), 2, 1.0, 1.0, 64, None, 64, None) == B.SOLO_EALIGN
        assert L.solo_grad_accumulate(p(data), p(data), 1.0, 0, -1, None, None, None, None) == B.SOLO_EALIGN
    for size in (2, 4):
        B._aligned([0, 64, 64 + size], size)
        for off in range(1, size):
            with pytest.raises(ValueError):
                B._aligned([0, 64 + off, 128], size)


def test_what_a_list_knows_of_others_goes_with_them(B):
    """A list of accumulators that sees new gradients in every step, between its own tensors, keeps nothing of the old ones."""
    import gc
    import weakref

    def gs(spans, dtype=0):
        g = object.__new__(B.GradSet)
        g._spans, g._in_order, g._apart, g.dtype, g._ref = spans, sorted(spans), True, dtype, spans
        g._low, g._high, g._clear_of = min(a for a, _ in spans), max(b for _, b in spans), weakref.WeakSet()
        return g

    acc = gs([(0, 10), (1000, 1010)])
    kept = [gs([(20, 30), (40 + k, 50 + k)]) for k in range(3)]
    for other in kept * 2:
        assert B._written(acc, other) is acc._ref
    assert len(acc._clear_of) == 3
    for k in range(200):
        B._written(acc, gs([(100 + k, 105 + k)]))
        with pytest.raises(ValueError):
            B._written(acc, gs([(100, 105), (5, 15)]))
    gc.collect()
    assert len(acc._clear_of) == 3 and len(list(acc._clear_of)) == 3
    del kept, other
    gc.collect()
    assert len(acc._clear_of) == 0
    assert B._written(acc, gs([(0, 10), (1000, 1010)])) is acc._ref             # the same tensors: in place


def test_workspaces_belong_to_streams_of_the_lists_device(B, monkeypatch):
    """With another device current the call is refused; what was zeroed for it must not stay under its stream's handle."""
    import torch
    g = object.__new__(B.GradSet)
    g._workspaces, g._workspace_bytes, g.device = {}, 64, torch.device("cuda", 0)
    made = []
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    monkeypatch.setattr(torch, "zeros", lambda n, dtype, device: made.append(device) or object())
    monkeypatch.setattr(B, "_current_device", lambda: 1)
    g._workspace(0)
    assert g._workspaces == {}
    monkeypatch.setattr(B, "_current_device", lambda: 0)
    ws = g._workspace(0)
    assert g._workspace(0) is ws and g._workspace(7) is not ws and len(g._workspaces) == 2 and len(made) == 3
