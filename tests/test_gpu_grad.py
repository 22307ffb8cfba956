"""Gradient lists before the step (norm, clipping, accumulation) against their formulas in 64 bits.

Tolerances.  u = 2^-24 is half a step of binary32, h = finfo(t).eps / 2 half a step of an output type.
  norm, p = 2   a thread adds at most 16 squares to each of two binary32 sums and joins them: 17 u on a sum of non-negative terms,
                halved by the root, plus u for the result: 9.5 u
  norm, p = 1   17 u and u: 18 u
  norm, max     one rounding: u
  clip          factor u, product u, result h (the last two are one if the result is binary32); with a norm of its own 9.5 u more
  accumulate    one rounding: u
Second-order terms are covered by rounding these up to whole u; the smallest subnormal's half is added where results may be
subnormal.
"""
import math

import pytest
import torch

from paper_2505_00347_b200 import synth

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF_SUBNORMAL = {torch.float32: 2.0 ** -150, torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}
NORM_TOL = {1: 18 * U, 2: 10 * U, math.inf: U}
TILE = 8192
RAGGED = (0, 1, 7, 8, 9, 255, 1000, TILE - 1, TILE, TILE + 1, 0, 0, 3 * TILE + 77, 300, 20 * TILE, 0)

LONG = RAGGED + (1500 * TILE + 5, 0, 17)        # more tiles than CTAs
LISTS = {"short": RAGGED, "long": LONG}


def lib():
    from paper_2505_00347_b200 import binding
    return binding


class Slab:
    """Tensors in one buffer, `gap` elements between them that have to stay as they are."""

    def __init__(self, sizes, dtype, shift=0, gap=8, fill=-7.0):
        starts, at = [], 64 + shift
        for n in sizes:
            starts.append(at)
            at += (n + gap + 7) // 8 * 8
        self.buf = torch.full((at + 64,), fill, dtype=dtype, device="cuda")
        self.views = [self.buf[a:a + n] for a, n in zip(starts, sizes)]
        self.inside = torch.zeros(at + 64, dtype=torch.bool, device="cuda")
        for a, n in zip(starts, sizes):
            self.inside[a:a + n] = True
        self.fill = fill

    def random(self, seed, loud=1.0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        for i, v in enumerate(self.views):
            v.copy_(torch.randn(v.numel(), generator=g, device="cuda") * (loud * 10.0 ** -(i % 5)))
        return self

    def flat(self):
        return self.buf[self.inside].double()

    def untouched(self):
        return bool((self.buf[~self.inside] == self.fill).all())


def norm64(x, p):
    x = x.double().abs()
    if x.numel() == 0:
        return 0.0
    return float(x.max() if p == math.inf else x.sum() if p == 1 else x.square().sum().sqrt())


def near(got, want, rel, tiny=0.0):
    got, want = got.double(), want.double()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    inf = torch.isinf(want)
    assert torch.equal(got[inf], want[inf])
    fine = torch.isfinite(want)
    off = (got[fine] - want[fine]).abs() - rel * want[fine].abs() - tiny
    assert off.numel() == 0 or float(off.max()) <= 0, (float(off.max()), got[fine][off.argmax()], want[fine][off.argmax()])


def near_number(got, want, rel):
    near(got.view(-1), torch.tensor([want], dtype=torch.float64, device=got.device), rel)


@pytest.mark.parametrize("p", [1, 2, math.inf])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("shift", [0, 1, 4])
def test_norm(p, dtype, shift):
    B = lib()
    for sizes in (RAGGED, LONG, (5,), (0,), (0, 0, 3), (TILE,), (2 * TILE + 3,) * 40, (2 * TILE + 3,) * 400, (700,) * 3000):
        s = Slab(sizes, DT[dtype], shift).random(3)
        total, per = B.solo_grad_norm(B.GradSet(s.views), norm_type=p, scale=-0.75, per_tensor=True)
        again = B.solo_grad_norm(B.GradSet(s.views), norm_type=p, scale=-0.75)
        assert total.shape == (1,) and per.shape == (len(sizes),) and total.dtype == torch.float32
        near_number(total, 0.75 * norm64(s.flat(), p), NORM_TOL[p])
        near_number(again, 0.75 * norm64(s.flat(), p), NORM_TOL[p])
        near(per, torch.tensor([0.75 * norm64(v, p) for v in s.views], device="cuda", dtype=torch.float64), NORM_TOL[p])
        assert s.untouched()


@pytest.mark.parametrize("p", [1, 2, math.inf])
def test_norm_of_values_whose_squares_binary32_cannot_hold(p):
    B = lib()
    n = 3 * TILE + 100
    for value in (1e30, 3e38, 1e-30, 1e-38, 1e-45, 0.0):
        for where in ("everywhere", "one", "tail"):
            for dtype in (torch.float32, torch.bfloat16):
                x = torch.zeros(n, device="cuda", dtype=dtype)
                if where == "everywhere":
                    x.fill_(value)
                else:
                    x[5 if where == "one" else n - 1] = -value
                got = B.solo_grad_norm(B.GradSet([x]), norm_type=p)
                want = norm64(x, p)
                want = math.inf if want > torch.finfo(torch.float32).max else want
                near(got, torch.tensor([want], device="cuda", dtype=torch.float64), NORM_TOL[p], 2.0 ** -150)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("p", [1, 2, math.inf])
def test_nan_and_infinity_come_through(p, dtype):
    B = lib()
    for bad in (math.nan, math.inf, -math.inf):
        for at in (0, TILE - 1, 2 * TILE + 9):
            x = torch.ones(2 * TILE + 10, device="cuda", dtype=DT[dtype])
            y = torch.ones(100, device="cuda", dtype=DT[dtype])
            x[at] = bad
            out = [torch.zeros_like(v) for v in (y, x)]
            total, per = B.solo_grad_clip_norm(B.GradSet([y, x]), 1.0, dst=B.GradSet(out), norm_type=p, per_tensor=True)
            same = math.isnan if math.isnan(bad) else math.isinf
            assert same(float(total)) and same(float(per[1])) and math.isfinite(float(per[0]))
            want = [v.double() * (math.nan if math.isnan(bad) else 0.0) for v in (y, x)]     # 0 * inf = NaN
            for o, w in zip(out, want):
                near(o, w, 0.0)


CLIP_PAIRS = [("f32", "f32"), ("f32", "bf16"), ("f32", "f16"), ("bf16", "bf16"), ("bf16", "f32"), ("bf16", "f16"), ("f16", "f16"),
              ("f16", "bf16"), ("f16", "f32")]


@pytest.mark.parametrize("src,dst", CLIP_PAIRS)
@pytest.mark.parametrize("shifts", [(0, 0), (1, 1), (0, 3), (4, 0)])
def test_clip(src, dst, shifts):
    B = lib()
    s = Slab(RAGGED, DT[src], shifts[0]).random(5)
    gs = B.GradSet(s.views)
    h = 0.0 if dst == "f32" else torch.finfo(DT[dst]).eps / 2
    for p in (1, 2, math.inf):
        parts = torch.tensor([3.0, 4.0, 0.0, 0.5], device="cuda")
        N = norm64(parts, p)
        for max_norm, scale in ((0.25 * N, 1.0), (3.0 * N, -0.5), (0.0, 1.0)):
            d = Slab(RAGGED, DT[dst], shifts[1])
            f = scale * min(1.0, float(torch.tensor(max_norm)) / (N + 1e-6))
            B.solo_grad_clip(gs, parts, max_norm, dst=B.GradSet(d.views), norm_type=p, scale=scale)
            near(d.flat(), s.flat() * f, h + 3 * U, HALF_SUBNORMAL[DT[dst]])
            assert d.untouched() and s.untouched()
    d = Slab(RAGGED, DT[dst], shifts[1])
    B.solo_grad_clip(gs, None, 0.0, dst=B.GradSet(d.views), scale=2.0 ** -3)
    near(d.flat(), s.flat() * 2.0 ** -3, h, HALF_SUBNORMAL[DT[dst]])


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("shift", [0, 1])
@pytest.mark.parametrize("sizes", LISTS)
def test_clip_norm_in_place(dtype, shift, sizes):
    B = lib()
    h = 0.0 if dtype == "f32" else torch.finfo(DT[dtype]).eps / 2
    for p in (1, 2, math.inf):
        s = Slab(LISTS[sizes], DT[dtype], shift).random(9)
        before, N = s.flat(), norm64(s.flat(), p)
        total = B.solo_grad_clip_norm(B.GradSet(s.views), 2.0 * N, norm_type=p)           # below the limit: as it was
        assert torch.equal(s.flat(), before)
        near_number(total, N, NORM_TOL[p])
        limit = float(torch.tensor(0.3 * N))
        B.solo_grad_clip_norm(B.GradSet(s.views), limit, norm_type=p)
        near(s.flat(), before * (limit / (N + 1e-6)), h + 3 * U + NORM_TOL[p], HALF_SUBNORMAL[DT[dtype]])
        assert s.untouched()


@pytest.mark.parametrize("src,dst", CLIP_PAIRS)
@pytest.mark.parametrize("sizes", LISTS)
def test_clip_norm_into_another_list(src, dst, sizes):
    B = lib()
    h = 0.0 if dst == "f32" else torch.finfo(DT[dst]).eps / 2
    for p in (1, 2, math.inf):
        for shifts in ((0, 0), (0, 4), (3, 3)):
            s, d = Slab(LISTS[sizes], DT[src], shifts[0]).random(10), Slab(LISTS[sizes], DT[dst], shifts[1])
            N = 0.125 * norm64(s.flat(), p)
            limit = float(torch.tensor(0.7 * N))
            total, per = B.solo_grad_clip_norm(B.GradSet(s.views), limit, dst=B.GradSet(d.views), norm_type=p, scale=0.125, per_tensor=True)
            near_number(total, N, NORM_TOL[p])
            near(per, torch.tensor([0.125 * norm64(v, p) for v in s.views], device="cuda", dtype=torch.float64), NORM_TOL[p])
            near(d.flat(), s.flat() * (0.125 * limit / (N + 1e-6)), h + 3 * U + NORM_TOL[p], HALF_SUBNORMAL[DT[dst]])
            assert s.untouched() and d.untouched()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("shifts", [(0, 0), (1, 1), (0, 3), (4, 0)])
@pytest.mark.parametrize("sizes", LISTS)
def test_accumulate(dtype, shifts, sizes):
    B = lib()
    acc = Slab(LISTS[sizes], torch.float32, shifts[0]).random(11)
    g = Slab(LISTS[sizes], DT[dtype], shifts[1]).random(12)
    al, gl = B.GradSet(acc.views), B.GradSet(g.views)
    for p in (None, 1, 2, math.inf):
        for first in (False, True):
            want = g.flat() * 0.375 + (0.0 if first else acc.flat())
            if first:
                for v in acc.views:
                    v.fill_(math.nan)                                   # not read
            got = B.solo_grad_accumulate(al, gl, scale=0.375, first=first, norm_type=p, per_tensor=p is not None)
            near(acc.flat(), want, U * (1 + 2.0 ** -20), 2.0 ** -150)
            if p is None:
                assert got is None
            else:
                near_number(got[0], norm64(acc.flat(), p), NORM_TOL[p])
                near(got[1], torch.tensor([norm64(v, p) for v in acc.views], device="cuda", dtype=torch.float64), NORM_TOL[p])
            assert acc.untouched() and g.untouched()


def test_norms_of_shards_make_the_norm_of_the_whole():
    from paper_2505_00347_b200 import shard
    B = lib()
    sizes = [n for n in RAGGED if n]
    s = Slab(sizes, torch.bfloat16).random(21)
    limit = 0.5
    for p in (1, 2, math.inf):
        norms, lists = [], []
        for pieces in shard.partition(sizes, 128, 3):
            lists.append(B.GradSet([s.views[q.tensor][q.elem_offset:q.elem_offset + q.numel] for q in pieces]))
            norms.append(B.solo_grad_norm(lists[-1], norm_type=p))
        before, N = s.flat(), norm64(s.flat(), p)
        for gl in lists:
            B.solo_grad_clip(gl, torch.cat(norms), limit, norm_type=p)
        near(s.flat(), before * min(1.0, limit / (N + 1e-6)), 2.0 ** -8 + 4 * U + NORM_TOL[p], HALF_SUBNORMAL[torch.bfloat16])
        s.random(22)


def test_accumulate_clip_and_step_together():
    """Three micro-batches, the clip by the last one's norm and the optimizer step, against the step on gradients made in torch."""
    B = lib()
    sizes = (2048 * 9 + 700, 643, 2048 * 4, 77)
    w = synth.workload(2, sizes=sizes)
    micro = [[synth.make_grad(w, i, t).cuda() for i in range(len(sizes))] for t in (1, 2, 3)]
    acc = [torch.full((n,), math.nan, device="cuda") for n in sizes]
    al = B.GradSet(acc)
    for t, g in enumerate(micro):
        norm = B.solo_grad_accumulate(al, B.GradSet(g), scale=1.0 / 3.0, first=t == 0, norm_type=2 if t == 2 else None)
    third = float(torch.tensor(1.0 / 3.0))
    grads = [torch.zeros(n, device="cuda", dtype=torch.bfloat16) for n in sizes]
    want = [sum(m[i].double() for m in micro) * third for i in range(len(sizes))]
    N = math.sqrt(sum(float(x.square().sum()) for x in want))
    limit = float(torch.tensor(0.25 * N))                                # the clip does something
    B.solo_grad_clip(al, norm, limit, dst=B.GradSet(grads))
    size = [sum(m[i].double().abs() for m in micro) * third for i in range(len(sizes))]
    for g, x, a in zip(grads, want, size):
        # three roundings of partial sums, none larger than the sum of magnitudes
        off = (g.double() - x * (limit / (N + 1e-6))).abs()
        assert bool((off <= x.abs() * (limit / N) * (2.0 ** -8 + 16 * U) + 4 * U * a * (limit / N)).all())
    p1 = [synth.make_param(w, i).cuda() for i in range(len(sizes))]
    p2 = [p.clone() for p in p1]
    h = B.hyper(lr=1e-3, beta1=0.6, weight_decay=0.01, seed=5)
    s1, s2 = B.State(list(sizes), 3, 3), B.State(list(sizes), 3, 3)
    B.solo_multi_step(B.TensorSet(p1, grads, s1), h, 1)
    B.solo_multi_step(B.TensorSet(p2, [g.clone() for g in grads], s2), h, 1)
    for a, b in zip(p1, p2):
        assert torch.equal(a, b)
    assert torch.equal(s1.raw_get("codes_v"), s2.raw_get("codes_v"))


def test_on_another_stream_and_in_graphs():
    """Calls on two streams at once share no memory; a captured pass replays on new data, beside another graph of the same list."""
    B = lib()
    sizes = (TILE * 50 + 3, 100, 0, TILE * 7)
    s = Slab(sizes, torch.bfloat16).random(31)
    gs = B.GradSet(s.views)
    torch.cuda.synchronize()
    side = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = []
    for k in range(20):
        with torch.cuda.stream(side[k % 2]):
            got.append(B.solo_grad_norm(gs, norm_type=2 if k % 2 else 1))
    torch.cuda.synchronize()
    for k in range(2, 20):
        assert torch.equal(got[k], got[k - 2])
    graphs, outs = [], []
    for k in range(2):
        d = Slab(sizes, torch.float32)
        dl = B.GradSet(d.views)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            total = B.solo_grad_clip_norm(gs, 0.125 * (k + 1), dst=dl)
        graphs.append(g)
        outs.append((d, dl, total))
    s.random(33)
    torch.cuda.synchronize()
    for _ in range(10):
        for k in range(2):
            with torch.cuda.stream(side[k]):
                graphs[k].replay()
    torch.cuda.synchronize()
    N = norm64(s.flat(), 2)
    for k, (d, _, total) in enumerate(outs):
        near_number(total, N, NORM_TOL[2])
        near(d.flat(), s.flat() * min(1.0, 0.125 * (k + 1) / (N + 1e-6)), 12 * U, 2.0 ** -150)


def test_captured_norms_of_every_tensor_and_many_parts():
    B = lib()
    for sizes in (RAGGED[:6], LONG):
        s, acc = Slab(sizes, torch.float16).random(51), Slab(sizes, torch.float32).random(52)
        gs, al = B.GradSet(s.views), B.GradSet(acc.views)
        eager = B.solo_grad_norm(gs, per_tensor=True)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            total, per = B.solo_grad_norm(gs, per_tensor=True)
            after, after_per = B.solo_grad_accumulate(al, gs, scale=0.5, norm_type=1, per_tensor=True)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(total, eager[0]) and torch.equal(per, eager[1])
        for seed in (53, 54):
            s.random(seed)
            graph.replay()
            torch.cuda.synchronize()
            near_number(total, norm64(s.flat(), 2), NORM_TOL[2])
            near(per, torch.tensor([norm64(v, 2) for v in s.views], device="cuda", dtype=torch.float64), NORM_TOL[2])
            near_number(after, norm64(acc.flat(), 1), NORM_TOL[1])
            near(after_per, torch.tensor([norm64(v, 1) for v in acc.views], device="cuda", dtype=torch.float64), NORM_TOL[1])
        assert torch.equal(B.solo_grad_norm(gs, per_tensor=True)[1], per)             # and outside of it again
    x = torch.ones(TILE + 1, device="cuda")
    parts = torch.rand(5000, device="cuda")
    for p in (1, 2, math.inf):
        y = torch.empty_like(x)
        B.solo_grad_clip(B.GradSet([x]), parts, 0.25, dst=B.GradSet([y]), norm_type=p)
        near(y, x.double() * (0.25 / (norm64(parts, p) + 1e-6)), 3 * U)


def test_threads_take_turns():
    """Several threads on one stream and several streams of one list: the last CTA's count and the second launches keep apart."""
    import threading
    B = lib()
    sizes = (TILE * 30 + 5, 9, 700) * 8
    s = Slab(sizes, torch.float16).random(41)
    gs = B.GradSet(s.views)
    want = {p: norm64(s.flat(), p) for p in (1, 2, math.inf)}
    each = {p: torch.tensor([norm64(v, p) for v in s.views], device="cuda", dtype=torch.float64) for p in want}
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    results, errors = [], []

    def work(k):
        try:
            with torch.cuda.stream(streams[k % 2]):
                for i in range(60):
                    p = (1, 2, math.inf)[(k + i) % 3]
                    per = (k + i) % 2 == 0
                    results.append((p, per, B.solo_grad_norm(gs, norm_type=p, per_tensor=per)))
        except Exception as e:                                            # noqa: BLE001
            errors.append(e)

    threads = [threading.Thread(target=work, args=(k,)) for k in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not errors and len(results) == 240
    for p, per, r in results:
        near_number(r[0] if per else r, want[p], NORM_TOL[p])
        if per:
            near(r[1], each[p], NORM_TOL[p])


def test_an_accumulator_as_its_own_gradient_and_lists_made_while_capturing():
    B = lib()
    x = torch.randn(3 * TILE + 11, device="cuda")
    gs, before = B.GradSet([x]), x.clone()
    B.solo_grad_accumulate(gs, gs, scale=0.5)
    near(x, before.double() * 1.5, U)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        with pytest.raises(B.SoloError) as e:
            arr, h = (B.C.c_int64 * 1)(4), B.C.c_void_p()
            B._check(B.lib().solo_grads_create(arr, 1, gs.geom.data_ptr(), B._stream(), B.C.byref(h)), "solo_grads_create")
        del gs                                                          # nothing of a list's end disturbs a capture
    assert e.value.status == B.SOLO_EINVAL
    graph.replay()
    torch.cuda.synchronize()


def test_a_tensor_beyond_32_bit_offsets():
    B = lib()
    n = (1 << 31) + 12345
    x = torch.zeros(n, device="cuda", dtype=torch.bfloat16)
    x[-1] = 3.0
    x[0] = 4.0
    gs = B.GradSet([x])
    assert float(B.solo_grad_norm(gs)) == 5.0
    acc = torch.zeros(n, device="cuda")
    assert float(B.solo_grad_accumulate(B.GradSet([acc]), gs, scale=2.0, norm_type=1)) == 14.0
    assert float(acc[-1]) == 6.0 and float(acc[0]) == 8.0
    B.solo_grad_clip(gs, torch.tensor([4.0], device="cuda"), 2.0)
    assert float(x[-1]) == 1.5


def test_refusals():
    B = lib()
    x, y = torch.ones(100, device="cuda"), torch.ones(101, device="cuda")
    a, b = B.GradSet([x]), B.GradSet([y])
    half = B.GradSet([x.half()])
    one = torch.ones(1, device="cuda")

    def refused(status, call):
        with pytest.raises(B.SoloError) as e:
            call()
        assert e.value.status == status

    refused(B.SOLO_ESTATE, lambda: B.solo_grad_clip(a, one, 1.0, dst=b))
    refused(B.SOLO_ESTATE, lambda: B.solo_grad_accumulate(a, b))
    refused(B.SOLO_EINVAL, lambda: B.solo_grad_accumulate(half, a))            # accumulators are fp32
    for bad in (-1.0, math.nan, math.inf):
        refused(B.SOLO_EINVAL, lambda: B.solo_grad_clip(a, one, bad))
        refused(B.SOLO_EINVAL, lambda: B.solo_grad_clip_norm(a, bad))
    for bad in (math.nan, math.inf):
        refused(B.SOLO_EINVAL, lambda: B.solo_grad_norm(a, scale=bad))
        refused(B.SOLO_EINVAL, lambda: B.solo_grad_clip(a, one, 1.0, scale=bad))
        refused(B.SOLO_EINVAL, lambda: B.solo_grad_clip_norm(a, 1.0, scale=bad))
        refused(B.SOLO_EINVAL, lambda: B.solo_grad_accumulate(a, a, scale=bad))
    for bad in (B.GradSet([x, x]), B.GradSet([x[:50], x[40:]])):               # memory written twice
        with pytest.raises(ValueError):
            B.solo_grad_clip(bad, one, 1.0)
        with pytest.raises(ValueError):
            B.solo_grad_clip_norm(bad, 1.0)
        with pytest.raises(ValueError):
            B.solo_grad_accumulate(bad, bad)
    assert float(B.solo_grad_norm(B.GradSet([x, x]), norm_type=1)) == 200.0
    z = torch.ones(300, device="cuda")
    lists = {k: B.GradSet(v) for k, v in dict(first=[z[:100], z[200:]], swapped=[z[200:], z[:100]],
                                              late=[z[4:104], z[200:]], between=[z[100:150], z[150:200]]).items()}
    for other in ("swapped", "late"):                                            # other tensors, some of the same memory
        for _ in range(2):
            with pytest.raises(ValueError):
                B.solo_grad_clip(lists["first"], None, 0.0, dst=lists[other])
            with pytest.raises(ValueError):
                B.solo_grad_accumulate(lists[other], lists["first"])
    again = B.GradSet([z[:100], z[200:]])
    for _ in range(2):
        B.solo_grad_clip(lists["first"], None, 0.0, dst=again, scale=2.0)          # the same tensors
        B.solo_grad_clip(B.GradSet([z[:50], z[200:250]]), None, 0.0, dst=lists["between"], scale=0.5)    # between them
    assert z[:100].eq(4).all() and z[200:].eq(4).all() and z[100:200].eq(2).all()
    B.solo_grad_clip(B.GradSet([z[:50], z[:50]]), None, 0.0, dst=lists["between"])  # read twice: no matter
    assert z[100:200].eq(4).all()
    for norms in (2.0, one.cpu(), one.double(), torch.ones(2, 2, device="cuda")[:, 0], one[:0]):
        with pytest.raises(ValueError):
            B.solo_grad_clip(a, norms, 1.0)
    with pytest.raises(ValueError):
        B.GradSet([x, x.half()])
    with pytest.raises(ValueError):
        B.GradSet([torch.ones(4, 4, device="cuda")[:, 0]])
    with pytest.raises(ValueError):
        B.GradSet([torch.ones(4, device="cuda", dtype=torch.int32)])
    ws = torch.zeros(a._workspace_bytes // 4 + 8, device="cuda")
    out = torch.zeros(1, device="cuda")
    L, p = B.lib(), B.C.byref(a.desc)
    assert L.solo_grad_norm(p, 2, 1.0, out.data_ptr(), None, ws.data_ptr() + 4, None) == B.SOLO_EALIGN
    assert L.solo_grad_norm(p, 3, 1.0, out.data_ptr(), None, ws.data_ptr(), None) == B.SOLO_EINVAL
    assert L.solo_grad_norm(p, 2, 1.0, None, None, ws.data_ptr(), None) == B.SOLO_EINVAL
    assert L.solo_grad_norm(p, 2, 1.0, out.data_ptr(), None, None, None) == B.SOLO_EINVAL
    assert L.solo_grad_clip(p, p, None, 1, 2, 1.0, 1.0, None) == B.SOLO_EINVAL
    assert L.solo_grad_clip(p, p, out.data_ptr(), -1, 2, 1.0, 1.0, None) == B.SOLO_EINVAL
    wrong = B.GradList(a.handle.value, a.ptrs.data_ptr(), 3)
    assert L.solo_grad_norm(B.C.byref(wrong), 2, 1.0, out.data_ptr(), None, ws.data_ptr(), None) == B.SOLO_EINVAL
    assert float(x.sum()) == 100.0


def test_norms_in_what_a_clip_writes():
    """Every CTA reads the norms for itself while others write: refused where they lie in dst, not beside or in what is only read."""
    B = lib()
    z = torch.ones(1000, device="cuda")
    far = torch.zeros(400, device="cuda")
    gs = B.GradSet([z[:100], z[200:300], z[400:400], z[500:700]])
    out = B.GradSet([far[:100], far[100:200], far[0:0], far[200:400]])
    for norms in (z[0:1], z[99:101], z[98:202], z[200:201], z[299:300], z[499:501], z[699:702], z[:900]):
        with pytest.raises(ValueError):
            B.solo_grad_clip(gs, norms, 0.5)
    assert bool((z == 1).all())
    B.solo_grad_clip(gs, z[99:101], 1.0, dst=out)                               # in the source, which is read alone
    near(far, torch.full_like(far, 1.0).double() / (math.sqrt(2.0) + 1e-6), 3 * U)
    beside = (z[100:101], z[300:400], z[400:401], z[499:500], z[700:702], z[999:])
    for k, norms in enumerate(beside):
        norms.fill_(1.0)
        want = z[0].double() * (0.5 / (math.sqrt(norms.numel()) + 1e-6))
        B.solo_grad_clip(gs, norms, 0.5)
        for part in (z[:100], z[200:300], z[500:700]):
            near(part, want.expand(part.shape), 4 * U * (k + 1))
        assert bool((norms == 1).all())


NO_MEMORY = r"""
#include <cstdlib>
#include <new>
static thread_local bool armed;
extern "C" void no_memory(int on) { armed = on != 0; }
void* operator new(std::size_t n) {
    void* const p = armed ? nullptr : std::malloc(n ? n : 1);
    if (!p) throw std::bad_alloc();
    return p;
}
void* operator new[](std::size_t n) { return operator new(n); }
void operator delete(void* p) noexcept { std::free(p); }
void operator delete[](void* p) noexcept { std::free(p); }
void operator delete(void* p, std::size_t) noexcept { std::free(p); }
void operator delete[](void* p, std::size_t) noexcept { std::free(p); }
"""

CALLS_WITHOUT_MEMORY = """
import ctypes as C, itertools, sys
sys.path.insert(0, sys.argv[1])
import torch
from paper_2505_00347_b200 import binding as B
no_memory = C.CDLL(sys.argv[2]).no_memory
types = (torch.float32, torch.bfloat16, torch.float16)
lists = [B.GradSet([torch.ones(9000, device="cuda", dtype=t), torch.ones(5, device="cuda", dtype=t)]) for t in types]
acc = B.GradSet([torch.ones(9000, device="cuda"), torch.ones(5, device="cuda")])
out = B.GradSet([torch.ones(9000, device="cuda"), torch.ones(5, device="cuda")])
ws = torch.zeros(lists[0]._workspace_bytes, dtype=torch.uint8, device="cuda")
norm = torch.zeros(1, device="cuda")
L, at, w, s = B.lib(), norm.data_ptr(), ws.data_ptr(), B._stream()
sizes, geom, handle = (C.c_int64 * 2)(9000, 5), torch.empty(5, dtype=torch.int64, device="cuda"), C.c_void_p()

def call(status, f, *args):
    torch.cuda.synchronize()
    no_memory(1)
    rc = f(*args)
    no_memory(0)
    assert rc == status, (f.__name__, rc)

call(B.SOLO_ENOMEM, L.solo_grads_create, sizes, 2, geom.data_ptr(), s, C.byref(handle))
assert not handle.value
for l, p in itertools.product(lists, (0, 1, 2)):
    call(B.SOLO_OK, L.solo_grad_norm, l._ref, p, 1.0, at, None, w, s)
    call(B.SOLO_OK, L.solo_grad_clip_norm, l._ref, out._ref, p, 1e9, 1.0, at, None, w, s)
    call(B.SOLO_OK, L.solo_grad_accumulate, acc._ref, l._ref, 1.0, 1, p, at, None, w, s)
    call(B.SOLO_OK, L.solo_grad_accumulate, acc._ref, l._ref, 1.0, 0, p, at, None, w, s)
torch.cuda.synchronize()
assert abs(float(norm) / (2.0 * 9005 ** 0.5) - 1) < 1e-6, float(norm)
print("done")
"""


def test_calls_without_host_memory(tmp_path):
    """Nothing throws: with no memory to be had, a list is refused and the other calls, which allocate nothing, run as ever."""
    import os
    import subprocess
    import sys
    shim, source = tmp_path / "no_memory.so", tmp_path / "no_memory.cpp"
    source.write_text(NO_MEMORY)
    subprocess.run(["g++", "-O1", "-shared", "-fPIC", "-o", str(shim), str(source)], check=True)
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", CALLS_WITHOUT_MEMORY, root, str(shim)], env={**os.environ, "LD_PRELOAD": str(shim)},
                       capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "done" in r.stdout, (r.returncode, r.stdout[-500:], r.stderr[-2000:])


def whole_numbers(n, seed, most=128):
    """Whole multiples of 2^-14 up to most 2^-14: bf16 holds them, and binary32 every sum of a few of them, so nothing is rounded."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randint(-most, most + 1, (n,), generator=g, device="cuda").float() * 2.0 ** -14).bfloat16()


def step_on(B, sizes, params, grads):
    """The optimizer's first step; parameters and state after it."""
    params, state = [p.clone() for p in params], B.State(list(sizes), 3, 3)
    B.solo_multi_step(B.TensorSet(params, grads, state), B.hyper(lr=1e-3, beta1=0.6, weight_decay=0.01, seed=5), 1)
    return params, [state.raw_get(k) for k in ("codes_m", "codes_v", "scale_m", "scale_v", "alpha")]


def same_step(a, b):
    for x, y in zip((*a[0], *a[1]), (*b[0], *b[1])):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))


@pytest.mark.parametrize("own_norm", [False, True])
def test_step_on_clipped_accumulators_and_on_gradients_made_in_torch(own_norm):
    """Accumulators of whole numbers hold exact sums; from the norm that the call returns, the clip is a factor in binary64, rounded
    to binary32, a product in binary32 and a rounding to bf16.  Torch makes the same gradients, bit for bit, and the same step."""
    B = lib()
    sizes = (2048 * 9 + 700, 643, 2048 * 4, 77)
    w = synth.workload(2, sizes=sizes)
    params = [synth.make_param(w, i).cuda() for i in range(len(sizes))]
    micro = [[whole_numbers(n, 10 * t + i) for i, n in enumerate(sizes)] for t in range(4)]
    acc = [torch.full((n,), math.nan, device="cuda") for n in sizes]
    grads = [torch.zeros(n, device="cuda", dtype=torch.bfloat16) for n in sizes]
    al, gl = B.GradSet(acc), B.GradSet(grads)
    for t, g in enumerate(micro):
        norm = B.solo_grad_accumulate(al, B.GradSet(g), scale=0.25, first=t == 0, norm_type=2 if t == 3 else None)
    sums = [sum(m[i].double() for m in micro) * 0.25 for i in range(len(sizes))]
    for a, x in zip(acc, sums):
        assert torch.equal(a.double(), x)
    N = math.sqrt(sum(float(x.square().sum()) for x in sums))
    near_number(norm, N, NORM_TOL[2])
    limit = float(torch.tensor(0.3 * N))
    if own_norm:
        norm = B.solo_grad_clip_norm(al, limit, dst=gl)
        near_number(norm, N, NORM_TOL[2])
        return same_step(step_on(B, sizes, params, grads), step_on(B, sizes, params, made_in_torch(sums, grads, limit, N)))
    B.solo_grad_clip(al, norm, limit, dst=gl)
    f = torch.tensor(min(1.0, limit / (float(norm) + 1e-6)), dtype=torch.float32, device="cuda")
    want = [(x.float() * f).bfloat16() for x in sums]
    for g, x in zip(grads, want):
        assert torch.equal(g, x) and int(x.count_nonzero()) > 0
    same_step(step_on(B, sizes, params, grads), step_on(B, sizes, params, want))


def made_in_torch(sums, grads, limit, N):
    """The clip's own norm is in binary64 and rounded for the caller only, so its factor is one of a few next to this one."""
    f = torch.tensor(limit / (N + 1e-6), dtype=torch.float32, device="cuda")
    for steps in range(-12, 13):                                        # 10 u of the norm and a rounding: 11 u, 2 u a step
        at = (f.view(torch.int32) + steps).view(torch.float32)
        want = [(x.float() * at).bfloat16() for x in sums]
        if all(torch.equal(g, x) for g, x in zip(grads, want)):
            return want
    raise AssertionError("no factor near the formula's gives these gradients")
