"""The gradient rows of an embedding against an addition in 64 bits.

Tolerance.  u = 2^-24.  A row of the result is acc + scale * S with one rounding for every 65,536 tokens, S the sum of a
token's rows: sums of fewer than 96 rows in binary32 (94 additions and one rounding to binary32 after the binary64 join: 95 u of the
sum of magnitudes A).  So |error| <= pieces * u * (|acc| + |scale| A) + 96 u |scale| A.
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
CHUNK = 65536
DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def lib():
    from paper_2505_00347_b200 import binding
    return binding


def tokens_of(kind, n, rows, seed=1):
    g = torch.Generator().manual_seed(seed)
    if kind == "same":
        return torch.full((n,), rows // 2)
    if kind == "distinct":
        return torch.randperm(max(n, rows), generator=g)[:n] % rows
    if kind == "sorted":
        return torch.randint(0, rows, (n,), generator=g).sort().values
    if kind == "outside":
        return torch.where(torch.rand(n, generator=g) < 0.5, -1 - torch.randint(0, 1000, (n,), generator=g), rows + torch.randint(0, 1 << 20, (n,), generator=g))
    if kind == "few":                                   # a few frequent tokens, padding between
        return torch.randint(0, 5, (n,), generator=g) * (rows // 4) - 1
    assert kind == "skewed"
    return (rows * torch.rand(n, generator=g) ** 4).long().clamp(0, rows - 1)


def check(acc, tok, grad, scale, **kw):
    B = lib()
    rows = acc.shape[0]
    g = grad.reshape(-1, acc.shape[1])
    t = tok.reshape(-1).long()
    keep = torch.nonzero((t >= 0) & (t < rows)).view(-1)
    want = acc.double()
    size = want.abs()
    s = float(torch.tensor(scale, dtype=torch.float32))
    want.index_add_(0, t[keep], g[keep].double() * s)
    added = torch.zeros_like(want).index_add_(0, t[keep], g[keep].double().abs() * abs(s))
    before = acc.clone()
    B.solo_grad_accumulate_rows(acc, tok, grad, scale=scale)
    chunks = -(-t.numel() // CHUNK)
    off = (acc.double() - want).abs() - chunks * U * (size + added) - 96 * U * added - 2.0 ** -149
    assert float(off.max()) <= 0, float(off.max())
    named = torch.zeros(rows, dtype=torch.bool, device="cuda")
    named[t[keep]] = True
    assert torch.equal(acc[~named], before[~named])
    return acc


@pytest.mark.parametrize("kind", ["same", "distinct", "sorted", "outside", "few", "skewed"])
@pytest.mark.parametrize("n", [1, 2, 31, 33, 63, 64, 65, 95, 96, 97, 128, 161, 1000, 1025, 2048, 2049, 4093, 4096, 4097, 5000, 16385, 65536])
def test_token_patterns(kind, n):
    gen = torch.Generator(device="cuda").manual_seed(n)
    for rows, width in ((50257, 16), (1000, 24), (3, 5), (1, 8)):
        acc = torch.randn(rows, width, generator=gen, device="cuda")
        grad = torch.randn(n, width, generator=gen, device="cuda").bfloat16()
        tok = tokens_of(kind, n, rows).cuda()
        check(acc, tok if n % 2 else tok.int(), grad, -0.375)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("width", [1, 7, 8, 17, 768, 2048, 2056, 4096, 5001])
def test_widths_and_types(dtype, width):
    gen = torch.Generator(device="cuda").manual_seed(width)
    for n in (1, 300, 3000):
        for shift in (0, 1, 8):
            base = torch.empty(shift + n * width, device="cuda", dtype=DT[dtype])[shift:]
            grad = base.view(n, width)
            grad.copy_(torch.randn(n, width, generator=gen, device="cuda"))
            acc = torch.randn(400 * width + shift, generator=gen, device="cuda")[shift:].view(400, width)
            check(acc, tokens_of("skewed", n, 400).cuda(), grad, 0.125)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n,width", [(6000, 4096), (6000, 4099), (20000, 1288), (65536, 300), (130000, 264)])
def test_more_rows_than_fill_the_gpu_once(dtype, n, width):
    gen = torch.Generator(device="cuda").manual_seed(width)
    for kind in ("same", "skewed", "few", "distinct"):
        acc = torch.randn(3000, width, generator=gen, device="cuda")
        grad = torch.empty(n, width, device="cuda", dtype=DT[dtype]).normal_(generator=gen)
        check(acc, tokens_of(kind, n, 3000).cuda(), grad, -1.5)


@pytest.mark.parametrize("over", [0, 1, 7, 8, 9, 15, 16, 17, 127, 128, 129, 136, 137, 256, 300])
def test_runs_over_the_borders_of_warps_and_ctas(over):
    """Runs that end `over` entries behind the 128th, 256th, ... entry of the sorted order, and what is left of them."""
    gen = torch.Generator(device="cuda").manual_seed(over)
    for lead in (0, 1, 120, 127):
        counts = [lead, 128 - lead + over, 3, 1, 250, 128 + over, 1, 1, 1, 700, 16, 16]
        tok = torch.repeat_interleave(torch.arange(len(counts)) * 2, torch.tensor(counts))
        tok = torch.cat([tok, torch.full((1100,), -1)])[torch.randperm(len(tok) + 1100, generator=torch.Generator().manual_seed(lead))]
        for width in (264, 7):
            grad = torch.randn(len(tok), width, generator=gen, device="cuda").half()
            check(torch.randn(30, width, generator=gen, device="cuda"), tok.cuda(), grad, 0.7)


def test_strides_and_shapes():
    gen = torch.Generator(device="cuda").manual_seed(4)
    for width, pad in ((64, 64), (64, 8), (64, 3), (5, 1)):
        grad = torch.randn(700, width + pad, generator=gen, device="cuda").half()[:, :width]
        check(torch.randn(90, width, generator=gen, device="cuda"), tokens_of("skewed", 700, 90).cuda(), grad, 1.0)
    one = torch.randn(1, 64, generator=gen, device="cuda").expand(700, 64)                # a row for all tokens
    check(torch.randn(90, 64, generator=gen, device="cuda"), tokens_of("skewed", 700, 90).cuda(), one, 1.0)
    grad = torch.randn(4, 175, 64, generator=gen, device="cuda")
    check(torch.randn(90, 64, generator=gen, device="cuda"), tokens_of("skewed", 700, 90).cuda().view(4, 175), grad, 1.0)


def test_more_tokens_than_one_sort_holds():
    gen = torch.Generator(device="cuda").manual_seed(5)
    for n in (CHUNK + 1, 2 * CHUNK + 12345):
        for kind in ("same", "skewed", "few"):
            acc = torch.randn(150000, 8, generator=gen, device="cuda")
            check(acc, tokens_of(kind, n, 150000).cuda(), torch.randn(n, 8, generator=gen, device="cuda").bfloat16(), 0.5)


def test_wide_vocabularies():
    gen = torch.Generator(device="cuda").manual_seed(6)
    for rows in (255, 256, 511, 512, 513, 65535, 65536, 262143, 262144, 3_000_000, (1 << 24) - 2, (1 << 24) - 1, (1 << 24) + 5):
        for n in (1500, 4000, 5000):                    # the order by counting and by the sort
            acc = torch.randn(rows, 4, generator=gen, device="cuda")
            tok = tokens_of("skewed", n, rows).cuda()
            tok[:3] = torch.tensor([rows - 1, rows, 0])
            tok[3:100] = rows - 1 - torch.arange(97, device="cuda") % min(rows, 50)
            check(acc, tok, torch.randn(n, 4, generator=gen, device="cuda"), 1.0)


def test_values_of_masked_rows_do_not_matter_and_others_come_through():
    B = lib()
    acc = torch.zeros(10, 16, device="cuda")
    grad = torch.ones(200, 16, device="cuda")
    tok = torch.full((200,), 4, device="cuda")
    tok[::3] = -100
    grad[::3] = math.nan
    tok[1], tok[2] = 7, 8
    grad[1, 3], grad[2, 5] = math.inf, math.nan
    B.solo_grad_accumulate_rows(acc, tok, grad)
    used = int((tok == 4).sum())
    assert bool((acc[4] == used).all()) and float(acc[7, 3]) == math.inf and math.isnan(float(acc[8, 5]))
    assert int(torch.isnan(acc).sum()) == 1 and int(torch.isinf(acc).sum()) == 1 and float(acc[:4].abs().sum()) == 0.0


def test_same_bits_every_time_on_two_streams_and_in_a_graph():
    B = lib()
    gen = torch.Generator(device="cuda").manual_seed(8)
    n, rows, width = 9000, 300, 520
    tok = tokens_of("skewed", n, rows).cuda()
    grad = torch.randn(n, width, generator=gen, device="cuda").bfloat16()
    start = torch.randn(rows, width, generator=gen, device="cuda")
    first = check(start.clone(), tok, grad, 0.25)
    torch.cuda.synchronize()
    side = [torch.cuda.Stream(), torch.cuda.Stream()]
    accs = [start.clone() for _ in range(16)]
    torch.cuda.synchronize()
    for k, a in enumerate(accs):
        with torch.cuda.stream(side[k % 2]):
            B.solo_grad_accumulate_rows(a, tok, grad, scale=0.25)
    torch.cuda.synchronize()
    for a in accs:
        assert torch.equal(a, first)
    acc = start.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.solo_grad_accumulate_rows(acc, tok, grad, scale=0.25)
    assert torch.equal(acc, start)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(acc, first)
    tok.copy_(tokens_of("few", n, rows))
    grad.copy_(torch.randn(n, width, generator=gen, device="cuda"))
    want = check(start.clone(), tok, grad, 0.25)
    acc.copy_(start)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(acc, want)


def test_an_accumulator_beyond_32_bit_offsets():
    B = lib()
    rows, width = 600_000, 4096
    acc = torch.zeros(rows, width, device="cuda")
    tok = torch.tensor([rows - 1, 0, rows - 1, 524_288], device="cuda")
    grad = torch.arange(1, 5, device="cuda", dtype=torch.float32)[:, None].expand(4, width).contiguous()
    B.solo_grad_accumulate_rows(acc, tok, grad)
    assert bool((acc[rows - 1] == 4).all()) and bool((acc[0] == 2).all()) and bool((acc[524_288] == 4).all())
    assert float(acc.sum(dtype=torch.float64)) == 10.0 * width


def test_rows_list_norm_and_step_together():
    """An embedding's rows go into the accumulator that the list's norm and clip then read."""
    B = lib()
    gen = torch.Generator(device="cuda").manual_seed(9)
    emb, rest = torch.zeros(1000, 64, device="cuda"), torch.randn(5000, generator=gen, device="cuda")
    tok = tokens_of("skewed", 2000, 1000).cuda()
    grad = torch.randn(2000, 64, generator=gen, device="cuda").bfloat16()
    gs = B.GradSet([emb, rest])
    B.solo_grad_accumulate_rows(emb, tok, grad, scale=0.5)
    total, per = B.solo_grad_norm(gs, per_tensor=True)
    want = torch.zeros(1000, 64, device="cuda", dtype=torch.float64).index_add_(0, tok, grad.double() * 0.5)
    # the same sums as above: 97 u of the magnitudes at most, far below 1e-5 of the norm
    assert abs(float(per[0]) / float(want.norm()) - 1) < 1e-5
    assert abs(float(total) ** 2 / float(want.square().sum() + rest.double().square().sum()) - 1) < 1e-5


def test_refusals():
    B = lib()
    acc, tok, grad = torch.zeros(5, 8, device="cuda"), torch.zeros(3, dtype=torch.int64, device="cuda"), torch.ones(3, 8, device="cuda")
    B.solo_grad_accumulate_rows(acc, tok[:0], grad[:0])                                     # nothing to add
    for a, t, g in ((acc.half(), tok, grad), (acc[:, :4], tok, grad), (acc.view(-1), tok, grad), (acc.cpu(), tok, grad),
                    (acc, tok.float(), grad), (acc, tok.cpu(), grad), (acc, tok, grad[:2]), (acc, tok, grad[:, :4]),
                    (acc, tok, grad.double()), (acc, tok, grad.t().contiguous().t())):
        with pytest.raises(ValueError):
            B.solo_grad_accumulate_rows(a, t, g)
    for bad in (math.nan, math.inf):
        with pytest.raises(B.SoloError):
            B.solo_grad_accumulate_rows(acc, tok, grad, scale=bad)
    assert float(acc.abs().sum()) == 0.0


def test_accumulators_next_to_and_over_what_is_read():
    """acc, the gradient's rows and the tokens in one buffer: refused where acc shares memory with either, added where it does not."""
    B = lib()
    gen = torch.Generator(device="cuda").manual_seed(12)
    refused = added = 0
    for n in (3, 1100):
        for rows, width, stride in ((5, 8, 8), (5, 8, 64), (2, 4, 13), (1, 16, 40), (3, 8, 0)):
            size, span = rows * width, (n - 1) * stride + width
            buf = torch.empty(size + span + 2 * size + 2 * n + 64, device="cuda")
            at = size + 8                                                           # where the gradient starts
            for acc_at in sorted({0, 8, 9, size, at, at + width - 1, at + width, at + stride, at + 2 * stride - size, at + 2 * stride - size + 1,
                                  at + span - 1, at + span, at + span + 5}):
                buf.normal_(generator=gen)
                tok_at = (at + span + size + 6 + 1) // 2
                tok = buf.view(torch.int64)[tok_at:tok_at + n] if buf.numel() % 2 == 0 else buf[:-1].view(torch.int64)[tok_at:tok_at + n]
                tok.copy_(tokens_of("skewed", n, rows))
                grad = torch.as_strided(buf, (n, width), (stride, 1), at)
                acc = buf[acc_at:acc_at + size].view(rows, width)
                read = set(range(2 * tok_at, 2 * tok_at + 2 * n))
                for i in range(n):
                    read.update(range(at + i * stride, at + i * stride + width))
                before = buf.clone()
                if read.isdisjoint(range(acc_at, acc_at + size)):
                    check(acc, tok, grad, 0.5)
                    added += 1
                else:
                    with pytest.raises(B.SoloError) as e:
                        B.solo_grad_accumulate_rows(acc, tok, grad, scale=0.5)
                    assert e.value.status == B.SOLO_EINVAL
                    assert torch.equal(buf.view(torch.int32), before.view(torch.int32))
                    refused += 1
    assert refused > 20 and added > 20
    acc = torch.zeros(5, 8, device="cuda")
    with pytest.raises(B.SoloError):
        B.solo_grad_accumulate_rows(acc, acc.view(torch.int64).view(-1)[:3], torch.ones(3, 8, device="cuda"))
    assert float(acc.abs().sum()) == 0.0


@pytest.mark.parametrize("n", [200, 1000, 1024, 1025, 4000, 5000, 65536, 140000])
@pytest.mark.parametrize("period", [1, 16, 17, 24, 33, 64, 96, 200, 1 << 20])
def test_few_additions_follow_one_another_in_binary32(n, period):
    """Fewer than 48, and one rounding besides for every 65,536 tokens.  A large row and then small ones, each a little over half
    of its last place: wherever such a one is added to a sum that begins with the large row, u of that sum is lost, always to the
    same side.  (Additions: 23 in a warp that takes 16 rows and 8 more, 7 over the warps, 1 to binary32; in the one-launch form 31,
    3 and 7.)"""
    B = lib()
    i = torch.arange(n, device="cuda")
    column = torch.where(i % period == 0, 1.0, 2.0 ** -24 * (1 + 2.0 ** -10))
    for width in (8, 5):
        grad = (column[:, None] * torch.tensor([1.0, 3.0, -1.0, 0.5, 1024.0, 1.0, 1.0, -7.0], device="cuda")[:width]).contiguous()
        for scale in (1.0, -0.375):
            acc = torch.zeros(3, width, device="cuda")
            B.solo_grad_accumulate_rows(acc, torch.ones(n, dtype=torch.int64, device="cuda"), grad, scale=scale)
            added = grad.double().abs().sum(0) * abs(scale)
            want = grad.double().sum(0) * scale
            off = (acc[1].double() - want).abs() - (48 + -(-n // CHUNK)) * U * added
            assert float(off.max()) <= 0, float(((acc[1].double() - want).abs() / (U * added)).max())
            assert float(acc[0].abs().sum()) + float(acc[2].abs().sum()) == 0.0


@pytest.mark.parametrize("n", [500, 3000, 9000])
def test_rows_clip_and_step_on_gradients_made_in_torch(n):
    """Rows of whole numbers into an embedding's accumulator, the clip of the whole list by its norm, the step: the same, bit for bit,
    as the step on gradients that torch made with the operations of the formulas."""
    from test_gpu_grad import same_step, step_on, whole_numbers
    B = lib()
    rows, width = 300, 40
    sizes = (rows * width, 5000)
    gen = torch.Generator(device="cuda").manual_seed(n)
    tok = tokens_of("skewed", n, rows, seed=n).cuda()
    tok[::7] = -100
    out, rest = whole_numbers(n * width, n, most=8).view(n, width), whole_numbers(sizes[1], n + 1)
    acc = [torch.zeros(rows, width, device="cuda"), torch.empty(sizes[1], device="cuda")]
    grads = [torch.empty(k, dtype=torch.bfloat16, device="cuda") for k in sizes]
    params = [torch.randn(k, generator=gen, device="cuda") for k in sizes]
    B.solo_grad_accumulate_rows(acc[0], tok, out, scale=0.5)
    B.solo_grad_accumulate(B.GradSet(acc[1:]), B.GradSet([rest]), scale=0.5, first=True)
    keep = tok >= 0
    table = torch.zeros(rows, width, dtype=torch.float64, device="cuda").index_add_(0, tok[keep], out[keep].double() * 0.5)
    assert torch.equal(acc[0].double(), table)                              # below 2^24 multiples of 2^-15: nothing is rounded
    whole = [table.view(-1), rest.double() * 0.5]
    al = B.GradSet(acc)
    norm = B.solo_grad_norm(al)
    N = math.sqrt(sum(float(x.square().sum()) for x in whole))
    assert abs(float(norm) / N - 1) <= 10 * U
    limit = float(torch.tensor(0.2 * N))
    B.solo_grad_clip(al, norm, limit, dst=B.GradSet(grads))
    f = torch.tensor(limit / (float(norm) + 1e-6), dtype=torch.float32, device="cuda")
    want = [(x.float() * f).bfloat16() for x in whole]
    for g, x in zip(grads, want):
        assert torch.equal(g, x) and int(x.count_nonzero()) > 0
    same_step(step_on(B, sizes, params, grads), step_on(B, sizes, params, want))
