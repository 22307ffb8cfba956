"""The gradient calls as a training step uses them: micro-batches into fp32 accumulators, the embedding's rows among them, the norm
and the clip into bf16, the optimizer step; over one worker and, with the norms of the shards, over three.  Gradients are checked
against 64 bits, the step's state and parameters against the oracle on the gradients that the clip wrote.

Tolerance of a gradient.  u = 2^-24.  An accumulator of k micro-batches has k roundings, each of at most u times the sum of magnitudes A
(of the embedding's rows: 48 additions in binary32 and two roundings besides, 50 u A); the factor has 10 u from the norm and two
roundings; bf16 half a step, 2^-8.
"""
import math

import numpy as np
import pytest
import torch

import oracle
import parity
from paper_2505_00347_b200 import shard, synth

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
VOCAB, WIDTH, BLOCK = 700, 72, 128
SIZES = (VOCAB * WIDTH, 2048 * 5 + 300, 777, 2048 * 2)
MICRO = 3


def lib():
    from paper_2505_00347_b200 import binding
    return binding


def micro_batch(step, k):
    """Gradients of all tensors but the embedding, tokens and the embedding's output gradient (some positions masked)."""
    g = torch.Generator().manual_seed(100 * step + k)
    rest = [(torch.randn(n, generator=g) * 1e-3).bfloat16().cuda() for n in SIZES[1:]]
    tok = (VOCAB * torch.rand(4, 512, generator=g) ** 3).long()
    tok[torch.rand(4, 512, generator=g) < 0.1] = -100
    out = (torch.randn(4, 512, WIDTH, generator=g) * 1e-3).bfloat16()
    return rest, tok.cuda(), out.cuda()


def gradients_64(step):
    """Sum over the micro-batches and the sum of magnitudes."""
    want = [torch.zeros(n, dtype=torch.float64, device="cuda") for n in SIZES]
    size = [w.clone() for w in want]
    third = float(torch.tensor(1.0 / MICRO))
    for k in range(MICRO):
        rest, tok, out = micro_batch(step, k)
        keep = tok.view(-1) >= 0
        rows = out.view(-1, WIDTH)[keep].double() * third
        want[0].view(VOCAB, WIDTH).index_add_(0, tok.view(-1)[keep], rows)
        size[0].view(VOCAB, WIDTH).index_add_(0, tok.view(-1)[keep], rows.abs())
        for w, a, r in zip(want[1:], size[1:], rest):
            w += r.double() * third
            a += r.double().abs() * third
    return want, size


@pytest.mark.parametrize("workers", [1, 3])
def test_training_steps(workers):
    B = lib()
    w = synth.workload(2, sizes=SIZES)
    params = [synth.make_param(w, i).cuda() for i in range(len(SIZES))]
    oparams = [p.cpu().numpy().copy() for p in params]
    kw = dict(lr=1e-3, beta1=0.6, beta2=0.999, weight_decay=0.01, seed=31)
    ho, hg = parity.hyper_pair(**kw)
    ostates = [oracle.State(n, 3, 3, BLOCK) for n in SIZES]
    state = B.State(list(SIZES), 3, 3, BLOCK)
    acc = [torch.empty(n, device="cuda") for n in SIZES]
    grads = [torch.empty(n, dtype=torch.bfloat16, device="cuda") for n in SIZES]
    ts = B.TensorSet(params, grads, state)
    rest = B.GradSet(acc[1:])
    pieces = shard.partition(SIZES, BLOCK, workers)
    cut = lambda ts_, mine: B.GradSet([ts_[p.tensor][p.elem_offset:p.elem_offset + p.numel] for p in mine])  # noqa: E731
    acc_of, grad_of = [cut(acc, mine) for mine in pieces], [cut(grads, mine) for mine in pieces]
    for step in (1, 2, 3):
        acc[0].zero_()
        for k in range(MICRO):
            g, tok, out = micro_batch(step, k)
            B.solo_grad_accumulate(rest, B.GradSet(g), scale=1.0 / MICRO, first=k == 0)
            B.solo_grad_accumulate_rows(acc[0].view(VOCAB, WIDTH), tok, out, scale=1.0 / MICRO)
        want, size = gradients_64(step)
        N = math.sqrt(sum(float(x.square().sum()) for x in want))
        limit = float(torch.tensor((0.3, 2.0, 0.7)[step - 1] * N))          # the second step is not clipped
        if workers == 1:
            norm = B.solo_grad_clip_norm(acc_of[0], limit, dst=grad_of[0])
        else:
            norm = torch.cat([B.solo_grad_norm(a) for a in acc_of])         # what an all-gather brings together
            for a, d in zip(acc_of, grad_of):
                B.solo_grad_clip(a, norm, limit, dst=d)
        # 60 u: the accumulators' own error, as above, and the norm's
        assert abs(float(norm.double().norm()) / N - 1) <= 60 * U * max(1.0, math.sqrt(sum(float(a.square().sum()) for a in size)) / N)
        f = min(1.0, limit / (N + 1e-6))
        for g, x, a in zip(grads, want, size):
            off = (g.double() - x * f).abs() - x.abs() * f * (2.0 ** -8 + 80 * U) - (50 + MICRO) * U * a * f
            assert float(off.max()) <= 0
        before = [g.clone() for g in grads]
        B.solo_multi_step(ts, hg, step)
        for i, g in enumerate(before):
            oracle.step(oparams[i], synth.bf16_bits(g), ostates[i], ho, step, tensor=i)
    torch.cuda.synchronize()
    assert state.status() == 0
    got, exp = parity.download_state(state), parity.join_state(ostates)
    for k in parity.KEYS:
        assert np.array_equal(got[k].view(np.uint8), exp[k].view(np.uint8)), k
    for p, o in zip(params, oparams):
        assert parity.close(p.cpu().numpy(), o).all()
    state.destroy()
