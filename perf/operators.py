"""The gradient operators that run between the backward pass and the optimizer step, as they are measured.

`run` computes a case in plain torch, or (with `own` true) through the library's Python entry points; `exact` does it in 64
bits from the definitions.  A list of tensors lies in one slab, as flattened gradient buffers do, every tensor a view of it
that starts on a multiple of `PAD` elements (plus `shift` elements, which takes the views off their 16-byte boundaries); what
lies between the tensors is zero, so that the plain forms and the outputs can take the slab as a whole.

  norm         N = |s| (sum |g|^p)^(1/p) over all tensors, p = 1, 2 or infinity (norm_type 0), and the same for each tensor
  clip         g -> round(g * f), f = s * min(1, max_norm / (N + 1e-6)), N put together from the norms of the shards
  clip_norm    the norm of the list, and the clip by it
  accumulate   acc <- acc + s * g in binary32, or s * g for the first micro-batch; with the norm of the result where asked for
  rows         acc[tok_i, :] += s * g[i, :]: the gradient of an embedding; tokens outside the table contribute nothing
"""
import math

import numpy as np
import torch

own = False

PAD = 1024
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}


# ---- tensor lists -----------------------------------------------------------------------------------------------------

def gpt_sizes(layers, d, vocab, positions):
    """Embeddings, per layer four vectors of norms, attention and MLP with their biases, and the last norm."""
    s = [vocab * d, positions * d] if vocab else []
    for _ in range(layers):
        s += [d, d, d * 3 * d, 3 * d, d * d, d, d, d, d * 4 * d, 4 * d, 4 * d * d, d]
    return s + [d, d]


def llama_sizes(layers, d, f, vocab):
    """Embedding, per layer four attention matrices, three of the gated MLP and two norms; the last norm and the head."""
    s = [vocab * d] if vocab else []
    for _ in range(layers):
        s += [d * d] * 4 + [d * f, d * f, f * d, d, d]
    return s + ([d, vocab * d] if vocab else [])


def ragged_sizes(count, largest, seed):
    rng = np.random.default_rng(seed)
    return [int(x) for x in np.clip(np.rint(np.exp(rng.uniform(0.0, math.log(largest), count))), 1, largest)]


def sizes_of(case):
    if case["set"] == "gpt":
        return gpt_sizes(case["layers"], case["d"], case["vocab"], case["positions"])
    if case["set"] == "llama":
        return llama_sizes(case["layers"], case["d"], case["f"], case["vocab"])
    if case["set"] == "ragged":
        return ragged_sizes(case["count"], case["largest"], case["count"] + case["largest"])
    return [case["numel"]]


def starts_of(sizes):
    """First element of every tensor in the slab, and the slab's length."""
    room = [-(-n // PAD) * PAD for n in sizes]
    ends = np.cumsum([0] + room)
    return [int(x) for x in ends[:-1]], int(ends[-1])


GPT125M = {"set": "gpt", "layers": 12, "d": 768, "vocab": 50257, "positions": 1024}
LLAMA7B = {"set": "llama", "layers": 32, "d": 4096, "f": 11008, "vocab": 32000}
FOUR_LAYERS = {"set": "llama", "layers": 4, "d": 4096, "f": 11008, "vocab": 0}
RAGGED = {"set": "ragged", "count": 4096, "largest": 4 << 20}


def listed():
    return [
        # one small tensor before every step: latency
        dict(name="norm 1Mi bf16", op="norm", set="one", numel=1 << 20, dtype="bf16", norm_type=2, scale=1.0, shift=0),
        # the whole gradient of a 7B model, with every tensor's norm for the training log
        dict(name="norm 7B bf16", op="norm", **LLAMA7B, dtype="bf16", norm_type=2, scale=1.0, shift=0),
        # thousands of tensors from one element to millions, by their largest element
        dict(name="norm ragged f32 max", op="norm", **RAGGED, dtype="f32", norm_type=0, scale=0.125, shift=1),
        # the second half of clipping in place, where the norm is known already
        dict(name="clip 125M bf16 in place", op="clip", **GPT125M, dtype="bf16", out="", norms=1, ratio=0.9, norm_type=2, scale=1.0, shift=0),
        # eight workers' norms; accumulators of four decoder layers become the step's bf16 gradients
        dict(name="clip 809M f32 to bf16", op="clip", **FOUR_LAYERS, dtype="f32", out="bf16", norms=8, ratio=0.3, norm_type=2, scale=0.125, shift=0),
        # norm and clip in one call, at the end of an accumulation
        dict(name="clip_norm 125M f32 to bf16", op="clip_norm", **GPT125M, dtype="f32", out="bf16", ratio=0.25, norm_type=2, scale=0.25, shift=0),
        # one decoder layer of a run in half precision with a loss scale
        dict(name="clip_norm layer f16 to bf16", op="clip_norm", set="gpt", layers=1, d=768, vocab=0, positions=0, dtype="f16", out="bf16",
             ratio=0.5, norm_type=2, scale=2.0 ** -10, shift=0),
        # a micro-batch into the accumulators
        dict(name="accumulate 125M bf16", op="accumulate", **GPT125M, dtype="bf16", first=False, scale=0.25, norm_type=-1, shift=0),
        # the last micro-batch, with the norm of what has been collected
        dict(name="accumulate 809M bf16 norm", op="accumulate", **FOUR_LAYERS, dtype="bf16", first=False, scale=0.125, norm_type=2, shift=0),
        # a short sequence of a small model in binary32: latency
        dict(name="rows 256x768 f32", op="rows", vocab=50257, d=768, tokens=256, dtype="f32", skew=1.0, outside=0.0, scale=1.0, shift=0),
        # sixteen sequences of 1024 tokens, some of them padding
        dict(name="rows 16384x768 bf16", op="rows", vocab=50257, d=768, tokens=16384, dtype="bf16", skew=1.0, outside=0.1, scale=0.25, shift=0),
        # four long sequences of a 7B model
        dict(name="rows 16384x4096 bf16", op="rows", vocab=32000, d=4096, tokens=16384, dtype="bf16", skew=1.0, outside=0.0, scale=0.125, shift=0),
    ]


def draw(rng):
    log = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))  # noqa: E731
    op = rng.choice(("norm", "clip", "clip_norm", "accumulate", "rows"))
    scale = 2.0 ** -rng.randrange(0, 8) * rng.uniform(0.5, 1.0)
    if op == "rows":
        d = log(17, 8192)
        return dict(op=op, vocab=log(100, 150000 if d < 2000 else 40000), d=d, tokens=log(1, min(40000, (16384 * 4096) // d)), dtype=rng.choice(("bf16", "f16", "f32")),
                    skew=rng.uniform(0.0, 1.3), outside=rng.choice((0.0, 0.2)), scale=scale, shift=rng.choice((0, 0, 1)))
    which = rng.choice(("one", "gpt", "llama", "ragged"))
    if which == "one":
        c = dict(set="one", numel=log(1, 1 << 28))
    elif which == "gpt":
        c = dict(set="gpt", layers=rng.randint(1, 12), d=log(64, 1024), vocab=log(256, 60000), positions=log(64, 4096))
    elif which == "llama":
        c = dict(set="llama", layers=rng.randint(1, 4), d=8 * log(32, 512), f=log(700, 11008), vocab=0)
    else:
        c = dict(set="ragged", count=log(2, 3000), largest=log(1000, 1 << 20))
    c.update(op=op, dtype=rng.choice(("bf16", "bf16", "f16", "f32")), scale=scale, shift=rng.choice((0, 0, 0, 1)))
    if op == "accumulate":
        c.update(first=rng.random() < 0.3, norm_type=rng.choice((-1, 2, 0)))
    else:
        c.update(norm_type=rng.choice((2, 2, 1, 0)))
    if op in ("clip", "clip_norm"):
        c.update(out=rng.choice(("bf16", "bf16", "f32")) if op == "clip_norm" else rng.choice(("", "bf16", "f32")), ratio=rng.uniform(0.1, 2.0))
    if op == "clip":
        c.update(norms=rng.choice((1, 2, 8, 64)))
    return c


# ---- inputs -----------------------------------------------------------------------------------------------------------

def zipf(case):
    """Chance of every token: natural text's counts fall about like a power of the rank."""
    w = np.arange(1, case["vocab"] + 1, dtype=np.float64) ** -case["skew"]
    return w / w.sum()


def slab(length, shift, dtype):
    return torch.zeros(length + shift, device="cuda", dtype=dtype)[shift:]


def gradients(case, sizes, starts, length, gen, dtype):
    """Normal values, every tensor with a scale of its own (1e-5 to 1e-2; times the loss scale for half precision)."""
    loud = 1024.0 if dtype == torch.float16 else 1.0
    scales = torch.exp(torch.rand(len(sizes), generator=gen, device="cuda") * 6.9 - 11.5).mul_(loud).tolist()
    g = slab(length, case["shift"], dtype)
    for n, at, s in zip(sizes, starts, scales):
        for lo in range(at, at + n, 1 << 28):
            hi = min(at + n, lo + (1 << 28))
            g[lo:hi] = torch.randn(hi - lo, generator=gen, device="cuda").mul_(s)
    return g


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed * 7919 + 17)
    st = {"case": case}
    if case["op"] == "rows":
        V, d, T = case["vocab"], case["d"], case["tokens"]
        names = torch.randperm(V, generator=gen, device="cuda")     # which token is the frequent one
        tok = names[torch.multinomial(torch.from_numpy(zipf(case)).cuda(), T, replacement=True, generator=gen)]
        if case["outside"]:
            off = torch.rand(T, generator=gen, device="cuda") < case["outside"]
            tok = torch.where(off, torch.where(torch.rand(T, generator=gen, device="cuda") < 0.5, -100, V), tok)
        st["tokens"] = tok.to(torch.int64)
        st["acc"] = (torch.randn(V * d, generator=gen, device="cuda") * 1e-2).view(V, d)
        g = slab(T * d, case["shift"], DTYPES[case["dtype"]])
        g.copy_(torch.randn(T * d, generator=gen, device="cuda") * 1e-2)
        st["grad"] = g.view(T, d)
        return st
    sizes = sizes_of(case)
    starts, length = starts_of(sizes)
    dtype = DTYPES[case["dtype"]]
    st["grad"] = gradients(case, sizes, starts, length, gen, dtype)
    of = np.repeat(np.arange(len(sizes)), [-(-n // PAD) for n in sizes])
    st["tensor_of_piece"] = torch.from_numpy(of).cuda()
    st["last_piece"] = torch.tensor(np.cumsum([-(-n // PAD) for n in sizes]) - 1, device="cuda")
    if case["op"] == "accumulate":
        st["acc"] = gradients(case, sizes, starts, length, gen, torch.float32)
    if case["op"] in ("clip", "clip_norm"):
        # the largest norm allowed is `ratio` of the one that these gradients have (measured once, as a run's history would tell)
        total = norm_64(st["grad"], case["norm_type"]) * case["scale"]
        st["max_norm"] = float(np.float32(total * case["ratio"]))
        st["out"] = slab(length, case["shift"], DTYPES[case["out"]]) if case["out"] else st["grad"]
    if case["op"] == "clip":
        part = torch.rand(case["norms"], generator=gen, device="cuda", dtype=torch.float64) + 0.1
        part = part * (total / combined(part, case["norm_type"]))
        st["norms"] = part.float()
    if own:                                     # the descriptors that a training program builds once
        from paper_2505_00347_b200 import binding as B
        for key in ("grad", "acc", "out"):
            if key in st:
                st["list_" + key] = B.GradSet([st[key][at:at + n] for at, n in zip(starts, sizes)])
    return st


def norm_64(g, p):
    """Norm of a whole slab in 64 bits, a few hundred million elements at a time."""
    parts = [combined(x.double().abs(), p) for x in g.split(1 << 27)]
    return float(combined(torch.stack(parts), p))


def combined(x, p):
    return x.max() if p == 0 else x.sum() if p == 1 else x.square().sum().sqrt()


# ---- plain forms ------------------------------------------------------------------------------------------------------

def powers(x, p):
    return x.abs() if p < 2 else x.square()


def plain_norms(g, st, p, scale):
    """Total and per-tensor norms: sums over pieces of PAD elements (a tensor is whole pieces), 64-bit sums over those."""
    t = powers(g.float(), p).view(-1, PAD)
    if p == 0:
        piece = t.amax(1)
        per = torch.zeros(st["last_piece"].numel(), device="cuda").scatter_reduce_(0, st["tensor_of_piece"], piece, "amax")
        return (per.max() * abs(scale)).view(1), per * abs(scale)
    upto = t.sum(1).double().cumsum(0)[st["last_piece"]]
    per = torch.diff(upto, prepend=upto.new_zeros(1))
    total = upto[-1:]
    if p == 2:
        per, total = per.clamp(min=0).sqrt(), total.sqrt()
    return (total * abs(scale)).float(), (per * abs(scale)).float()


def plain_factor(total, max_norm, scale):
    return scale * torch.clamp(max_norm / (total + 1e-6), max=1.0)


def run(st):
    case = st["case"]
    op, scale = case["op"], case["scale"]
    if own:
        return run_own(st, case, op, scale)
    if op == "norm":
        total, per = plain_norms(st["grad"], st, case["norm_type"], scale)
        return {"total": total, "per_tensor": per}
    if op == "clip":
        f = plain_factor(combined(st["norms"].float(), case["norm_type"]), st["max_norm"], scale)
        st["out"].copy_(st["grad"].float() * f)
        return {"out": st["out"]}
    if op == "clip_norm":
        total, _ = plain_norms(st["grad"], st, case["norm_type"], scale)
        st["out"].copy_(st["grad"].float() * plain_factor(total, st["max_norm"], scale))
        return {"out": st["out"], "total": total}
    if op == "accumulate":
        if case["first"]:
            torch.mul(st["grad"].float(), scale, out=st["acc"])
        else:
            st["acc"].add_(st["grad"].float() * scale)
        if case["norm_type"] < 0:
            return {"acc": st["acc"]}
        return {"acc": st["acc"], "total": plain_norms(st["acc"], st, case["norm_type"], 1.0)[0]}
    tok = st["tokens"]
    valid = (tok >= 0) & (tok < case["vocab"])
    g = torch.where(valid[:, None], st["grad"].float() * scale, 0.0)
    st["acc"].index_add_(0, torch.where(valid, tok, 0), g)
    return {"acc": st["acc"]}


def norm_type_of(case):
    return math.inf if case["norm_type"] == 0 else case["norm_type"]


def run_own(st, case, op, scale):
    from paper_2505_00347_b200 import binding as B
    if op == "norm":
        total, per = B.solo_grad_norm(st["list_grad"], norm_type=norm_type_of(case), scale=scale, per_tensor=True)
        return {"total": total, "per_tensor": per}
    if op == "clip":
        B.solo_grad_clip(st["list_grad"], st["norms"], st["max_norm"], dst=st["list_out"], norm_type=norm_type_of(case), scale=scale)
        return {"out": st["out"]}
    if op == "clip_norm":
        total = B.solo_grad_clip_norm(st["list_grad"], st["max_norm"], dst=st["list_out"], norm_type=norm_type_of(case), scale=scale)
        return {"out": st["out"], "total": total}
    if op == "accumulate":
        if case["norm_type"] < 0:
            B.solo_grad_accumulate(st["list_acc"], st["list_grad"], scale=scale, first=case["first"])
            return {"acc": st["acc"]}
        total = B.solo_grad_accumulate(st["list_acc"], st["list_grad"], scale=scale, first=case["first"], norm_type=norm_type_of(case))
        return {"acc": st["acc"], "total": total}
    B.solo_grad_accumulate_rows(st["acc"], st["tokens"], st["grad"], scale=scale)
    return {"acc": st["acc"]}


# ---- what a pass cannot do without, and the results in 64 bits ---------------------------------------------------------

def work(case):
    e = BYTES[case["dtype"]]
    if case["op"] == "rows":
        n = case["tokens"] * case["d"]
        inside = case["tokens"] * (1.0 - case["outside"])
        rows = float((1.0 - np.exp(inside * np.log1p(-np.minimum(zipf(case), 1.0 - 1e-12)))).sum())     # expected distinct tokens
        return {"bytes": inside * case["d"] * e + case["tokens"] * 8 + rows * case["d"] * 8, "flops": 2.0 * n}
    n = sum(sizes_of(case))
    if case["op"] == "norm":
        return {"bytes": n * e, "flops": 2.0 * n}
    if case["op"] == "accumulate":
        return {"bytes": n * (e + (4 if case["first"] else 8)), "flops": 2.0 * n}
    return {"bytes": n * (e + BYTES[case["out"] or case["dtype"]]), "flops": (1.0 if case["op"] == "clip" else 3.0) * n}


def exact(case, seed):
    st = prepare(case, seed)
    scale = float(np.float32(case["scale"]))            # the library takes its factors in binary32
    if case["op"] == "rows":
        tok = st["tokens"]
        keep = torch.nonzero((tok >= 0) & (tok < case["vocab"])).view(-1)
        acc = st["acc"].double()
        acc.index_add_(0, tok[keep], st["grad"][keep].double() * scale)
        return {"acc": acc}
    p = case["norm_type"]
    sizes = sizes_of(case)
    starts, _ = starts_of(sizes)
    if case["op"] == "norm":
        per = torch.tensor([norm_64(st["grad"][at:at + n], p) for at, n in zip(starts, sizes)], dtype=torch.float64, device="cuda") * scale
        return {"total": combined(per, p).view(1), "per_tensor": per}
    if case["op"] == "accumulate":
        acc = st["grad"].double().mul_(scale)
        if not case["first"]:
            acc += st["acc"]
        return {"acc": acc} if p < 0 else {"acc": acc, "total": torch.tensor([norm_64(acc, p)], dtype=torch.float64)}
    if case["op"] == "clip":
        total = float(combined(st["norms"].double(), p))
    else:
        total = norm_64(st["grad"], p) * scale
    f = scale * min(1.0, st["max_norm"] / (total + 1e-6))
    out = st["grad"].double().mul_(f)
    return {"out": out} if case["op"] == "clip" else {"out": out, "total": torch.tensor([total], dtype=torch.float64)}
