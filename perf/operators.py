"""Low-rank adapters beside a shared projection, and the clipping of gradients: the calls whose speed matters to a user who
fine-tunes a frozen stack for several tasks and serves the results together.

Kinds of case:

  step    one token for each of several requests, each with its own adapter or none, through one projection
  prompt  the prompts of several requests, one after another in one call, through one projection
  train   the same rows forward and backward: the output, the gradient of the input and those of the adapters
  clip    the global norm of many gradients, and the gradients scaled down to it

Projections are those of Mamba-2 blocks (d_model = 32 * heads in, 129 * heads + 256 out, and 64 * heads in, d_model out) with
24, 32, 64 and 80 heads: the 130M, 350M, 1.3B and 2.7B widths; drawn cases have other widths too.
"""
import math

import torch

own = False

HEADS = (24, 32, 64, 80)
RANKS = (8, 16, 24, 32, 40, 64, 96, 128)
MAX_NORM = 1.0


def listed():
    return [
        # one token of one request: the smallest product there is, one row against a stack's widest projection
        dict(name="step-1", kind="step", rows=1, inner=2560, outer=10576, rank=16, adapters=8, requests=1, bare=0),
        # a full serving batch of the framework, every request with an adapter of its own
        dict(name="step-16", kind="step", rows=16, inner=2560, outer=10576, rank=16, adapters=16, requests=16, bare=0),
        # a larger serving batch in which some requests take the projection as it is
        dict(name="step-64", kind="step", rows=64, inner=5120, outer=2560, rank=32, adapters=24, requests=64, bare=25),
        # prompts of odd lengths at the smallest width
        dict(name="prompt-130m", kind="prompt", rows=333, inner=768, outer=3352, rank=24, adapters=5, requests=7, bare=10),
        # prompts of odd lengths through the output projection
        dict(name="prompt-2.7b-out", kind="prompt", rows=1905, inner=5120, outer=2560, rank=8, adapters=6, requests=9, bare=10),
        # long prompts through the input projection, adapters of a large rank
        dict(name="prompt-2.7b-in", kind="prompt", rows=8192, inner=2560, outer=10576, rank=64, adapters=4, requests=4, bare=0),
        # a short training step of a small model
        dict(name="train-350m", kind="train", rows=600, inner=1024, outer=4384, rank=8, adapters=3, requests=5, bare=0),
        # a segment of the 2.7B stack, several tasks trained together
        dict(name="train-2.7b-in", kind="train", rows=4096, inner=2560, outer=10576, rank=16, adapters=4, requests=6, bare=0),
        # a long segment through the output projection, lengths that differ widely
        dict(name="train-2.7b-out", kind="train", rows=16384, inner=5120, outer=2560, rank=32, adapters=8, requests=11, bare=5),
        # the gradients of one small block's adapters: little data, latency counts
        dict(name="clip-block-130m", kind="clip", what="adapters", layers=1, heads=24, rank=8, source="f32", result="f32"),
        # the gradients of all adapters of a 64-layer stack: many tensors of middling size
        dict(name="clip-adapters-2.7b", kind="clip", what="adapters", layers=64, heads=80, rank=16, source="f32", result="f32"),
        # the gradients of whole blocks, fp32 sums to what a bf16 parameter takes
        dict(name="clip-blocks-2.7b", kind="clip", what="blocks", layers=4, heads=80, rank=0, source="f32", result="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _widths(rng):
    """A projection of one of the blocks, or one of generic sizes (multiples of 8, as all projections have)."""
    heads = rng.choice(HEADS)
    generic = (8 * _log(rng, 16, 640), 8 * _log(rng, 16, 1300))
    inner, outer = rng.choice([(32 * heads, 129 * heads + 256), (64 * heads, 32 * heads), generic])
    return tuple(n + 8 if n == 3072 else n for n in (inner, outer))


def draw(rng):
    kind = rng.choice(("step", "prompt", "train", "clip"))
    if kind == "clip":
        what = rng.choice(("adapters", "blocks"))
        return dict(kind=kind, what=what, layers=_log(rng, 1, 64) if what == "adapters" else rng.randint(1, 4),
                    heads=rng.choice(HEADS), rank=rng.choice(RANKS[:6]) if what == "adapters" else 0,
                    source=rng.choice(("f32", "bf16", "mixed")), result=rng.choice(("f32", "bf16")))
    inner, outer = _widths(rng)
    rank, adapters = rng.choice(RANKS), _log(rng, 1, 32)
    if kind == "step":
        rows = requests = _log(rng, 1, 256)
    else:
        rows = _log(rng, 17, 16384 if kind == "prompt" else 8192)
        most = (8e11 if kind == "prompt" else 4e11) / (2 * inner * outer)     # no more work than the largest listed case
        rows = min(rows, int(most))
        requests = min(rows, _log(rng, 1, 48))
    return dict(kind=kind, rows=rows, inner=inner, outer=outer, rank=rank, adapters=adapters, requests=requests,
                bare=rng.choice((0, 0, 10, 40)))


def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _row_adapters(case, g):
    """The adapter of every row (-1: none): requests one after another, of lengths from a row to most of them."""
    rows, requests = case["rows"], case["requests"]
    first = torch.zeros(rows, dtype=torch.int64, device="cuda")
    first[torch.randperm(rows - 1, generator=g, device="cuda")[:requests - 1] + 1] = 1 if requests > 1 else 0
    request = first.cumsum(0)
    of_request = torch.randint(0, case["adapters"], (requests,), generator=g, device="cuda")
    if case["kind"] == "step" and requests <= case["adapters"]:
        of_request = torch.randperm(case["adapters"], generator=g, device="cuda")[:requests]
    of_request[100 * torch.rand(requests, generator=g, device="cuda") < case["bare"]] = -1
    return of_request[request].to(torch.int32)


def _projection_inputs(case, seed):
    """Normalised activations, weights that keep their variance, adapters as training leaves them: a change of the output of
    about a third of its size."""
    g = _generator(seed)
    rows, inner, outer, rank, n = (case[k] for k in ("rows", "inner", "outer", "rank", "adapters"))

    def normal(*shape, by=1.0):
        return torch.randn(shape, generator=g, device="cuda").mul_(by).to(torch.bfloat16)

    s = dict(x=normal(rows, inner), w=normal(outer, inner, by=inner ** -0.5), a=normal(n, rank, inner, by=inner ** -0.5),
             b=normal(n, outer, rank, by=0.3 * rank ** -0.5), scale=0.5 + 1.5 * torch.rand(n, generator=g, device="cuda"),
             row_adapter=_row_adapters(case, g))
    if case["kind"] == "train":
        s["dout"] = normal(rows, outer, by=1e-3)
    return s


def _gradient_shapes(case):
    h, r = case["heads"], case["rank"]
    d, inner, wide, conv = 32 * h, 64 * h, 129 * h + 256, 64 * h + 256
    if case["what"] == "adapters":
        block = [(r, d), (wide, r), (r, inner), (d, r)]
    else:
        block = [(wide, d), (conv, 4), (conv,), (h,), (h,), (h,), (inner,), (d, inner), (d,)]
    return block * case["layers"]


def _gradients(case, seed):
    """Gradients whose sizes differ between tensors by orders of magnitude."""
    g = _generator(seed)
    shapes = _gradient_shapes(case)
    sizes = torch.exp(2 * torch.randn(len(shapes), generator=torch.Generator().manual_seed(seed)) - 5).tolist()
    kinds = {"f32": (torch.float32,), "bf16": (torch.bfloat16,), "mixed": (torch.float32, torch.bfloat16)}[case["source"]]
    return [torch.randn(s, generator=g, device="cuda").mul_(by).to(kinds[i % len(kinds)]) for i, (s, by) in enumerate(zip(shapes, sizes))]


def prepare(case, seed):
    if case["kind"] == "clip":
        grads = _gradients(case, seed)
        to = torch.bfloat16 if case["result"] == "bf16" else torch.float32
        flat = torch.empty(sum(t.numel() for t in grads), dtype=to, device="cuda")    # what an optimizer or an all-reduce takes whole
        s = dict(case=case, grads=grads, flat=flat, outs=[o.view_as(t) for o, t in zip(flat.split([t.numel() for t in grads]), grads)])
        if own:
            import paper_2411_19460_amd as pk
            s["plan"] = pk.ssd_grad_plan(grads, s["outs"])
        return s
    s = dict(case=case, **_projection_inputs(case, seed))
    if own:
        import paper_2411_19460_amd as pk
        # one for a batch of requests: it serves every projection of every layer, and every token until the batch changes
        s["plan"] = pk.ssd_adapter_plan(s["row_adapter"], case["adapters"])
    return s


def run(s):
    kind = s["case"]["kind"]
    if own:
        import paper_2411_19460_amd as pk
        if kind == "clip":
            return dict(norm=pk.ssd_grad_clip(s["plan"], MAX_NORM), clipped=s["flat"])
        if kind != "train":
            return dict(out=pk.ssd_adapter_linear_fwd(s["x"], s["w"], s["a"], s["b"], s["scale"], s["plan"])["out"])
        f = pk.ssd_adapter_linear_fwd(s["x"], s["w"], s["a"], s["b"], s["scale"], s["plan"], want_hidden=True)
        g = pk.ssd_adapter_linear_bwd(s["x"], s["w"], s["a"], s["b"], s["scale"], s["plan"], s["dout"], hidden=f["hidden"])
        return dict(out=f["out"], dx=g["dx"], da=g["da"], db=g["db"])
    return _plain_clip(s) if kind == "clip" else _plain_projection(s)


def _plain_projection(s):
    """All adapters side by side as one of rank adapters * rank, of which a row keeps the values of its own."""
    n, rank, inner = s["a"].shape
    x, w = s["x"].float(), s["w"].float()
    a = s["a"].float().reshape(n * rank, inner)
    b = s["b"].float().permute(1, 0, 2).reshape(-1, n * rank)
    of_column = torch.arange(n * rank, device=x.device) // rank
    mine = s["row_adapter"][:, None] == of_column[None, :]
    scale, zero = s["scale"][of_column][None, :], x.new_zeros(())
    hidden = torch.where(mine, (x @ a.t()) * scale, zero)
    out = (x @ w.t() + hidden @ b.t()).to(torch.bfloat16)
    if "dout" not in s:
        return dict(out=out)
    dout = s["dout"].float()
    dhidden = torch.where(mine, (dout @ b) * scale, zero)
    dx = (dout @ w + dhidden @ a).to(torch.bfloat16)
    da = (dhidden.t() @ x).reshape(n, rank, inner)
    db = (dout.t() @ hidden).reshape(-1, n, rank).permute(1, 0, 2)
    return dict(out=out, dx=dx, da=da, db=db.contiguous())


def _plain_clip(s):
    grads = [g.float() for g in s["grads"]]
    norm = torch.sqrt(sum(torch.sum(g * g) for g in grads))
    by = torch.clamp(MAX_NORM / (norm + 1e-6), max=1.0)
    _ = [torch.mul(g, by, out=o) for g, o in zip(grads, s["outs"])]
    return dict(norm=norm.reshape(1), clipped=s["flat"])


def work(case):
    if case["kind"] == "clip":
        values = [math.prod(shape) for shape in _gradient_shapes(case)]
        size = {"f32": (4, 4), "bf16": (2, 2), "mixed": (4, 2)}[case["source"]]
        to = 2 if case["result"] == "bf16" else 4
        return dict(bytes=sum(v * (size[i % 2] + to) for i, v in enumerate(values)), flops=3 * sum(values))
    rows, inner, outer, rank, n = (case[k] for k in ("rows", "inner", "outer", "rank", "adapters"))
    used = min(n, case["requests"])                   # adapters that a row has, at most
    weights = 2 * inner * outer + 2 * used * rank * (inner + outer) + 4 * rows
    shared, low = 2 * rows * inner * outer, 2 * rows * rank * (inner + outer)
    if case["kind"] != "train":
        return dict(bytes=weights + 2 * rows * (inner + outer), flops=shared + low)
    return dict(bytes=weights + 4 * rows * (inner + outer) + 4 * n * rank * (inner + outer), flops=2 * shared + 3 * low)


def exact(case, seed):
    if case["kind"] == "clip":
        grads = [g.double() for g in _gradients(case, seed)]
        norm = math.sqrt(math.fsum(float(torch.dot(g.flatten(), g.flatten())) for g in grads))
        by = min(1.0, MAX_NORM / (norm + 1e-6))
        return dict(norm=torch.tensor([norm], dtype=torch.float64), clipped=torch.cat([g.mul_(by).flatten() for g in grads]))
    s = _projection_inputs(case, seed)
    x, w, a, b, scale = (s[k].double() for k in ("x", "w", "a", "b", "scale"))
    out = x.matmul(w.t())
    train = case["kind"] == "train"
    if train:
        dout = s["dout"].double()
        dx, da, db = dout.matmul(w), torch.zeros_like(a), torch.zeros_like(b)
    for i in range(case["adapters"]):
        rows = torch.nonzero(s["row_adapter"] == i)[:, 0]
        down = scale[i] * x[rows].matmul(a[i].t())
        out[rows] += down.matmul(b[i].t())
        if train:
            up = scale[i] * dout[rows].matmul(b[i])
            dx[rows] += up.matmul(a[i])
            da[i], db[i] = up.t().matmul(x[rows]), dout[rows].t().matmul(down)
    return dict(out=out, dx=dx, da=da, db=db) if train else dict(out=out)
