#!/usr/bin/env python3
"""Fine-tunes a frozen stack of Mamba-2 blocks for several tasks at once and serves the results together: low-rank adapters beside
both projections of every block (`adapter_linear`), their gradients clipped by the global norm (`ssd_grad_clip`), then one token a step
for every request, each with its own adapter (`ssd_adapter_linear_fwd` on a plan of the batch).

    python -m paper_2411_19460_amd.adapt [--tasks 4] [--tokens 512] [--layers 2] [--heads 24] [--rank 8] [--steps 30] [--generate 16]

The stack is randomly initialised; a task is a set of adapters drawn at random, and what is learnt is its output on random inputs.
Prints one JSON line per step and one for the generation.
"""
import argparse
import json
import math
import time

import torch
from torch.autograd.function import once_differentiable

import paper_2411_19460_amd as pk

P, N = 64, 128          # head dimension and state


class _Conv(torch.autograd.Function):
    """The block's convolution with frozen parameters."""

    @staticmethod
    def forward(ctx, u, w, bias):
        ctx.save_for_backward(u, w, bias)
        return pk.ssd_conv1d_fwd(u, w, bias, want_state=False)[0]

    @staticmethod
    @once_differentiable
    def backward(ctx, dout):
        return pk.ssd_conv1d_bwd(*ctx.saved_tensors, None, dout.contiguous(), want_dstate=False)["du"], None, None


class _Norm(torch.autograd.Function):
    """The (gated) RMS normalisation with a frozen weight."""

    @staticmethod
    def forward(ctx, y, z, w):
        ctx.save_for_backward(y, w, *(() if z is None else (z,)))
        return pk.ssd_gated_norm_fwd(y, z, w)

    @staticmethod
    @once_differentiable
    def backward(ctx, dout):
        y, w, *z = ctx.saved_tensors
        g = pk.ssd_gated_norm_bwd(y, z[0] if z else None, w, dout.contiguous())
        return g["dy"], g["dz"], None


class Block:
    """A frozen pre-norm Mamba-2 block whose two projections take adapters {in: (a, b), out: (a, b)}."""

    def __init__(self, heads, g):
        d, di, cd = 32 * heads, 64 * heads, 64 * heads + 2 * N
        rand = lambda *s: torch.randn(s, generator=g, device="cuda")
        self.heads, self.d_inner, self.conv_dim = heads, di, cd
        self.W_in = (rand(di + cd + heads, d) / math.sqrt(d)).bfloat16()
        self.W_out = (rand(d, di) / math.sqrt(di)).bfloat16()
        self.conv_w, self.conv_b = 0.5 * rand(cd, 4), 0.2 * rand(cd)
        dt = torch.exp(math.log(1e-3) + torch.rand(heads, generator=g, device="cuda") * math.log(100.0))
        self.dt_bias = dt + torch.log(-torch.expm1(-dt))
        self.A = -torch.exp(torch.rand(heads, generator=g, device="cuda") * math.log(16.0))
        self.D = rand(heads)
        self.pre_w, self.norm_w = 1 + 0.3 * rand(d), 1 + 0.3 * rand(di)

    def __call__(self, u, adapters, scale, plan, state=None, keep_state=False):
        """u [sequences, tokens, d_model] -> (u + block(u), the states behind it).  state: (convolution, SSM) of every sequence; with
        one, tokens go through the recurrence one by one."""
        S, L, d = u.shape
        rows = u.reshape(S * L, d)
        zx = pk.adapter_linear(_Norm.apply(rows, None, self.pre_w), self.W_in, *adapters["in"], scale, plan)
        z, u_conv, dt = zx.split([self.d_inner, self.conv_dim, self.heads], dim=1)
        u_conv = u_conv.reshape(S, L, self.conv_dim).contiguous()
        dt = torch.nn.functional.softplus(dt.float() + self.dt_bias).bfloat16().reshape(S, L, self.heads)
        conv = ssm = None
        if state is None and not keep_state:
            c = _Conv.apply(u_conv, self.conv_w, self.conv_b)
        else:
            c, conv = pk.ssd_conv1d_fwd(u_conv, self.conv_w, self.conv_b, None if state is None else state[0])
        x, B, C = (t.contiguous() for t in c.split([self.d_inner, N, N], dim=2))
        x, B, C = x.view(S, L, self.heads, P), B.view(S, L, 1, N), C.view(S, L, 1, N)
        if state is None:
            y, ssm = pk.ssd_scan(x, dt, self.A, B, C, self.D, 64, -(-L // 64) * 64)
        else:
            ssm = state[1]
            y = pk.ssd_decode(x, dt, self.A, B, C, self.D, ssm)          # ssm is replaced in place
        y = _Norm.apply(y.reshape(S * L, self.d_inner), z, self.norm_w)
        out = pk.adapter_linear(y, self.W_out, *adapters["out"], scale, plan)
        return u + out.view(S, L, d), (conv, ssm)


def adapters_for(blocks, tasks, rank, g):
    """The tasks' adapters of every block."""
    def pair(w):
        o, i = w.shape
        a = torch.randn((tasks, rank, i), generator=g, device="cuda") / math.sqrt(i)
        b = 0.25 * torch.randn((tasks, o, rank), generator=g, device="cuda") / math.sqrt(rank)
        return a.bfloat16(), b.bfloat16()
    return [{"in": pair(bl.W_in), "out": pair(bl.W_out)} for bl in blocks]


def start_from(adapters):
    """What training starts from: the same a, b zero (nothing is changed before the first step)."""
    return [{k: (a.clone(), torch.zeros_like(b)) for k, (a, b) in ad.items()} for ad in adapters]


def run(blocks, adapters, u, scale, plan, states=None, keep_states=False):
    out = []
    for i, (bl, ad) in enumerate(zip(blocks, adapters)):
        u, s = bl(u, ad, scale, plan, None if states is None else states[i], keep_states)
        out.append(s)
    return u, out


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, default in (("tasks", 4), ("tokens", 512), ("layers", 2), ("heads", 24), ("rank", 8), ("steps", 30), ("generate", 16), ("seed", 0)):
        ap.add_argument("--" + name, type=int, default=default)
    ap.add_argument("--lr", type=float, default=2e-3)
    ap.add_argument("--max-norm", type=float, default=1.0)
    args = ap.parse_args(argv)
    g = torch.Generator(device="cuda").manual_seed(args.seed)
    d = 32 * args.heads
    blocks = [Block(args.heads, g) for _ in range(args.layers)]
    scale = torch.full((args.tasks,), 2.0, device="cuda")
    teacher = adapters_for(blocks, args.tasks, args.rank, g)
    student = start_from(teacher)

    # one plan for the batch: it serves both projections of every block, forward and backward, in every step
    rows_of = lambda tokens: torch.arange(args.tasks, dtype=torch.int32, device="cuda").repeat_interleave(tokens)
    plan = pk.ssd_adapter_plan(rows_of(args.tokens), args.tasks)
    params = [t.requires_grad_() for ad in student for pair in ad.values() for t in pair]
    masters = [t.detach().float() for t in params]
    for t, m in zip(params, masters):
        t.grad, m.grad = torch.zeros_like(t), torch.zeros_like(m)       # kept: the plan below holds their addresses
    clip = pk.ssd_grad_plan([t.grad for t in params], [m.grad for m in masters])
    opt = torch.optim.AdamW(masters, lr=args.lr, weight_decay=0.0)
    losses = []
    for step in range(args.steps):
        u = torch.randn((args.tasks, args.tokens, d), generator=g, device="cuda").bfloat16()
        with torch.no_grad():
            want = run(blocks, teacher, u, scale, plan)[0].float()
        torch._foreach_zero_([t.grad for t in params])
        loss = (run(blocks, student, u, scale, plan)[0].float() - want).square().mean()
        loss.backward()
        norm = pk.ssd_grad_clip(clip, args.max_norm)                     # bf16 gradients -> the fp32 masters' gradients, clipped
        opt.step()
        with torch.no_grad():
            torch._foreach_copy_(params, masters)
        losses.append(float(loss.detach()))
        print(json.dumps({"step": step, "loss": losses[-1], "grad_norm": float(norm)}), flush=True)

    # Serving: a prompt for every task, then one token a step for all of them together.
    with torch.no_grad():
        prompt = torch.randn((args.tasks, args.tokens, d), generator=g, device="cuda").bfloat16()
        tokens = torch.randn((args.tasks, args.generate, d), generator=g, device="cuda").bfloat16()
        states = run(blocks, student, prompt, scale, plan, keep_states=True)[1]
        one = pk.ssd_adapter_plan(rows_of(1), args.tasks)
        got = []
        torch.cuda.synchronize()
        t0 = time.perf_counter()
        for t in range(args.generate):
            o, states = run(blocks, student, tokens[:, t:t + 1].contiguous(), scale, one, states)
            got.append(o)
        torch.cuda.synchronize()
        us = (time.perf_counter() - t0) / max(1, args.generate) * 1e6
        both = torch.cat([prompt, tokens], dim=1)
        whole = run(blocks, student, both, scale, pk.ssd_adapter_plan(rows_of(both.shape[1]), args.tasks))[0][:, args.tokens:]
        diff = float((torch.cat(got, dim=1).float() - whole.float()).abs().max() / whole.float().abs().max()) if got else 0.0
    result = {"requests": args.tasks, "us_per_step": round(us, 1), "difference_to_whole_sequence": diff}
    print(json.dumps(result), flush=True)
    return {"losses": losses, **result}


if __name__ == "__main__":
    main()
