"""A device type measured on the card at hand, and plans evaluated with it.

The paper's workload layer profiles a model's layers on every device type
(Sec. 4.2, [C1]); the evaluator takes a type's TFLOP/s and GB/s instead.  This
command runs the training step of a transformer layer's MLP block with the
layer operators (ops.py) -- norms around the block, 8-bit products with their
gradients, an AdamW step with 8-bit moments -- at the size that one rank of a
tensor-parallel group holds, takes the two rates from the time of its products
and of its norms, and evaluates random plans of the model on a cluster of such
devices beside ones half as fast.

What the figures are: the TFLOP/s are those of 8-bit products with the rounding
of their operands, while the evaluator counts the model's bytes per element as
its description gives them; and the optimizer step's time is printed, but no
plan's time contains one.

    python -m paper_2508_05370_amd.calibrate --model llama-70b --tp 8

It prints one JSON line.
"""
import argparse
import json

import torch
import torch.nn.functional as F

from . import binding as B
from . import ops
from . import workloads as W

HYPER = dict(lr=1e-3, beta1=0.9, beta2=0.95, eps=1e-8)


class MlpBlock:
    """The MLP block of a layer with the residual stream around it, as one tensor-parallel rank holds it:

        h1 = h + y;  x1 = rms(h1) w1;  o = act(x1 W_in^T) W_out^T;  h2 = h1 + gate * rms(o) w2;  x2 = rms(h2) w3

    (y: the attention block's output; x2: the next block's input).  Parameters in 32 bits with a copy of the matrices in 16, moments
    in 8."""

    def __init__(self, hidden, ffn, gated=True, seed=0, dtype=torch.bfloat16, device="cuda"):
        g = torch.Generator(device=device).manual_seed(seed)

        def normal(*shape, scale):
            return torch.empty(shape, device=device).normal_(0.0, scale, generator=g)
        self.gated, self.dtype, self.steps, self.seed = gated, dtype, 0, seed
        self.params = dict(w_in=normal((2 if gated else 1) * ffn, hidden, scale=hidden ** -0.5), w_out=normal(hidden, ffn, scale=ffn ** -0.5),
                           w1=torch.ones(hidden, device=device), w2=torch.ones(hidden, device=device), w3=torch.ones(hidden, device=device))
        self.gate = torch.full((1, hidden), 0.5, dtype=dtype, device=device)
        self.copies = {k: v.to(dtype) for k, v in self.params.items()}
        self.moments = [[torch.zeros(v.numel(), dtype=torch.uint8, device=device).view(ops.E4M3) for v in self.params.values()]
                        for _ in range(2)]
        self.scales = [[torch.zeros(-(-v.numel() // ops.BLOCK), device=device) for v in self.params.values()] for _ in range(2)]

    def _activation(self, u):
        if not self.gated:
            return F.gelu(u)
        a, b = u.chunk(2, dim=1)
        return F.silu(a) * b

    def forward(self, h, y):
        """(h2, x2), and what backward takes."""
        p, c = self.params, self.copies
        first = ops.norm_block(h, y, pre_weight=p["w1"], pre="rms")
        u, saved_in = ops.linear_forward(first.x, c["w_in"])
        with torch.enable_grad():
            u = u.requires_grad_()
            a = self._activation(u)
        o, saved_out = ops.linear_forward(a.detach(), c["w_out"])
        second = ops.norm_block(first.h, o, gate=self.gate, post_weight=p["w2"], pre_weight=p["w3"], post="rms", pre="rms")
        return second.h, second.x, (y, first, u, a, saved_in, o, saved_out, second)

    def backward(self, saved, dh2, dx2):
        """Gradients of h and y, and of the parameters, from those of h2 (None: zero) and x2."""
        p = self.params
        y, first, u, a, saved_in, o, saved_out, second = saved
        g2 = ops.norm_block_backward(dh2, dx2, second.h, o, gate=self.gate, post_weight=p["w2"], pre_weight=p["w3"],
                                     post_stats=second.post_stats, pre_stats=second.pre_stats, post="rms", pre="rms")
        da, dw_out = ops.linear_backward(g2.dy, saved_out)
        du, = torch.autograd.grad(a, u, da)
        dx1, dw_in = ops.linear_backward(du, saved_in)
        g1 = ops.norm_block_backward(g2.dh, dx1, first.h, y, pre_weight=p["w1"], pre_stats=first.pre_stats, pre="rms")
        grads = dict(w_in=dw_in, w_out=dw_out, w1=g1.dpre_weight, w2=g2.dpost_weight, w3=g2.dpre_weight)
        return g1.dh, g1.dy, grads

    def update(self, grads, **hyper):
        """One AdamW step over all parameters; the matrices decay."""
        self.steps += 1
        p, (m, v), (ms, vs) = self.params, self.moments, self.scales
        for keys, decay in ((("w_in", "w_out"), 0.1), (("w1", "w2", "w3"), 0.0)):
            at = [list(p).index(k) for k in keys]

            def pick(x):
                return [x[i] for i in at]
            ops.adamw([p[k].view(-1) for k in keys], [grads[k].reshape(-1) for k in keys], pick(m), pick(v),
                      copies=[self.copies[k].view(-1) for k in keys], exp_avg_scales=pick(ms), exp_avg_sq_scales=pick(vs),
                      step=self.steps, weight_decay=decay, seed=self.seed, **{**HYPER, **hyper})


def _seconds(f, reps):
    f()
    start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    start.record()
    for _ in range(reps):
        f()
    end.record()
    end.synchronize()
    return start.elapsed_time(end) / 1e3 / reps


def measure(model, tp, tokens, reps=10):
    """Rates and times of the block's training step at the sizes of one rank: products in TFLOP/s (with the rounding of their
    operands), norms in GB/s, the whole step and its AdamW part in seconds."""
    hidden = model["h"]
    ffn = (model["expert_ffn"] if model["experts"] else model["ffn"]) // tp
    block = MlpBlock(hidden, ffn, bool(model["gated"]))
    g = torch.Generator(device="cuda").manual_seed(1)
    h, y, dx = (torch.empty((tokens, hidden), device="cuda").normal_(generator=g).to(block.dtype) for _ in range(3))
    wide = block.copies["w_in"].shape[0]

    def step():
        _, _, saved = block.forward(h, y)
        grads = block.backward(saved, None, dx)[2]
        block.update(grads)

    def products():
        for x, w, dy in ((h, block.copies["w_in"], out_in), (act, block.copies["w_out"], y)):
            _, saved = ops.linear_forward(x, w)
            ops.linear_backward(dy, saved)

    def norms():
        r = ops.norm_block(h, y, gate=block.gate, post_weight=block.params["w2"], pre_weight=block.params["w3"], post="rms", pre="rms")
        ops.norm_block_backward(h, dx, r.h, y, gate=block.gate, post_weight=block.params["w2"], pre_weight=block.params["w3"],
                                post_stats=r.post_stats, pre_stats=r.pre_stats, post="rms", pre="rms")
    out_in = torch.empty((tokens, wide), device="cuda").normal_(generator=g).to(block.dtype)
    act = torch.empty((tokens, ffn), device="cuda").normal_(generator=g).to(block.dtype)
    flops = 6.0 * tokens * hidden * (wide + ffn)
    moved = tokens * hidden * 2.0 * (4 + 6)          # forward h, y, h', x; backward dh', dx, h', y, dh, dy
    grads = block.backward(block.forward(h, y)[2], None, dx)[2]
    update = _seconds(lambda: block.update(grads), reps)
    params = sum(v.numel() for v in block.params.values())
    return dict(tflops=flops / _seconds(products, reps) / 1e12, GBps=moved / _seconds(norms, reps) / 1e9, step_s=_seconds(step, reps),
                adamw_s=update, adamw_params_per_s=params / update, tokens=tokens, hidden=hidden, ffn=ffn)


def cluster(rates, nodes):
    """Two pools of `nodes` nodes of eight devices: ones with the measured rates, and ones half as fast; links as of the workloads'
    accelerators (450 GB/s fabric, PCIe and NICs of 400 Gb/s)."""
    types = []
    for part in (1, 2):
        types.append(dict(n_nodes=nodes, dev_per_node=8, tflops=max(1, int(rates["tflops"] / part)),
                          hbm_GBps=max(1, int(rates["GBps"] / part)), intra_MBps=450_000, pcie_MBps=64_000, nic_MBps=W.nic_MBps(400),
                          intra_alpha_ps=W.alpha_from_gbps(3600), pcie_alpha_ps=143_750, nic_alpha_ps=W.alpha_from_gbps(400)))
    return dict(types=types, nic_MBps_dev=None, intra_MBps_node=None)


def best_plan(model, clus, n_plans, seed=0xCA11B):
    """Iteration time (ps) and index of the best of n_plans random plans."""
    sim = B.Sim(model, clus)
    times = sim.eval_plans(B.device_plans(W.random_plans(model, clus, seed, 0, n_plans)))
    best = B.best_tuple(sim.argmin(times))
    sim.close()
    return best


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--model", default="llama-70b", choices=sorted(W.MODELS))
    ap.add_argument("--tp", type=int, default=8, help="tensor-parallel degree whose rank is measured")
    ap.add_argument("--tokens", type=int, default=0, help="tokens of a micro-batch (default: the model's sequence)")
    ap.add_argument("--nodes", type=int, default=16, help="nodes of each of the cluster's two pools")
    ap.add_argument("--plans", type=int, default=1 << 17)
    a = ap.parse_args(argv)
    model = W.model(a.model)
    if model["experts"]:
        model["load_q16"] = W.dirichlet_q16(model["L"], model["experts"])
    rates = measure(model, a.tp, a.tokens or model["seq"])
    time_ps, index = best_plan(model, cluster(rates, a.nodes), a.plans)
    print(json.dumps(dict(model=a.model, tp=a.tp, rates=rates, plans=a.plans, best_plan=index,
                          best_iteration_s=time_ps / 1e12 if index >= 0 else None)))


if __name__ == "__main__":
    main()
