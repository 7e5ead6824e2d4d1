"""The layer operators together: a block's training step, and a device type measured with it."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("gated", [True, False])
@pytest.mark.parametrize("tokens,hidden,ffn", [(70, 256, 384), (33, 200, 130)])
def test_block_gradients(gated, tokens, hidden, ffn):
    """Against 32-bit autograd of the same block: what differs is the rounding to 8 bits."""
    from paper_2508_05370_amd.calibrate import MlpBlock
    b = MlpBlock(hidden, ffn, gated, seed=3)
    g = torch.Generator(device="cuda").manual_seed(5)
    h, y, dx = (torch.randn(tokens, hidden, generator=g, device="cuda").bfloat16() for _ in range(3))
    h2, x2, saved = b.forward(h, y)
    dh, dy, grads = b.backward(saved, None, dx)

    leaves = {k: b.copies[k].float().requires_grad_() if k.startswith("w_") else v.clone().requires_grad_()
              for k, v in b.params.items()}
    hl, yl = h.float().requires_grad_(), y.float().requires_grad_()

    def rms(v, w):
        return v * torch.rsqrt(v.square().mean(1, keepdim=True) + 1e-6) * w
    h1 = hl + yl
    o = b._activation(rms(h1, leaves["w1"]) @ leaves["w_in"].t()) @ leaves["w_out"].t()
    r = h1 + b.gate.float() * rms(o, leaves["w2"])
    x = rms(r, leaves["w3"])
    (x * dx.float()).sum().backward()
    # three roundings to e4m3 (2^-4 at most, about 2.6 % each as the root of the mean square) on the way of a value, more of them on
    # a gradient's: 10 % and 20 % are wide of that, and far from a wrong term
    assert float((x2.float() - x).norm() / x.norm()) < 0.1
    for got, want in [(dh, hl.grad), (dy, yl.grad)] + [(grads[k], leaves[k].grad) for k in grads]:
        assert float((got.float() - want).norm() / want.norm()) < 0.2


def test_block_learns():
    """A few steps on one batch bring its output nearer to a target."""
    from paper_2508_05370_amd.calibrate import MlpBlock
    b = MlpBlock(256, 512, seed=1)
    g = torch.Generator(device="cuda").manual_seed(2)
    h, y, target = (torch.randn(128, 256, generator=g, device="cuda").bfloat16() for _ in range(3))
    losses = []
    for _ in range(30):
        _, x, saved = b.forward(h, y)
        d = x.float() - target.float()
        losses.append(float(d.square().mean()))
        b.update(b.backward(saved, None, (2 * d / d.numel()).bfloat16() * 1024)[2], lr=3e-3)
    assert losses[-1] < 0.7 * losses[0] and all(l == l for l in losses)


def test_measured_device_type():
    from paper_2508_05370_amd import calibrate
    from paper_2508_05370_amd import workloads as W
    model = W.model("gpt2-small")
    rates = calibrate.measure(model, 1, 256, reps=2)
    assert rates["tflops"] > 1 and rates["GBps"] > 1 and rates["step_s"] > rates["adamw_s"] > 0
    time_ps, index = calibrate.best_plan(W.model("llama-7b"), calibrate.cluster(rates, 4), 4096)
    assert 0 <= index < 4096 and time_ps > 0


def test_command(capsys):
    import json
    from paper_2508_05370_amd import calibrate
    calibrate.main(["--model", "llama-7b", "--tp", "8", "--tokens", "512", "--plans", "8192", "--nodes", "8"])
    out = json.loads(capsys.readouterr().out)
    assert out["best_plan"] >= 0 and out["rates"]["tflops"] > 1


def test_no_history_is_lost_silently():
    """What autograd records is refused by every argument; the same calls under no_grad, and on detached tensors, are as ever."""
    from paper_2508_05370_amd import ops
    g = torch.Generator(device="cuda").manual_seed(5)
    h, y, x, w = (torch.randn(*s, generator=g, device="cuda") for s in ((6, 256), (6, 256), (6, 256), (256,)))
    codes, scales = ops.quantize(x, 128)
    norms = dict(h=h, y=y, gate=torch.ones_like(w), post_weight=w, post_bias=w, pre_weight=w, pre_bias=w)
    f = ops.norm_block(post="rms", pre="layer", **norms)
    back = dict(norms, dh=y, dx=x, h=f.h, post_stats=f.post_stats, pre_stats=f.pre_stats)
    for call, kw in ((lambda **k: ops.norm_block(post="rms", pre="layer", **k), dict(norms, out=torch.empty_like(h))),
                     (lambda **k: ops.norm_block_backward(post="rms", pre="layer", **k), back),
                     (ops.linear, dict(x=x, codes=codes, scales=scales, out=torch.empty(6, 6, device="cuda"))),
                     (lambda **k: ops.matmul(k=256, **k), dict(a=codes, a_scales=scales, b=codes, b_scales=scales,
                                                               out=torch.empty(6, 6, device="cuda")))):
        call(**kw)
        for name in kw:
            if kw[name].dtype == ops.E4M3:
                continue
            recorded = dict(kw, **{name: kw[name].detach().clone().requires_grad_()})
            with pytest.raises(ValueError, match="no_grad"):
                call(**recorded)
            with torch.no_grad():
                call(**recorded)


def test_writes_are_seen_by_autograd():
    """What a call writes into counts as changed: a saved tensor that was overwritten is an error in backward, as after torch's own
    in-place functions."""
    from paper_2508_05370_amd import ops
    x = torch.ones(4, 256, device="cuda")
    q, s = ops.quantize(x)

    def writes(t, call):
        before = t._version
        call()
        assert t._version > before
    out = torch.zeros(4, 4, device="cuda")
    writes(out, lambda: ops.matmul(q, s, q, s, 256, out=out))
    writes(out, lambda: ops.linear(x, q, s, out=out))
    out = torch.zeros(4, 256, device="cuda")
    writes(out, lambda: ops.norm_block(x, x, out=out))
    reads = [t._version for t in (x, q, s)]
    for bits in (32, 8):
        p, g, copy = (torch.ones(256, device="cuda") for _ in range(3))
        m, v, scales = [torch.zeros(256, device="cuda") for _ in range(2)], None, {}
        if bits == 8:
            m, v = zip(*(ops.quantize(t[None]) for t in m))
            m, v = [t[0] for t in m], [t[:, 0] for t in v]
            scales = dict(exp_avg_scales=v[:1], exp_avg_sq_scales=v[1:])
        for t in (p, copy, *m, *(v or ())):
            writes(t, lambda: ops.adamw([p], [g], m[:1], m[1:], copies=[copy], step=1, lr=1e-3, **scales))
        assert g._version == 0
    assert reads == [t._version for t in (x, q, s)]
    w = torch.nn.Parameter(torch.ones(256, device="cuda"))
    loss = w.square().sum()
    ops.adamw([w], [g], [torch.zeros_like(g)], [torch.zeros_like(g)], step=1, lr=1e-3)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()
    with torch.inference_mode():          # (tensors without a counter)
        out = torch.zeros(4, 4, device="cuda")
        ops.matmul(q, s, q, s, 256, out=out)
