"""The layer operators of libhetsim.so (include/hetsim_ops.h) on torch tensors.

Torch provides device memory (outputs and workspaces come from its allocator)
and the current HIP stream; the work is done by the library's HIP kernels, and
there is no host fallback.  Checks and calls are native (csrc/ops_torch.cpp,
built in-tree as _ops.so): a call on one token takes the card 3 us.  A wrong
type, shape or device raises ValueError; what the library refuses raises
binding.SimError.

Autograd does not see these calls: gradients are the *_backward calls' results.
So a tensor that requires its gradient is refused (ValueError) while autograd
records, adamw's lists excepted: pass it detached, or call under torch.no_grad().
"""
import collections
import os

import torch

from . import _build, binding
from .binding import SimError  # noqa: F401  (raised by every call here)

if not os.path.exists(_build.OPS):
    _build.build_ops()
from . import _ops  # noqa: E402

binding.lib()       # built, and loaded, before the operators are looked up in it
_ops.load(os.environ.get("HETSIM_LIB") or _build.LIB)

BLOCK = 128
E4M3 = torch.float8_e4m3fn
_KINDS = {None: 0, "none": 0, "rms": 1, "layer": 2}


def padded(k):
    """k rounded up to whole blocks."""
    return -(-k // BLOCK) * BLOCK


# ---------------------------------------------------------------- the 8-bit block form and its products
def quantize(x, block_rows=1, rows=True, transposed=False):
    """x [r, c] in e4m3 with a 32-bit scale for each 128 columns of a row (or, with block_rows=128, each 128 x 128 block).

    Returns (codes [r, c padded to 128], scales [c blocks, r or r blocks]); with `transposed` also the same of x's transpose
    (codes [c, r padded to 128], ...), from the same pass over x; with rows=False only that."""
    return _ops.quantize(x, block_rows, rows, transposed)


def dequantize(codes, scales, k):
    """32-bit values [rows, k] of a block form (for checks and inspection; plain torch)."""
    rows = codes.shape[0]
    s = scales.t()
    if s.shape[0] != rows:
        s = s.repeat_interleave(BLOCK, 0)[:rows]
    return codes[:, :k].float() * s.repeat_interleave(BLOCK, 1)[:, :k]


def matmul(a, a_scales, b, b_scales, k, out_dtype=torch.bfloat16, out=None, accumulate=False):
    """A B^T of two matrices in the block form, A [m, k] and B [n, k], as [m, n] of out_dtype; into `out` where given, added
    to it with `accumulate`."""
    return _ops.matmul(a, a_scales, b, b_scales, k, out_dtype, out, accumulate)


def linear(x, codes, scales, out=None):
    """x W^T for x [tokens, k] in 16 or 32 bits and a weight W [n, k] that is laid out in the block form (quantize(w, 128));
    x is brought to 8 bits with a scale for each row and 128 columns on the way.  [tokens, n] in x's type."""
    return _ops.linear(x, codes, scales, out)


LinearSaved = collections.namedtuple("LinearSaved", "tokens n k w_t w_t_scales x_t x_t_scales dtype")


def linear_forward(x, w):
    """Forward pass of a training step of y = x W^T in 8 bits: x [tokens, k], w [n, k].  Returns (y, what linear_backward
    takes): the transposes of both operands leave with the operands, in 8 bits."""
    if x.dim() != 2 or w.dim() != 2 or w.shape[1] != x.shape[1]:
        raise ValueError("x [tokens, k] and w [n, k]")
    (t, k), n = x.shape, w.shape[0]
    xq, xs, xt, xts = quantize(x, transposed=True)
    wq, ws, wt, wts = quantize(w, BLOCK, transposed=True)
    return matmul(xq, xs, wq, ws, k, x.dtype), LinearSaved(t, n, k, wt, wts, xt, xts, w.dtype)


def linear_backward(dy, saved, dw=None):
    """Gradients (dx, dw) of linear_forward for dy [tokens, n].  dw has the weight's type; a given `dw` (of any type) is added
    to, as over the micro-batches of a step."""
    s = saved
    if tuple(dy.shape) != (s.tokens, s.n):
        raise ValueError("dy: [%d, %d]" % (s.tokens, s.n))
    q, sc, qt, sct = quantize(dy, transposed=True)
    dx = matmul(q, sc, s.w_t, s.w_t_scales, s.n, dy.dtype)
    return dx, matmul(qt, sct, s.x_t, s.x_t_scales, s.tokens, s.dtype, out=dw, accumulate=dw is not None)


# ---------------------------------------------------------------- the norms around a block
Norm = collections.namedtuple("Norm", "h x x_scale post_stats pre_stats")
NormGrad = collections.namedtuple("NormGrad", "dh dy dgate dpost_weight dpost_bias dpre_weight dpre_bias")


def _kind(kind):
    try:
        return _KINDS[kind]
    except (KeyError, TypeError):
        raise ValueError("a norm is 'rms', 'layer' or 'none', not %r" % (kind,)) from None


def norm_block(h, y=None, gate=None, post_weight=None, post_bias=None, pre_weight=None, pre_bias=None, post="none", pre="rms",
               alpha=1.0, beta=1.0, eps=1e-6, rows_per_gate=None, quantized=False, out=None, act_dtype=None):
    """The end of a block and the beginning of the next, for h (residual stream) and y (the block's output), [tokens, hidden]:

        r = alpha h + beta gate * post(y);  x = pre(r)

    with post and pre "rms", "layer" or "none", their weights and biases [hidden] in 32 bits, and gate [groups, hidden], of
    which a row serves rows_per_gate tokens (None: all).  Returns Norm(h=r in h's type, x, x_scale, post_stats, pre_stats); x is
    in y's type, or with `quantized` the codes of the block form (x_scale: its scales).  `out` takes h's place (it may be h).
    Without y: r = h, and x has h's type or act_dtype."""
    return Norm._make(_ops.norm(h, y, gate, post_weight, post_bias, pre_weight, pre_bias, _kind(post), _kind(pre), alpha, beta, eps,
                                rows_per_gate, quantized, out, act_dtype))


def norm_block_backward(dh, dx, h, y=None, gate=None, post_weight=None, post_bias=None, pre_weight=None, post_stats=None,
                        pre_stats=None, post="none", pre="rms", alpha=1.0, beta=1.0, rows_per_gate=None, pre_bias=None):
    """Gradients of norm_block from those of its h (dh, None: zero) and its x (dx; None with pre="none"): h is its output h, the
    other arguments are its own and its statistics.  Returns NormGrad; what the forward pass had no input for is None.  The
    weights' gradients are there for every norm, the biases' for every layer norm and for an rms norm whose bias is given here
    as it was to norm_block; all of them in 32 bits, like dgate."""
    return NormGrad._make(_ops.norm_backward(dh, dx, h, y, gate, post_weight, post_bias, pre_weight, post_stats, pre_stats,
                                             _kind(post), _kind(pre), alpha, beta, rows_per_gate, pre_bias))


# ---------------------------------------------------------------- AdamW
def adamw(params, grads, exp_avgs, exp_avg_sqs, copies=None, exp_avg_scales=None, exp_avg_sq_scales=None, *, step, lr, beta1=0.9,
          beta2=0.999, eps=1e-8, weight_decay=0.01, grad_scale=None, skip=None, seed=0):
    """One AdamW step, in place, over lists of contiguous tensors (one type in each list).

    Moments in float32, or in 8 bits: e4m3 codes with a scale for each 128 elements in exp_avg_scales and exp_avg_sq_scales
    ([ceil(n / 128)] each; the second moment's codes hold its square root), rounded by numbers made from seed, step and the
    element's place in the list (every tensor takes a multiple of 128 places).  `copies` get the new parameters in another
    type.  step counts from 1; weight_decay is a number or one for each tensor; grad_scale (one float32 on the device)
    multiplies every gradient, and where skip (one int32 on the device) is not zero nothing changes."""
    decays = weight_decay if isinstance(weight_decay, (list, tuple)) else (weight_decay,)
    _ops.adamw(params, grads, exp_avgs, exp_avg_sqs, copies, exp_avg_scales, exp_avg_sq_scales, step, lr, beta1, beta2, eps, decays,
               grad_scale, skip, seed)
