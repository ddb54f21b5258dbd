"""Plain 64-bit statements of a decoding step's operators, for the tests.  Tensors are torch CPU tensors."""
import torch


def f32(x):
    """The double value of the float32 nearest to x (what the C ABI receives)."""
    return float(torch.tensor(x, dtype=torch.float32))


def rms(v, eps):
    return v / torch.sqrt((v * v).mean(-1, keepdim=True) + f32(eps))


def block_stream(x, residual, post_weight, post_eps, gate, scale, residual_scale, offset):
    """residual_scale * residual + scale * gate * norm(x), not rounded, and the size of what is added up."""
    n = x.double()
    if post_weight is not None:
        n = rms(n, post_eps) * (post_weight.double() + f32(offset))
    if gate is not None:
        n = n * gate.double()
    a, b = f32(residual_scale) * residual.double(), f32(scale) * n
    return a + b, a.abs() + b.abs()
