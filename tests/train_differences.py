"""Gradients of a block's training against differences of its output in 64 bits (train_ref.Ref.forward), without any formula of a derivative."""
import copy

import torch

WHAT = ("x", "gate", "w1", "w3", "w2")


def moved(ref, what, by):
    """The block with one of its inputs moved."""
    r = copy.copy(ref)
    if what == "x":
        r.x = r.x + by
    elif what == "gate":
        r.g = r.g + by.reshape(-1)
    else:
        i = ("w1", "w3", "w2").index(what)
        r.w = [tuple(m + by[e] if j == i else m for j, m in enumerate(w)) for e, w in enumerate(r.w)]
    return r


def misfit(ref, d_out, what, grad, way, step=1e-4):
    """How far <grad, way> is from the derivative of sum(out * d_out) along `way`, in lengths of grad (way has length 1).

    What roundings can do: d_a, d_u and g h are rounded to fp16 once (2^-11 of each element), and the kept rows a and u, from which they come, another time each: u goes into them as a
    factor, 2^-11 again; a moves silu' by |a silu''(a)| 2^-11 <= 0.65 2^-11, beside a root mean square of silu' of 0.6 for rows of length 1.  So the operands of the last products are off by no
    more than 4 * 2^-11 = 1.95e-3 of their length, and the gradient by that much of its own; |<error, way>| <= |error|.  The differences themselves are off by step^2 and 1e-14 / step."""
    way = way / way.norm()
    value = lambda s: float((moved(ref, what, s * way).forward()[2][0] * d_out.double()).sum())  # noqa: E731
    slope = (value(step) - value(-step)) / (2 * step)
    return abs(slope - float((grad * way).sum())) / float(grad.norm())


LIMIT = 2e-3


def ways(grad, formula, seed):
    """Directions that a gradient is looked at along: its own and its formula's, each as it is and with every element stretched by 0 to 2.  The slope along these is about the gradient's
    length, beside which roundings are 2e-3; along a random direction it would be a hundredth of it."""
    g = torch.Generator(device=grad.device).manual_seed(seed)
    for v in (grad, formula):
        yield v
        yield v * (2 * torch.rand(v.shape, generator=g, device=v.device, dtype=v.dtype))


def worst(ref, d_out, what, grad, formula, seed=6):
    grad = grad.double()
    return max(misfit(ref, d_out, what, grad, way, 1e-4) for way in ways(grad, formula.double(), seed))
