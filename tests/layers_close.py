"""Bounds for the linear layers and the norm as wholes: |result - exact| / |exact|, in norm, of a tensor.

tests/layers_ref.py bounds every value by the sum of its terms' magnitudes, which holds whatever the inputs but grows with the square of the
terms where values grow with their root.  Here inputs are given, of random signs or of one sign, and errors are what the kernels do to them.
u = 2^-24, half a step of fp32.  The tensor cores cut off what they add, sum and products alike: in a run of 512 terms, whose products still have
their low bits, a step (2 u of what the sum has come to) at most is lost with every 16 terms.  In a long sum of one sign the 16 products lose half a
quarter of a step each, 4 u of what it has come to, 2 u of what it ends as.  Runs, splits of the rows and blocks' parts are added in fp32,
rounded to nearest.
  random signs   what a sum has come to is below what it ends as, in norm: 2 u a step of a run, u for every run and part added
  one sign       it grows evenly, and all errors are alike: half of that
A sum ends after 512 terms where the result is fp32, after 32768 where it is bf16.
fp32 values: six of the nine products of three bf16 parts; what is left out is 2 products below 2^-25, u at most.  Two u for the last additions.
A rounding to bf16 is off by 2^-8 at most, and off at random.
"""
import torch

U, H8 = 2.0 ** -24, 2.0 ** -8
RUN, LONG_RUN = 512, 32768


def rel(got, want):
    return ((got.double() - want).norm() / want.norm()).item()


def parts_added(parts):
    """Roundings, one after another, where `parts` partial sums are added: each 32nd by one warp, then 32 of these."""
    return parts if parts <= 32 else parts / 32 + 32


def random_signs(terms, parts=1):
    steps, runs = min(terms, RUN) / 16, -(-terms // RUN)
    return U * (1 + 2 * steps + (runs - 1) + parts_added(parts) + 2)


def long_run(terms):
    """Of bf16 results of one sign, without their own rounding."""
    return U * (2 * min(terms, LONG_RUN) / 16 + terms / LONG_RUN)


def one_sign(terms, parts=1):
    steps, runs = min(terms, RUN) / 16, -(-terms // RUN)
    return U * (1 + (steps + 1) + runs / 2 + parts_added(parts) / 2 + 2)


# ---- what the kernels do, in 64 bits, for checks of the bounds themselves ------------------------------------------------------


def three(x):
    """The bf16 parts of fp32 values."""
    x = x.float()
    hi = x.bfloat16().float()
    mid = (x - hi).bfloat16().float()
    return [t.double() for t in (hi, mid, (x - hi - mid).bfloat16().float())]


SIX = [(0, 0), (0, 1), (1, 0), (0, 2), (2, 0), (1, 1)]


def product(x, w, pairs):
    """x w^T, with some of the parts' products."""
    a, b = three(x), three(w)
    return sum(a[i] @ b[j].t() for i, j in pairs)


def towards_zero(v):
    """fp32, cut off."""
    near = v.float().double()
    return torch.where(near.abs() > v.abs(), torch.nextafter(near.float(), torch.zeros(())).double(), near)


def truncated(terms, run):
    """Sums over the last axis of `terms` that are cut off to fp32 with every 16 and end after `run`, in 64 bits."""
    total = torch.zeros(terms.shape[:-1], dtype=torch.float64)
    for part in terms.double().split(run, -1):
        s = torch.zeros_like(total)
        for piece in part.split(16, -1):
            s = towards_zero(s + piece.sum(-1))
        total = (total + s).float().double()
    return total
