"""Inputs of which every result is one token's value row: a missing, doubled or misplaced
key or value anywhere shows, and a bound that only rounding fits in."""
import math

D = 128


def rows(torch, heads, n, k, seed):
    """[heads][n][D] float32: rows whose k largest components are +-1 or nearly, apart from
    every other row's: their products are k, and far less with each other."""
    g = torch.Generator().manual_seed(seed)
    x = (torch.randint(0, 2, (heads, n, D), generator=g) * 2 - 1).float()
    keep = torch.rand(heads, n, D, generator=g).argsort(-1) < k
    return torch.where(keep, x, x * 2.0 ** -6)


def sharpness(k):
    """What a held row is multiplied by for a score of 181 with itself."""
    return 2048.0 / k


def gap(torch, K):
    """By how much the scores of rows sharpness() times a held row lie above their others."""
    s = K.double() @ K.double().T * sharpness(K.double().square().sum(-1).min().item()) / math.sqrt(D)
    own = s.diagonal().clone()
    s.fill_diagonal_(-math.inf)
    return (own - s.amax(1)).min().item()


def misses(torch, got, V, half, turned=False):
    """How many times its bound the worst element of got [rows][D] is off V, the value rows
    meant: the others weigh e^-40 in all (keys' gap of 50 at least), the weight itself is
    divided by a sum that has it, a few steps of 2^-24 in either; a turn back sums 128 products
    in float32; half: half a step of the result's type."""
    V = V.double()
    size = V.norm(dim=-1, keepdim=True).max() if turned else V.abs().max()
    tol = V.abs() * (half + 8 * 2.0 ** -24) + size * ((128 if turned else 0) * 2.0 ** -24 +
                                                      math.exp(-40))
    err = (got.double() - V).abs()
    return (torch.where(torch.isfinite(err), err, torch.full_like(err, math.inf)) /
            tol.clamp_min(2.0 ** -25)).max().item()
