"""What the norm of a float32 product's error may be, and that it tells the mistakes apart that elementwise bounds let pass.  No GPU.

The tensor cores add 16 products at a time to an accumulator and cut.  Of a run of 512 leading products, 32 additions cut half a unit in the last place
each on average, all towards zero, of sums that grow as the root of their number: 32 * 2/3 * 2^-24 = 1.27e-6 of the run, and of a sum of runs.  The
smaller partial products make one run: up to 5632 * 5 / 16 additions of sums about 2^-9 * sqrt(2) as large, 0.19e-6.  Adding up the runs, rounded to
nearest, is 0.1e-6, and the three partial products left out 0.02e-6.
"""
import pytest
import torch

F32_NORM = 1.6e-6


def parts(v):
    out, rest = [], v.clone()
    for _ in range(3):
        p = rest.float().bfloat16().double()
        out.append(p)
        rest = rest - p
    return out


def cut(v):
    """A float64 number to 24 bits, towards zero."""
    f = v.float()
    over = f.double().abs() > v.abs()
    return torch.where(over, torch.nextafter(f, torch.zeros_like(f)), f).double()


def emulated(x, w, keep, run):
    """x w^T by partial products `keep`, each 16 of them added up and cut in, `run` leading ones to a run."""
    a, b = parts(x), parts(w)
    k = x.shape[1]
    small = torch.zeros(x.shape[0], w.shape[0], dtype=torch.float64)
    for i, j in keep:
        if i + j:
            for c in range(0, k, 16):
                small = cut(small + a[i][:, c:c + 16] @ b[j][:, c:c + 16].t())
    total = small.float()
    for r in range(0, k, run):
        s = torch.zeros_like(small)
        for c in range(r, min(k, r + run), 16):
            s = cut(s + a[0][:, c:c + 16] @ b[0][:, c:c + 16].t())
        total = total + s.float()
    return total.double()


SIX = [(2, 0), (1, 1), (0, 2), (1, 0), (0, 1)]


@pytest.mark.parametrize("k", [2048, 4096])
def test_the_bound_tells_mistakes_apart(k):
    g = torch.Generator().manual_seed(k)
    x, w = torch.randn(48, k, generator=g).double(), (torch.randn(40, k, generator=g) * k ** -0.5).double()
    want = x @ w.t()

    def off(keep, run):
        return float((emulated(x, w, keep, run) - want).norm() / want.norm())

    assert off(SIX, 512) <= F32_NORM
    assert off([(1, 1), (1, 0), (0, 1)], 512) > F32_NORM          # without the third parts
    assert off([(2, 0), (0, 2), (1, 0), (0, 1)], 512) > F32_NORM    # without the product of the second parts
    assert off(SIX, k) > F32_NORM                                   # summed in one go
