"""Rows of logits for the tests over the vocabulary, and how far a result may be from the oracle's."""
import torch

STEP = 2.0 ** -24                        # half a step of an fp32 value, relative to it
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
# Relative error of a row's sum of exponentials: the exponent's argument is rounded three times and its factor
# once (4 |d| 2^-24), terms count down to d = -40 (160 steps), an exponential is off by a step (2), and a
# thread's chain and the trees above it are at most 94 additions at the tests' sizes.
SUM_TOL = 256 * STEP
FLUSHED = 2.0 ** -125                    # products of the smallest normal numbers may be taken as 0

KINDS = ("plain", "peaked", "equal", "masked", "one", "few", "empty", "lowest", "all_lowest", "ascending", "descending", "ties",
         "zeros", "huge", "nan", "inf")


def rows(seed, kinds, vocab, dtype, ld=None):
    """[T, vocab] logits, a kind per row, as a view of rows `ld` apart whose other values are NaN."""
    g = torch.Generator().manual_seed(seed)
    ld = ld or vocab
    buf = torch.full((len(kinds), ld), float("nan"), dtype=dtype)
    low = torch.finfo(dtype).min
    for t, kind in enumerate(kinds):
        z = 2.5 * torch.randn(vocab, generator=g)
        at = int(torch.randint(0, vocab, (1,), generator=g))
        if kind == "peaked":
            z[at] = 25.0
        elif kind == "equal":
            z[:] = 1.25
        elif kind == "masked":
            z[torch.rand(vocab, generator=g) < 0.7] = -torch.inf
            z[at] = 0.5
        elif kind == "one":
            z[:] = -torch.inf
            z[at] = -3.0
        elif kind == "few":
            z[torch.rand(vocab, generator=g) < 0.995] = -torch.inf
            z[at] = 1.0
        elif kind == "empty":
            z[:] = -torch.inf
        elif kind == "lowest":
            z[torch.rand(vocab, generator=g) < 0.7] = low
            z[at] = 0.5
        elif kind == "all_lowest":
            z[:] = low
        elif kind == "ascending":
            z = torch.sort(z).values
        elif kind == "descending":
            z = torch.sort(z, descending=True).values
        elif kind == "ties":
            z = torch.randint(-3, 4, (vocab,), generator=g).float()
        elif kind == "zeros":
            z = torch.where(torch.rand(vocab, generator=g) < 0.5, 0.0, -0.0)
        elif kind == "huge":
            z = torch.where(torch.rand(vocab, generator=g) < 0.5, 0.99 * -low, 0.99 * low)
        elif kind == "nan":
            z[at] = torch.nan
            z[int(torch.randint(0, vocab, (1,), generator=g))] = -torch.nan
        elif kind == "inf":
            z[at] = torch.inf
        buf[t, :vocab] = z.clamp(low, -low).to(dtype) if kind not in ("masked", "one", "few", "empty", "nan", "inf") else z.to(dtype)
    return buf[:, :vocab]


def log_probs(z, tau, stats):
    """ln p of every token in fp64 from the oracle's statistics."""
    d = (z.double() - stats[:, :1]) / tau
    return torch.where(torch.isneginf(stats[:, :1]), -torch.inf, d - torch.log1p(stats[:, 1:])), d


def close(got, want, tol, what):
    """|got - want| <= tol where want is finite as fp32; infinities and NaN in the same places."""
    got, want = got.cpu().double(), want.double()
    want32 = want.float().double()
    fin = torch.isfinite(want32)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), f"{what}: NaN in other places"
    inf = torch.isinf(want32)
    assert torch.equal(got[inf], want32[inf]), f"{what}: infinities differ"
    err = (got - want).abs()
    bad = fin & ~(err <= tol + FLUSHED)
    assert not bool(bad.any()), (f"{what}: {int(bad.sum())} of {want.numel()} off, first at {torch.nonzero(bad)[0].tolist()}: got "
                                 f"{got[bad][0]:.9e} want {want[bad][0]:.9e} tol {tol.expand_as(want)[bad][0]:.2e}")


def log_p_tol(stats, d, lp):
    """of ln p = d - log1p(rest): two roundings of d (and of its divisor), the sum, the result."""
    share = (stats[:, 1] / (1.0 + stats[:, 1])).abs()
    share = share.reshape(-1, *([1] * (d.dim() - 1)))
    return SUM_TOL * share + 4 * STEP * d.abs() + 2 * STEP * lp.abs()


def grad_tol(z, tau, stats, factor):
    """of factor * p_v: p's own relative error and the sum's."""
    lp, d = log_probs(z, tau, stats)
    p = torch.exp(lp)
    return factor.abs() * p * (SUM_TOL + (4 * d.abs().clamp(max=110.0) + 8) * STEP)
