"""Plain 64-bit statements of window attention, the paged cache, key weights and eviction, and what rounding may add."""
import math

import torch

U32 = 2.0 ** -24                                   # half a step of fp32, relative
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: U32}


def sees(pos, L, window, sinks, start=0):
    """[rows, L]: whether the query at position pos[r] sees key j (window 0: no window)."""
    i, j = pos[:, None], torch.arange(L, device=pos.device)[None]
    seen = (j <= i) & (j >= start) if not torch.is_tensor(start) else (j <= i) & (j >= start[:, None])
    first = start if not torch.is_tensor(start) else start[:, None]
    return seen & ((j > i - window) | (j - first < sinks)) if window else seen


def attend(q, K, V, seen):
    """Rows q [n, d] over K, V [L, d] in 64 bits.  Returns O, lse, the probabilities, sum p |v|, and a bound on the error of a
    score whose products are summed in fp32 in any order: d U sum |q k| / sqrt(d), plus the rounding of its scaling."""
    d = q.shape[1]
    q, K, V = q.double(), K.double(), V.double()
    K = torch.where(seen.any(0)[:, None], K, 0.0)
    V = torch.where(seen.any(0)[:, None], V, 0.0)
    x = (q @ K.T / math.sqrt(d)).masked_fill(~seen, -math.inf)
    lse = torch.logsumexp(x, 1) if seen.shape[1] else torch.full((q.shape[0],), -math.inf, dtype=torch.float64, device=q.device)
    p = torch.where(seen, torch.exp(x - lse[:, None]), 0.0)
    size = (q.abs() @ K.abs().T / math.sqrt(d)).masked_fill(~seen, 0.0)
    delta = (d + 4) * U32 * (size.amax(1) if seen.shape[1] else lse * 0)
    return p @ V, lse, p, p @ V.abs(), delta


def check_rows(O, lse, q, K, V, seen, rounded_p=False, what=""):
    """Rows of an output against 64 bits.  A probability is off by 2 delta (its score's and its denominator's) and by the steps
    of exp2 and of the sums of n terms, n + 16 of them; rounding the probabilities to bf16 takes up to 2^-8 from numerator
    and denominator; O is rounded once."""
    ref, ref_lse, p, size, delta = attend(q, K, V, seen)
    none = ~seen.any(1)
    assert (O[none] == 0).all(), what
    n = int(seen.sum(1).max()) if seen.numel() else 0
    rel = 2 * delta[:, None] + (n + 16) * U32 + (2 * 2.0 ** -8 / (1 - 2.0 ** -8) if rounded_p else 0.0)
    tol = rel * size * 1.01 + (1 + rel) * HALF[O.dtype] * ref.abs() + 1e-30
    err = (O.double() - ref).abs()
    assert (err <= tol)[~none].all(), (what, float((err / tol)[~none].max()), float(err[~none].max()))
    if lse is not None:
        assert (lse[none] == -math.inf).all(), what
        tol = delta + (n + 16) * U32 + 4 * U32 * ref_lse.abs()
        err = (lse.double() - ref_lse).abs()
        assert (err <= tol)[~none].all(), (what, "lse", float((err / tol)[~none].max()))
    return p, delta, n


def fill_pages(cache, order, lengths):
    """Hands the pages of `order` out to sequences of these lengths."""
    page, width = cache.K.shape[2], cache.table.shape[1]
    table = torch.full(cache.table.shape, -1, dtype=torch.int32)
    at = 0
    for b, n in enumerate(lengths):
        used = -(-n // page)
        assert used <= width
        table[b, :used] = order[at:at + used]
        at += used
    cache.table.copy_(table)
    cache.length.copy_(torch.tensor(lengths, dtype=torch.int32))


def positions(cache, b, n, kv, what):
    """The first n positions of sequence b and KV head kv, [n, d] or [n]; and which of them have a page."""
    page = cache.K.shape[2]
    t = torch.arange(n, device=cache.K.device)
    e = cache.table[b].long()[t // page] if n else t
    good = (e >= 0) & (e < cache.K.shape[0])
    return getattr(cache, what)[torch.where(good, e, 0), kv, t % page], good
