"""The verification of drafts where a token hangs on the last bits of running sums: borders next to tokens that cannot be drawn.
What is right is computed in whole numbers.
"""

import random
from fractions import Fraction

import pytest
import torch

from paper_2004_09362_gb300 import gar

I64 = torch.int64


def _f32(x):
    """The largest 32-bit float up to x, a positive fraction."""
    y = torch.tensor(float(x), dtype=torch.float32)
    while Fraction(float(y)) > x:
        y = torch.nextafter(y, torch.zeros(()))
    return float(y)


def _border_case(rng, vocab, border, some):
    """({token: probability}, u) for which u times the sum is less than the running sum before token `border` by 2^-70 of it; `some`: the tokens
    that have weight, beside the last four.  Values spread over 40 powers of two, so that sums take more bits than twice 32-bit ones have."""
    r = {v: _f32(Fraction(rng.uniform(0.5, 1.0)) * Fraction(1, 2 ** rng.randint(12, 52))) for v in some}
    r[border - 1] = _f32(Fraction(rng.uniform(0.5, 1.0)) * Fraction(1, 2 ** 12))
    below, whole = sum(Fraction(x) for v, x in r.items() if v < border), sum(map(Fraction, r.values()))
    while True:
        u = rng.randrange(1, 2 ** 24) / 2 ** 24
        rest = below / Fraction(u) - whole       # what is missing to a sum of below / u
        if 0 < rest < 2:
            break
    for i in range(vocab - 4, vocab):
        r[i] = min(_f32(rest), 1.0) if rest > Fraction(1, 2 ** 120) else 0.0
        rest -= Fraction(r[i])
    return r, u


@pytest.mark.gpu
@pytest.mark.parametrize("vocab,batch,step,skipped,every", [(128, 800, 4, 3, 1), (32768, 150, 1024, 512, 64)])
def test_a_token_that_cannot_be_drawn_is_never_drawn(vocab, batch, step, skipped, every):
    """The goal lies next to the border before a group of four tokens, or a warp's run of 512, that begins with tokens without weight."""
    rng = random.Random(5)
    target, uniform, cases = torch.zeros(batch, 1, vocab), torch.zeros(batch, 1), []
    for b in range(batch):
        border = step * rng.randrange(3, vocab // step - 3)
        some = [v for v in range(every - 1, vocab - 4, every) if not border <= v < border + skipped]
        r, u = _border_case(rng, vocab, border, some)
        target[b, 0, list(r)], uniform[b, 0] = torch.tensor(list(r.values())), u
        cases.append(r)
    none = torch.zeros((batch, 0), dtype=I64, device="cuda")
    got, _ = gar.gar_verify_drafts(target.cuda(), target[:, :0].cuda(), none, uniform.cuda())
    got, bad, far = got[:, 0].tolist(), 0, Fraction(0)
    for b, t in enumerate(got):
        if cases[b].get(t, 0.0) == 0.0:
            bad += 1
            continue
        whole, below = sum(map(Fraction, cases[b].values())), sum(Fraction(x) for v, x in cases[b].items() if v < t)
        goal = Fraction(float(uniform[b, 0])) * whole
        far = max(far, (goal - below - Fraction(cases[b][t])) / whole, (below - goal) / whole)
    # A sum of two is off by 2^-47 of it at most (the low part's rounding, once as it is added up and once as it is put right), of which
    # a border here is made of 16 in turn at most: sums in a lane and over lanes, runs and pieces, and the product.
    assert bad == 0 and far <= Fraction(1, 2 ** 43), (bad, float(far))
