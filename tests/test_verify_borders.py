"""The verification of drafts where a token hangs on the last bits of running sums: borders next to tokens that cannot be drawn,
sums of very many probabilities, and sums of very small ones.  What is right is computed in whole numbers.
"""

import math
import random
from fractions import Fraction

import pytest
import torch

from paper_2004_09362_gb300 import gar
from test_serving_operators import _verify_case, _verify_reference

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


@pytest.mark.gpu
@pytest.mark.parametrize("vocab", [1_000_003, 100_000_007])
def test_sums_of_many_probabilities(vocab):
    """Dense probabilities, multiples of 2^-24, and numbers u that come within 2^-41.5 to 2^-40 of a border between two tokens."""
    g = torch.Generator(device="cuda").manual_seed(3)
    m = torch.randint(1, 1 << 24, (vocab,), generator=g, device="cuda")
    upto = m.cumsum(0)
    total = int(upto[-1])
    j = torch.arange(1, 1 << 24, device="cuda")
    low = j * (total & 0xffffff)
    whole, part = j * (total >> 24) + (low >> 24), low & 0xffffff     # u times the sum, and its fraction in 2^-24
    token = torch.searchsorted(upto, whole, right=True)
    above, below = upto[token] - whole, whole - torch.where(token > 0, upto[(token - 1).clamp(min=0)], 0)
    off = torch.minimum(above.double() - part.double() / 2 ** 24, below.double() + part.double() / 2 ** 24) / total
    near = ((off >= 2.0 ** -41.5) & (off < 2.0 ** -40) & (token > 0) & (token < vocab - 1)).nonzero().flatten()
    near = near[torch.linspace(0, near.numel() - 1, min(64, near.numel()), device="cuda").long()]
    assert near.numel() >= 4
    n = near.numel()
    target = (m.float() / 2 ** 24)[None, None].expand(n, 1, vocab)
    none = torch.zeros((n, 0), dtype=I64, device="cuda")
    got, _ = gar.gar_verify_drafts(target, target[:, :0], none, (j[near].double() / 2 ** 24).float()[:, None])
    wrong = (got[:, 0] != token[near]).sum()
    assert int(wrong) == 0, (int(wrong), n)


@pytest.mark.gpu
@pytest.mark.parametrize("value", [8751087, 9007193, 8456019])
def test_sums_of_many_equal_probabilities(value):
    """Half of the tokens have one probability, half another: every addition of a lane rounds the same way."""
    vocab, half, other = 400_000_000, 200_000_000, 1 << 22
    target = torch.full((1, 1, vocab), value / 2 ** 24, device="cuda")
    target[..., half:] = other / 2 ** 24
    rng = random.Random(value)
    j = [rng.randrange(1, 1 << 24) for _ in range(16)]
    want = []
    for i in j:
        goal = i * (value + other) * half           # in 2^-24 of a value's step
        head = value * half << 24
        want.append(goal // (value << 24) if goal < head else half + (goal - head) // (other << 24))
    u = torch.tensor([[i / 2 ** 24] for i in j], device="cuda")
    none = torch.zeros((16, 0), dtype=I64, device="cuda")
    got, _ = gar.gar_verify_drafts(target.expand(16, 1, vocab), target.expand(16, 1, vocab)[:, :0], none, u)
    assert got[:, 0].tolist() == want, [a - b for a, b in zip(got[:, 0].tolist(), want)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_long_rows(dtype):
    """Drafts over a vocabulary whose rows are summed part by part; nothing left of the target; rows aligned alike and not."""
    vocab, n = 2_300_003, 4
    target, draft, tokens, uniform = _verify_case(n, 2, vocab, dtype, seed=6)
    draft[1] = target[1, :2] * 2
    uniform[1, 0], uniform[2:, 0] = 0.9, 0.99
    more = torch.full((n, 3, vocab + 5), math.nan, dtype=target.dtype, device="cuda")
    more[..., 1:1 + vocab] = target
    want, want_accepted = _verify_reference(target, draft, tokens, uniform)
    for p in (target, more[..., 1:1 + vocab]):
        got, accepted = gar.gar_verify_drafts(p, draft, tokens, uniform)
        assert torch.equal(got.cpu(), want) and torch.equal(accepted.cpu(), want_accepted)


@pytest.mark.gpu
@pytest.mark.parametrize("drafts", [0, 1])
def test_sums_of_the_smallest_numbers(drafts):
    """Eight tokens of 2^-149 each, all that there is or all that is left over of a draft: each is drawn by an eighth of the numbers."""
    vocab, n = 24, 64
    target = torch.zeros(n, drafts + 1, vocab, dtype=torch.float64)
    target[:, 0, 1::3] = 2.0 ** -149
    draft = torch.zeros(n, drafts, vocab, dtype=torch.float64)
    uniform = torch.zeros(n, drafts + 1)
    if drafts:
        target[:, 0, ::3] = 0.0625
        draft[:, 0, ::3] = 0.0625
        draft[:, 0, 2::3] = 0.0625               # the refused one: token 2
    uniform[:, -1] = (torch.arange(n) + 0.5) / n
    tokens = torch.full((n, drafts), 2, dtype=I64, device="cuda")
    got, accepted = gar.gar_verify_drafts(target.float().cuda(), draft.float().cuda(), tokens, uniform.cuda())
    assert bool((accepted == 0).all())
    assert got[:, 0].tolist() == [3 * (i // 8) + 1 for i in range(n)]
