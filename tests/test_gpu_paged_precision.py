"""How exactly attention over the key-value cache sums probabilities times values: where the sum cancels, far below the largest
probability, at scores near the types' limits and with values that are not finite."""
import math

import pytest
import torch

from paper_2407_09105_amd import binding
from tests.paged_util import CACHES, DEV, DTYPES, TOPS, Setup, attend64

pytestmark = pytest.mark.gpu


def _scores_in(t, x):
    """Scores near x as the sum of two elements of type t, exact in fp32: (first, second, sum)."""
    first = x.to(t).double()
    second = (x - first).to(t).double()
    return first, second, first + second


def _worst_in_16_bits(p):
    """Of p (float64) the two whose rounding to 16 significant bits changes them most, up and down: nearly 2^-16 of themselves.  (The ninth
    bit is set, so that two parts of 8 bits are 16; none lies so near to a tie that the exponential's own error turns it over.)"""
    step = torch.exp2(torch.floor(torch.log2(p)) - 15)
    rest = p / step - torch.round(p / step)
    worth = torch.where((torch.floor(p / step) % 256 >= 128) & (rest.abs() < 0.45), rest * step / p, 0.0)
    assert worth.min() < -0.8 * 2.0 ** -16 and worth.max() > 0.8 * 2.0 ** -16
    return int(worth.argmin()), int(worth.argmax())


CANCELLING = [("bf16", "plain", 64, 16), ("bf16", "plain", 128, 16), ("bf16", "plain", 72, 16), ("bf16", "plain", 256, 5), ("bf16", "plain", 34, 16),
              ("bf16", "plain", 33, 16), ("f16", "plain", 64, 16), ("f16", "plain", 128, 5), ("f16", "plain", 256, 16), ("f16", "plain", 33, 16),
              ("bf16", "i8", 128, 16), ("bf16", "i8", 64, 5), ("f16", "i8", 128, 16), ("bf16", "e4m3", 128, 16), ("f16", "e4m3", 256, 16),
              ("f16", "e4m3", 80, 24), ("f32", "plain", 64, 16), ("f32", "i8", 64, 16), ("f32", "e4m3", 128, 16)]


@pytest.mark.parametrize("dtype,kind,d,page", CANCELLING)
def test_probabilities_are_as_wide_as_fp32(dtype, kind, d, page):
    """Keys 1 and 2 have probabilities (over 8 bits: products of them and the scale of V) whose bits behind the first 16 are worth nearly
    2^-16 of them, one up and one down, and values of opposite signs; keys 3.. take away what is left of their sum, so that O is far
    smaller than its terms and the rounding of the result with it.  Key 0 holds the maximum, 0, and has no value.

    Off by, relative to A = sum_j P_j |v_j|: the exponent x = (S - max) log2 e, |x| <= X = 4 log2 e, is formed with three roundings, and a
    fourth where an 8-bit key has a scale, 2^-24 X each and times ln 2 in P; the exponential 2^-22; P times the scale of V 2^-24; up to three
    partial products for each of n keys and the four waves' results are added, 2^-23 of A each.  O is rounded once."""
    hkv, n, t = 2, 10, DTYPES[dtype]
    g = torch.Generator().manual_seed(d)
    many = -(0.5 + 3.4 * torch.rand(20000, generator=g, dtype=torch.float64))
    if kind == "plain":
        first, second, many = _scores_in(t, many)
    else:
        many = -(-many / TOPS[kind]).float().double() * TOPS[kind]
    used = [*_worst_in_16_bits(torch.exp(many))] + torch.randint(len(many), (n - 3,), generator=g).tolist()
    S = torch.cat([torch.zeros(1, dtype=torch.float64), many[used]])
    P = torch.exp(S)
    width = -(-n // page)
    k = torch.zeros((width, hkv, page, d), dtype=torch.float64)
    v, ks, vs = torch.zeros_like(k), torch.ones(width, hkv, page), torch.ones(width, hkv, page)
    left = torch.zeros((hkv, d), dtype=torch.float64)
    for j in range(n):
        at, row = j // page, j % page
        if kind != "plain":
            ks[at, :, row] = (-S[j] / TOPS[kind]).float()
            k[at, :, row, 0] = -TOPS[kind]
        elif j > 0:
            k[at, :, row, 0], k[at, :, row, 1] = first[used[j - 1]], second[used[j - 1]]
        want = (torch.zeros_like(left) if j == 0 else 1 + torch.rand((hkv, d), generator=g, dtype=torch.float64) if j == 1 else -left / P[j])
        if kind == "plain":
            v[at, :, row] = want = want.to(t).double()
        else:
            s = (want.abs().amax() / TOPS[kind]).float().expand(hkv)
            if j in (1, 2):    # P and the scale are one factor: the product is what has to be wide
                wider = s[0] * (1 + torch.rand(20000, generator=g))
                s = wider[_worst_in_16_bits(P[j] * wider.double())[j - 1]].expand(hkv)
            vs[at, :, row] = s
            steps = want / torch.where(s > 0, s, 1.0).double()[:, None]
            v[at, :, row] = steps = steps.round() if kind == "i8" else steps.float().to(CACHES[kind]).double()
            want = steps * s.double()[:, None]
        left += P[j] * want
    elements = t if kind == "plain" else CACHES[kind]
    scales = (None, None) if kind == "plain" else (ks.to(DEV), vs.to(DEV))
    cache = (k.float().to(elements).to(DEV), v.float().to(elements).to(DEV), *scales)
    q = torch.zeros((1, 2 * hkv, d), dtype=t)
    q[:, :, :2] = 1     # scores are the sums of the keys' first two columns
    q = q.to(DEV)
    table, lens = torch.arange(width, dtype=torch.int32, device=DEV)[None], torch.tensor([n], dtype=torch.int32, device=DEV)
    O, _, A, _ = attend64(q, cache, table, lens, 1.0)
    assert (O.abs() < 2.0 ** -14 * A).all()
    o, _ = binding.paged_attn_fwd(q, cache, table, lens, 1.0)
    rel = 4 * 2.0 ** -24 * 4 + 2.0 ** -22 + 2.0 ** -24 + (3 * n + 4) * 2.0 ** -23
    err = (o.cpu().double() - O).abs()
    tol = A * rel + torch.finfo(t).eps / 2 * O.abs() + torch.finfo(t).smallest_normal * torch.finfo(t).eps
    print("off by %.2e of the terms, tolerance %.2e" % (float((err / A).max()), rel))
    assert (err <= tol).all(), float((err / tol).max())


@pytest.mark.parametrize("dtype,kind,d,page,n", [("f16", "plain", 64, 16, 20000), ("f16", "plain", 128, 16, 9000), ("f16", "plain", 40, 24, 300),
                                                 ("f16", "plain", 33, 16, 9000), ("f16", "plain", 256, 32, 9000), ("f16", "i8", 64, 16, 9000),
                                                 ("f16", "e4m3", 128, 5, 9000), ("bf16", "plain", 64, 16, 9000), ("bf16", "i8", 64, 16, 300)])
@pytest.mark.parametrize("below", [12.0, 16.0, 18.0, 20.0, 22.0, 26.0])
def test_probabilities_far_below_the_largest(dtype, kind, d, page, n, below):
    """One key holds nearly all of the softmax and no value; the others, equal ones some nats below it, are all that O is made of.  Each
    is as exact as one near the largest.

    Relative to O (all terms have one sign): the exponent x = below log2 e, formed with four roundings of 2^-24 x; the exponential 2^-22; P
    times V's scale 2^-24; sums in fp32, of at most 75 keys in a wave (parts of 256 keys, or 300 uncut) and then of the waves and n / 256 parts,
    2^-23 each.  O is rounded once."""
    t, width = DTYPES[dtype], -(-n // page)
    g = torch.Generator().manual_seed(int(below))
    k, v = torch.zeros((width, 1, page, d)), torch.randint(1, 16, (width, 1, page, d), generator=g).float()
    at, row = n // 2 // page, n // 2 % page
    v[at, 0, row] = 0.0
    if kind == "plain":
        k[at, 0, row, 0] = below
        cache = (k.to(t).to(DEV), (v * 2048).to(t).to(DEV), None, None)
    else:
        k[at, 0, row, 0] = TOPS[kind]
        ks, vs = torch.ones((width, 1, page)), torch.full((width, 1, page), 2048.0)
        ks[at, 0, row] = below / TOPS[kind]
        cache = (k.to(CACHES[kind]).to(DEV), v.to(CACHES[kind]).to(DEV), ks.to(DEV), vs.to(DEV))
    q = torch.zeros((1, 2, d), dtype=t, device=DEV)
    q[:, :, 0] = 1
    table, lens = torch.arange(width, dtype=torch.int32, device=DEV)[None], torch.tensor([n], dtype=torch.int32, device=DEV)
    O, LSE, _, _ = attend64(q, cache, table, lens, 1.0)
    o, lse = binding.paged_attn_fwd(q, cache, table, lens, 1.0)
    fi = torch.finfo(t)
    rel = 4 * 2.0 ** -24 * below + 2.0 ** -22 + 2.0 ** -24 + (75 + 4 + n / 256) * 2.0 ** -23
    tol = (rel + fi.eps / 2) * O.abs() + fi.smallest_normal * fi.eps / 2
    err = (o.cpu().double() - O).abs()
    print("off by %.2e of O, tolerance %.2e" % (float((err / O).max()), rel + fi.eps / 2))
    assert (err <= tol).all(), float((err / tol).max())
    assert ((lse.cpu().double() - LSE).abs() <= 2.0 ** -22 * LSE.abs() + rel).all()


@pytest.mark.parametrize("dtype,kind,lens", [("bf16", "plain", [40, 9]), ("bf16", "plain", [3000, 700]), ("f32", "plain", [3000, 2]), ("f32", "i8", [40, 2600]),
                                             ("bf16", "plain", [150000])])
@pytest.mark.parametrize("sign", [-1.0, 1.0])
def test_scores_near_the_types_limits(dtype, kind, lens, sign):
    """Scores of 1 and 0.9 times the largest bf16 number, of either sign and in sequences that are cut or are not: the larger ones share the
    softmax, the others have nothing of it, and LSE is that score (the logarithm of some thousand changes nothing)."""
    t, page, d, n_pages = DTYPES[dtype], 16, 64, sum(-(-n // 16) for n in lens)
    width = max(-(-n // page) for n in lens)
    g = torch.Generator().manual_seed(len(lens))
    big = torch.finfo(torch.bfloat16).max
    less = float(torch.tensor(0.9 * big).bfloat16())
    high, low = sign * (big if sign > 0 else less), sign * (less if sign > 0 else big)
    k, v = torch.zeros((n_pages, 1, page, d)), torch.randint(-8, 9, (n_pages, 1, page, d), generator=g).float()
    table = torch.full((len(lens), width), -1, dtype=torch.int32)
    at = 0
    for b, n in enumerate(lens):
        table[b, :-(-n // page)] = torch.arange(at, at + -(-n // page))
        at += -(-n // page)
    scores = torch.full((n_pages, page), high)
    scores[::3] = low       # pages of the smaller scores, the first of them among these
    scales = (None, None)
    if kind == "plain":
        k[:, 0, :, 0] = scores
    else:
        k[:, 0, :, 0] = 1.0 if sign > 0 else -1.0
        scales = (scores.abs()[:, None].contiguous().to(DEV), torch.ones(n_pages, 1, page, device=DEV))
    elements = t if kind == "plain" else CACHES[kind]
    cache = (k.to(elements).to(DEV), v.to(elements).to(DEV), *scales)
    q = torch.zeros((len(lens), 2, d), dtype=t, device=DEV)
    q[:, :, 0] = 1
    given = torch.tensor(lens, dtype=torch.int32, device=DEV)
    o, lse = binding.paged_attn_fwd(q, cache, table.to(DEV), given, 1.0)
    for b, n in enumerate(lens):
        rows = v[table[b, :-(-n // page)].long(), 0].reshape(-1, d)[:n].double()
        mine = scores[table[b, :-(-n // page)].long()].reshape(-1)[:n]
        top = float(mine.max())
        want = rows[mine == top].mean(0)
        # whole numbers below 2^21 are added exactly; the sum of the weights (ones) too; one division and one rounding
        assert ((o[b].cpu().double() - want).abs() <= (torch.finfo(t).eps / 2 + 2.0 ** -22) * want.abs()).all()
        assert ((lse[:, b].cpu().double() - top).abs() <= 2.0 ** -23 * abs(top)).all()


@pytest.mark.parametrize("kind", ["plain", "i8", "e4m3"])
@pytest.mark.parametrize("bits", [0x7f800001, -0x7fffff, 0x7fc00000])
def test_nan_in_a_query_whatever_its_bits(kind, bits):
    """Of some NaNs only the last of the 24 bits tells them from infinity."""
    s = Setup("f32", kind, 2, 1, 64, 16, [40, 700])
    s.q.view(torch.int32)[:, 1, 3] = bits
    o, lse = s.attend()
    assert torch.isnan(o[:, 1]).all() and torch.isnan(lse[1]).all()
    assert torch.isfinite(o[:, 0]).all() and torch.isfinite(lse[0]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("below", [1.0, 20.0, 40.0, 60.0])
def test_infinite_values_of_small_probabilities(dtype, below):
    """An infinity in V comes out as one however little its key weighs, as long as it weighs anything; its sign and column are kept."""
    t = DTYPES[dtype]
    k, v = torch.zeros((4, 1, 16, 64)), torch.ones((4, 1, 16, 64))
    k[:, :, :, 0] = -below
    k[0, 0, 3, 0] = 0.0       # the key that holds the softmax
    v[1, 0, 5, 9], v[3, 0, 15, 40] = math.inf, -math.inf
    q = torch.zeros((1, 2, 64), dtype=t, device=DEV)
    q[:, :, 0] = 1
    table, lens = torch.arange(4, dtype=torch.int32, device=DEV)[None], torch.tensor([64], dtype=torch.int32, device=DEV)
    o, lse = binding.paged_attn_fwd(q, (k.to(t).to(DEV), v.to(t).to(DEV), None, None), table, lens, 1.0)
    assert (o[0, :, 9] == math.inf).all() and (o[0, :, 40] == -math.inf).all() and torch.isfinite(lse).all()
    others = torch.ones(64, dtype=torch.bool)
    others[[9, 40]] = False
    assert ((o[0][:, others.to(DEV)].float() - 1).abs() <= 2.0 ** -20).all()
