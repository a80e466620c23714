"""Quantised fp32 rows: every stored element is the nearest step, or the other neighbour of a quotient next to a tie."""
import pytest
import torch

from paper_2407_09105_amd import binding
from tests.paged_util import CACHES, DEV, TOPS

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["i8", "e4m3"])
@pytest.mark.parametrize("d", [128, 64, 100, 33])
def test_fp32_rows_are_off_at_ties_only(d, kind):
    """Elements of all magnitudes down to 2^-14 of the row's largest, e4m3's smallest step among them, both signs.  The quotient m x / a is
    formed with the roundings of m x, of 1 / f and of two fused multiply-adds, 2^-24 each: within 4 * 2^-24 of itself.  A stored element
    other than the nearest step to the exact quotient is the step on the other side of a tie that near."""
    n, hkv, page, top = 600, 3, 16, TOPS[kind]
    g = torch.Generator().manual_seed(d)
    x = torch.randn((n, hkv, d), generator=g) * torch.exp2(-14 * torch.rand((n, hkv, d), generator=g))
    x *= torch.exp2(torch.randint(-40, 41, (n, hkv, 1), generator=g).float())
    # and rows whose quotients lie on ties but for a rounding: x = a (i + 1/2) / m
    a = x[:50].abs().amax(-1, keepdim=True)
    steps = torch.arange(d).remainder(100) + 0.5
    x[:50] = a * steps / top
    x[:50, :, 0] = a[..., 0]
    cache = binding.paged_cache(-(-n // page), page, hkv, d, CACHES[kind], DEV)
    table = torch.arange(-(-n // page), dtype=torch.int32, device=DEV)[None]
    pos, seq = torch.arange(n, device=DEV), torch.zeros(n, dtype=torch.int32, device=DEV)
    binding.paged_cache_write(x.to(DEV), -x.to(DEV), cache, table, pos, seq)
    got = [c.cpu().float().double().transpose(1, 2).reshape(-1, hkv, d)[:n] for c in cache[:2]]
    assert torch.equal(got[0], -got[1])
    t = x.double() * top / x.double().abs().amax(-1, keepdim=True)
    step = torch.ones_like(t) if kind == "i8" else torch.exp2(torch.floor(torch.log2(t.abs().clamp(min=2.0 ** -6))) - 3)
    whole = t / step
    near = torch.round(whole)
    want = near * step
    other = got[0] != want
    tie = (whole.abs() - torch.floor(whole.abs()) - 0.5).abs() * step <= 4 * 2.0 ** -24 * t.abs()
    assert (tie | ~other).all()
    neighbour = (torch.floor(whole) + torch.ceil(whole) - near) * step
    assert torch.equal(got[0][other], neighbour[other])
    assert (t.abs() < 2.0 ** -6).any() and tie.any() and int(other.sum()) < int(tie.sum()) + 1
