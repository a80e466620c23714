"""The key-value cache at sizes that take more than one launch, more parts than a wave has lanes or a workgroup threads."""
import pytest
import torch

from paper_2407_09105_amd import binding
from tests.paged_util import DEV, Setup

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d,kind,tokens", [(1, "i8", 1_048_544 + 5003), (129, "plain", 262_136 + 1001), (129, "i8", 262_136 + 77)])
def test_rows_of_more_than_one_launch(d, kind, tokens):
    """64 heads, 2^24 - 1 workgroups at most in a launch.  Rows of 129 elements are read, and stored as they are, one to a workgroup: a launch
    ends at (2^24 - 1) / 64 - 7 = 262136 tokens; quantised ones of 1 or 129 are stored four to a workgroup, and end at 1048544."""
    hkv, page = 64, 64
    n_pages = -(-tokens // page)
    token, head, column = (torch.arange(n, dtype=torch.int32, device=DEV) for n in (tokens, hkv, d))
    # whole numbers of -125 .. 125 that neighbouring tokens, heads and columns do not share
    k = ((token[:, None] * 7 + head * 13) % 251)[..., None]
    k = ((k + column * 5) % 251 - 125).to(torch.bfloat16)
    if kind == "i8" and d > 1:   # the row's largest element is the largest step: scales of 1
        k[..., 0] = 127
    v = -k
    cache = binding.paged_cache(n_pages, page, hkv, d, torch.bfloat16 if kind == "plain" else torch.int8, DEV)
    table = torch.arange(n_pages, dtype=torch.int32, device=DEV).flip(0)[None]
    seq = torch.zeros(tokens, dtype=torch.int32, device=DEV)
    binding.paged_cache_write(k, v, cache, table, token, seq)
    full = tokens // page * page
    for pages, rows in ((cache.k, k), (cache.v, v)):
        if kind == "i8" and d == 1:   # all of them are their rows' largest
            rows = rows.sign() * 127
        stored = pages.flip(0).transpose(1, 2)     # [pages in the order of tokens, page, head, d]
        assert torch.equal(stored[:full // page].reshape(full, hkv, d).to(torch.bfloat16), rows[:full])
        assert torch.equal(stored[-1, :tokens - full].to(torch.bfloat16), rows[full:]) and not stored[-1, tokens - full:].any()
    if kind == "i8" and d > 1:
        assert all(int((s != 1).sum()) == hkv * (n_pages * page - tokens) for s in cache[2:])
    del stored, pages, rows
    out = binding.paged_cache_read(cache, table, token, seq)
    assert torch.equal(out[0], k) and torch.equal(out[1], v)


@pytest.mark.parametrize("d", [40, 128, 200])
def test_one_sequence_of_more_parts_than_a_workgroup_has_threads(d):
    """80000 keys for one head: 313 parts of 256."""
    Setup("bf16", "plain", 1, 1, d, 64, [80000], seed=d, garbage=False).check()


@pytest.mark.parametrize("kind", ["plain", "i8"])
def test_a_long_sequence_among_empty_ones(kind):
    """64 sequences for one head may have 768 more parts than one each, and one of them has 651 of three times 128 keys."""
    lens = [0] * 64
    lens[3], lens[40] = 17, 249_900
    Setup("f16", kind, 2, 1, 16, 256, lens, seed=5, garbage=False).check()


@pytest.mark.parametrize("d,hq", [(64, 1), (96, 3), (256, 5)])
def test_a_long_sequence_among_many_short_ones(d, hq):
    """300 sequences have room for fewer than eight parts each; one of them has 79."""
    lens = [(13 * b) % 50 for b in range(300)]
    lens[170] = 20_000
    Setup("bf16", "plain", hq, 1, d, 16, lens, seed=d, garbage=False).check()
