"""The key-value cache on the GPU against plain 64-bit arithmetic: rows in (quantised or not), rows out, attention of one token."""
import math

import pytest
import torch

from paper_2407_09105_amd import binding, workloads as wl
from tests.paged_util import CACHES, DEV, DTYPES, TOPS, Setup, attend64, cache_dtype, check_attention, place, quantise64, values64

pytestmark = pytest.mark.gpu


# ---- rows in and out -----------------------------------------------------------------------------------


def _rows(n, hkv, d, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    return [torch.randn((n, hkv, d), generator=g).to(DTYPES[dtype]).to(DEV) for _ in "kv"]


def _stream(lens, page, seed, spare=3, pad=0):
    """(table, position ids, sequence ids) of packed prompts of these lengths, `pad` tokens of no sequence behind them."""
    g = torch.Generator().manual_seed(seed)
    counts = [-(-n // page) for n in lens]
    order = torch.randperm(sum(counts) + spare, generator=g).to(torch.int32)
    table, at = torch.full((len(lens), max(counts + [1])), -1, dtype=torch.int32), 0
    for b, c in enumerate(counts):
        table[b, :c], at = order[at:at + c], at + c
    pos = torch.cat([torch.arange(n) for n in (*lens, pad)])
    seq = torch.cat([torch.full((n,), b, dtype=torch.int32) for b, n in enumerate((*lens, pad))])
    return table, pos, seq, sum(counts) + spare


def _expected(cache, k, v, table, pos, seq, kind):
    """The cache after a write, as values in float64 (k, v) and scales, from the cache before it."""
    before = [x.clone().cpu() if x is not None else None for x in cache]
    vals = [before[0].float().double(), before[1].float().double()]
    scales = [x.double() if x is not None else None for x in before[2:]]
    n_pages, _, page, _ = before[0].shape
    for i, x in enumerate((k, v)):
        x = x.cpu().double()
        s = None
        if kind != "plain":
            x, s = quantise64(x, kind)
        for t in range(len(pos)):
            at = place(table, page, n_pages, int(seq[t]), int(pos[t]))
            if at is not None:
                vals[i][at[0], :, at[1]] = x[t]
                if s is not None:
                    scales[i][at[0], :, at[1]] = s[t]
    return vals, scales


@pytest.mark.parametrize("kind", ["plain", "i8", "e4m3"])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("d,hkv,page", [(128, 2, 16), (64, 3, 1), (80, 1, 24), (256, 2, 7), (8, 5, 64), (33, 2, 5), (200, 1, 128), (1, 1, 3)])
def test_write_and_read(d, hkv, page, dtype, kind):
    lens = [37, 1, 64, 5]
    table, pos, seq, n_pages = _stream(lens, page, seed=d, pad=6)
    k, v = _rows(len(pos), hkv, d, dtype, seed=d + 1)
    cache = binding.paged_cache(n_pages, page, hkv, d, cache_dtype(dtype, kind), DEV)
    for x in cache:   # whatever lies in the cache stays but for the rows of the stream
        if x is not None:
            x.view(torch.uint8).fill_(3)
    vals, scales = _expected(cache, k, v, table, pos, seq, kind)
    binding.paged_cache_write(k, v, cache, table.to(DEV), pos.to(DEV), seq.to(DEV))
    for i in range(2):
        got = cache[i].cpu().float().double()
        if dtype == "f32" and kind != "plain":   # a quotient in fp32 may fall on the other side of a tie, one step away
            off = (got - vals[i]).abs()
            assert (off <= torch.maximum(vals[i].abs() / 8, torch.tensor(1.0))).all() and (off > 0).double().mean() < 1e-3
        else:
            assert torch.equal(got, vals[i])
        if kind != "plain":
            assert ((cache[2 + i].cpu().double() - scales[i]).abs() <= 2.0 ** -23 * scales[i]).all()
    # read back, in another order, tokens of no sequence among them: the cached value, rounded once
    order = torch.randperm(len(pos), generator=torch.Generator().manual_seed(5))
    out = binding.paged_cache_read(cache, table.to(DEV), pos[order].to(torch.int32).to(DEV), seq[order].to(DEV), dtype=DTYPES[dtype])
    for i in range(2):
        now = values64(cache[i], cache[2 + i])
        want = torch.zeros(len(pos), hkv, d, dtype=torch.float64)
        for t in range(len(pos)):
            at = place(table, page, n_pages, int(seq[order[t]]), int(pos[order[t]]))
            if at is not None:
                want[t] = now[at[0], :, at[1]]
        got = out[i].cpu().double()
        # the product with the scale is rounded to fp32 first
        assert ((got - want).abs() <= (torch.finfo(DTYPES[dtype]).eps / 2 + 2.0 ** -23) * want.abs() + torch.finfo(DTYPES[dtype]).tiny).all()
        if kind == "plain":
            assert torch.equal(got, want)


@pytest.mark.parametrize("kind", ["plain", "i8", "e4m3"])
@pytest.mark.parametrize("d,hkv,dtype,lens", [(80, 3, "bf16", [1500, 1, 1200]), (96, 2, "f16", [2000, 333]), (33, 2, "f32", [501, 600]),
                                              (72, 5, "f16", [2100]), (24, 1, "bf16", [9000]), (100, 1, "f32", [2500]), (8, 64, "bf16", [4200])])
def test_many_rows_of_odd_sizes(d, hkv, dtype, lens, kind):
    """Streams of many groups of tokens, the last of them ragged, rows that share memory lines with their neighbours'."""
    page = 13
    table, pos, seq, n_pages = _stream(lens, page, seed=d, pad=3)
    k, v = _rows(len(pos), hkv, d, dtype, seed=d + 7)
    cache = binding.paged_cache(n_pages, page, hkv, d, cache_dtype(dtype, kind), DEV)
    order = torch.randperm(len(pos), generator=torch.Generator().manual_seed(9))   # tokens of one page far apart
    binding.paged_cache_write(k[order.to(DEV)], v[order.to(DEV)], cache, table.to(DEV), pos[order].to(DEV), seq[order].to(DEV))
    n = sum(lens)
    pages, rows = table[seq[:n].long(), pos[:n] // page].long(), pos[:n] % page
    for i, x in enumerate((k, v)):
        want, scale = (x[:n].cpu().double(), None) if kind == "plain" else quantise64(x[:n].cpu().double(), kind)
        got = cache[i].cpu().float().double()[pages, :, rows]
        if dtype == "f32" and kind != "plain":   # as in test_write_and_read
            off = (got - want).abs()
            assert (off <= torch.maximum(want.abs() / 8, torch.tensor(1.0))).all() and (off > 0).double().mean() < 1e-3
        else:
            assert torch.equal(got, want)
        if scale is not None:
            assert ((cache[2 + i].cpu().double()[pages, :, rows] - scale).abs() <= 2.0 ** -23 * scale).all()
        used = torch.zeros(n_pages, page, dtype=torch.bool)
        used[pages, rows] = True
        assert (cache[i].cpu().float().transpose(1, 2)[~used] == 0).all()
    out = binding.paged_cache_read(cache, table.to(DEV), pos.to(DEV), seq.to(DEV), dtype=DTYPES[dtype])
    for i in range(2):
        want = values64(cache[i], cache[2 + i])[pages, :, rows]
        got = out[i].cpu().double()
        assert (got[n:] == 0).all()
        assert ((got[:n] - want).abs() <= (torch.finfo(DTYPES[dtype]).eps / 2 + 2.0 ** -23) * want.abs() + torch.finfo(DTYPES[dtype]).tiny).all()


@pytest.mark.parametrize("kind", ["i8", "e4m3"])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_rows_that_are_hard_to_quantise(dtype, kind):
    """Ties (a row whose largest element makes every half step exact), zeros, the type's largest and smallest numbers, and rows
    that are not finite, whose scale becomes NaN; their neighbours keep theirs."""
    fi = torch.finfo(DTYPES[dtype])
    d, top = 64, TOPS[kind]
    steps = torch.arange(d, dtype=torch.float64)
    amax = 127.0 if kind == "i8" else 448.0   # the row's largest element is the largest step itself: x = q
    half = torch.cat([steps[:-1] + 0.5, torch.tensor([amax], dtype=torch.float64)])
    rows = [half, -half, torch.zeros(d), torch.full((d,), fi.max), torch.full((d,), fi.tiny), torch.linspace(-1, 1, d) * fi.max,
            torch.linspace(-1, 1, d) * fi.tiny * 64, torch.cat([torch.tensor([float("nan")]), steps[1:]]),
            torch.cat([steps[:-1], torch.tensor([-float("inf")])]), steps, steps * 2.0 ** -10]
    x = torch.stack([r.double() for r in rows]).to(DTYPES[dtype])
    n = len(rows)
    k = x[:, None].contiguous().to(DEV)
    cache = binding.paged_cache(1, n, 1, d, CACHES[kind], DEV)
    table, pos = torch.zeros((1, 1), dtype=torch.int32, device=DEV), torch.arange(n, device=DEV)
    binding.paged_cache_write(k, k, cache, table, pos, torch.zeros(n, dtype=torch.int32, device=DEV))
    bad = [7, 8]
    fine = [i for i in range(n) if i not in bad]
    q, s = quantise64(x[fine].double(), kind)
    for i in range(2):
        got, scale = cache[i].cpu().float().double()[0, 0], cache[2 + i].cpu().double()[0, 0]
        assert torch.equal(got[fine], q)
        assert torch.isnan(scale[bad]).all() and (got[bad] == 0).all()
        assert ((scale[fine] - s).abs() <= 2.0 ** -23 * s + 2.0 ** -149).all()
    out, _ = binding.paged_cache_read(cache, table, pos, torch.zeros(n, dtype=torch.int32, device=DEV), dtype=torch.float32)
    assert torch.isnan(out[bad]).all() and torch.isfinite(out[fine]).all()


@pytest.mark.parametrize("kind", ["plain", "i8"])
def test_tokens_without_a_place(kind):
    """Sequences, positions and pages that do not exist, in 32 and 64 bits, store nothing and read as zeros."""
    page, hkv, d, n_pages = 4, 2, 64, 5
    table = torch.tensor([[1, -1, 7, 4], [5, 2, 0, -2 ** 31]], dtype=torch.int32)
    seq = torch.tensor([0, 0, 0, 0, 0, 1, 1, 1, 1, 2, -1, 2 ** 31 - 1, 0, 1], dtype=torch.int32)
    pos = torch.tensor([0, 3, 4, 8, 15, 0, 4, 11, 12, 0, 0, 0, 16, -1])
    cache = binding.paged_cache(n_pages, page, hkv, d, cache_dtype("bf16", kind), DEV)
    k, v = _rows(len(pos), hkv, d, "bf16", 3)
    vals, _ = _expected(cache, k, v, table, pos, seq, kind)
    for wide in (False, True):
        p = pos.clone() if wide else pos.to(torch.int32)
        if wide:
            p[12], p[13] = 2 ** 32, -2 ** 32 + 2    # low halves that would be places
        binding.paged_cache_write(k, v, cache, table.to(DEV), p.to(DEV), seq.to(DEV))
        for i in range(2):
            assert torch.equal(cache[i].cpu().float().double(), vals[i])
        out = binding.paged_cache_read(cache, table.to(DEV), p.to(DEV), seq.to(DEV))
        none = torch.tensor([place(table, page, n_pages, int(s), int(t)) is None for s, t in zip(seq, pos)])
        assert int(none.sum()) == 9
        for x in out:
            assert (x[none.to(DEV)] == 0).all() and (x[~none.to(DEV)] != 0).any(-1).all()
    # nothing at all
    binding.paged_cache_write(k[:0], v[:0], cache, table.to(DEV), pos[:0].to(DEV), seq[:0].to(DEV))
    assert binding.paged_cache_read(cache, table.to(DEV), pos[:0].to(DEV))[0].shape == (0, hkv, d)
    binding.paged_cache_write(k[:2], v[:2], cache, table[:, :0].contiguous().to(DEV), pos[:2].to(DEV))
    assert torch.equal(cache[0].cpu().float().double(), vals[0])


def test_one_new_token_of_every_sequence():
    """Without sequence ids token t is sequence t's; a table that is a part of a wider one; tensors at odd addresses."""
    page, hkv, d, B = 8, 3, 40, 11
    wide = torch.full((B, 9), 3, dtype=torch.int32)
    wide[:, 2:6] = torch.randperm(44, generator=torch.Generator().manual_seed(1)).view(B, 4)
    wide = wide.to(DEV)
    table, pos = wide[:, 2:6], (torch.arange(B) * 3 % 32).to(DEV)
    rows = torch.randn(2, B * hkv * d + 1, device=DEV).bfloat16()
    k, v = rows[0, 1:].view(B, hkv, d), rows[1, 1:].view(B, hkv, d)   # not on 16 bytes
    for kind in ("plain", "i8", "e4m3"):
        cache = binding.paged_cache(44, page, hkv, d, cache_dtype("bf16", kind), DEV)
        vals, _ = _expected(cache, k, v, table.cpu(), pos.cpu(), torch.arange(B), kind)
        binding.paged_cache_write(k, v, cache, table, pos)
        for i in range(2):
            assert torch.equal(cache[i].cpu().float().double(), vals[i])
        out = torch.full((2, B * hkv * d + 1), 7.0, device=DEV).bfloat16()
        got = binding.paged_cache_read(cache, table, pos, out=(out[0, 1:].view(B, hkv, d), out[1, 1:].view(B, hkv, d)))
        aligned = binding.paged_cache_read(cache, table, pos)
        assert torch.equal(got[0], aligned[0]) and torch.equal(got[1], aligned[1]) and (out[:, 0] == 7).all()
        if kind == "plain":
            assert torch.equal(got[0], k) and torch.equal(got[1], v)


# ---- attention -----------------------------------------------------------------------------------------

LENS = [0, 1, 2, 15, 16, 17, 31, 33, 64, 127, 128, 129, 300]


@pytest.mark.parametrize("kind", ["plain", "i8", "e4m3"])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("hq,hkv,d,page", [(4, 1, 128, 16), (2, 2, 64, 32), (16, 1, 64, 1), (20, 1, 128, 48), (6, 2, 256, 64), (3, 3, 80, 16),
                                           (8, 2, 96, 24), (5, 1, 72, 16), (4, 2, 33, 16), (4, 2, 8, 7), (40, 1, 136, 5), (1, 1, 1, 3)])
def test_attention(hq, hkv, d, page, dtype, kind):
    Setup(dtype, kind, hq, hkv, d, page, LENS, seed=d + page).check()


@pytest.mark.parametrize("kind", ["plain", "i8", "e4m3"])
@pytest.mark.parametrize("dtype,lens,page,hq,hkv,d", [
    ("bf16", [5000], 16, 4, 1, 128), ("f16", [4097, 3], 32, 2, 2, 64), ("bf16", [1, 2600, 700, 0], 7, 16, 2, 128),
    ("f32", [3000], 16, 2, 1, 64), ("bf16", [2049] * 3, 64, 2, 1, 256), ("bf16", [3001, 1], 1, 17, 1, 80),
    ("f16", [1500, 20], 24, 3, 1, 33), ("bf16", [1111, 600], 16, 2, 2, 72), ("f32", [900, 2000], 5, 4, 2, 100), ("f16", [1300], 48, 2, 1, 200)])
def test_long_sequences(dtype, lens, page, hq, hkv, d, kind):
    Setup(dtype, kind, hq, hkv, d, page, lens, seed=len(lens) + page).check()


@pytest.mark.parametrize("dtype,kind,hq,hkv,d,page", [
    ("f32", "plain", 4, 2, 33, 16), ("f32", "plain", 2, 2, 5, 4), ("f32", "plain", 3, 1, 66, 7), ("f32", "plain", 2, 1, 131, 16),
    ("f32", "plain", 2, 1, 255, 8), ("f32", "i8", 4, 2, 100, 16), ("f32", "e4m3", 4, 2, 20, 1), ("f32", "i8", 2, 1, 252, 3),
    ("f32", "e4m3", 2, 2, 60, 24), ("bf16", "plain", 4, 1, 42, 16), ("f16", "plain", 2, 2, 10, 5), ("bf16", "plain", 2, 1, 250, 16),
    ("f16", "plain", 17, 1, 126, 3), ("bf16", "i8", 4, 1, 36, 16), ("f16", "e4m3", 2, 2, 124, 7), ("bf16", "e4m3", 2, 1, 244, 16),
    ("f16", "i8", 2, 1, 28, 2), ("bf16", "i8", 3, 1, 12, 16), ("f16", "plain", 2, 1, 6, 16), ("f32", "plain", 2, 1, 3, 16)])
def test_rows_that_end_inside_a_chunk(dtype, kind, hq, hkv, d, page):
    Setup(dtype, kind, hq, hkv, d, page, [0, 1, 31, 33, 257, 700], seed=d).check()


@pytest.mark.parametrize("kind", ["i8", "e4m3"])
@pytest.mark.parametrize("d,page", [(64, 16), (100, 5), (128, 32), (33, 16), (256, 1)])
def test_fp32_queries_of_many_magnitudes(d, page, kind):
    """All bits of a query's element count: large ones that cancel, small ones beside them, and one that is not finite."""
    s = Setup("f32", kind, 4, 2, d, page, [300, 40, 5], seed=3)
    g = torch.Generator().manual_seed(4)
    s.q *= (10 ** (torch.rand(s.q.shape, generator=g) * 6 - 5)).to(DEV)
    s.check()
    s.q[1, 2, 3], s.q[2, 0, 1] = float("nan"), float("inf")
    o, lse = s.attend()
    want, log = attend64(s.q, s.cache, s.table, s.lens)[:2]
    assert torch.equal(torch.isnan(o.cpu()), torch.isnan(want)) and torch.equal(torch.isnan(lse.cpu()), torch.isnan(log))
    assert int(torch.isnan(o).sum()) == 2 * d
    assert torch.equal(lse.cpu() == float("inf"), log == float("inf"))


@pytest.mark.parametrize("kind", ["plain", "i8"])
@pytest.mark.parametrize("dtype,lens", [("bf16", [700, 3]), ("f16", [2500]), ("f32", [1500, 40])])
def test_scores_of_infinity(dtype, lens, kind):
    """O is NaN as softmax is, and LSE infinity, unless a score is NaN."""
    s = Setup(dtype, kind, 4, 2, 64, 16, lens)
    s.q[0, 0, 5], s.q[-1, 2, 7], s.q[-1, 3, 9] = float("inf"), -float("inf"), float("nan")
    o, lse = s.attend()
    want, log = attend64(s.q, s.cache, s.table, s.lens)[:2]
    assert torch.equal(torch.isnan(o.cpu()), torch.isnan(want))
    assert torch.equal(torch.isnan(lse.cpu()), torch.isnan(log)) and torch.equal(lse.cpu() == float("inf"), log == float("inf"))


@pytest.mark.parametrize("dtype,kind,d,off", [("bf16", "plain", 128, 2), ("f32", "plain", 64, 1), ("f16", "i8", 128, 4), ("bf16", "e4m3", 256, 4),
                                              ("f16", "plain", 64, 1), ("bf16", "i8", 64, 1)])
def test_pages_at_odd_addresses(dtype, kind, d, off):
    s = Setup(dtype, kind, 4, 2, d, 16, [130, 0, 77])
    moved = []
    for x in s.cache[:2]:
        y = torch.zeros(x.numel() + off, dtype=x.dtype, device=DEV)[off:].view(x.shape)
        moved.append(y.copy_(x))
    s.cache = (*moved, *s.cache[2:])
    s.check()


@pytest.mark.parametrize("kind", ["plain", "i8"])
def test_many_sequences(kind):
    """More sequences than a wave has lanes, than the chip has room for parts of."""
    lens = [(7 * b * b + b) % 190 for b in range(333)]
    lens[200] = 2500
    Setup("bf16", kind, 2, 1, 64, 16, lens, seed=9).check()


@pytest.mark.parametrize("page", [16, 48, 5])
@pytest.mark.parametrize("kind", ["plain", "i8", "e4m3"])
def test_entries_that_are_no_page(page, kind):
    """Their tokens are left out, wherever they stand; a sequence of none but such entries is empty; the lengths may pass the table."""
    s = Setup("bf16", kind, 8, 2, 64, page, [5 * page, 4 * page + 1, 3 * page, 40 * page], seed=page, width=40)
    t = s.table
    t[0, 0], t[0, 3] = -1, s.cache[0].shape[0]
    t[1, 4] = 2 ** 31 - 1
    t[2, :3] = -2 ** 31
    t[3, 1:30:2] = -1
    s.lens[0], s.lens[3] = 5 * page, 2 ** 31 - 1
    o, lse = s.check()
    assert (o[2] == 0).all() and (lse[:, 2] == -math.inf).all()
    s.lens[1] = -5
    o, lse = s.check()
    assert (o[1] == 0).all() and (lse[:, 1] == -math.inf).all()


@pytest.mark.parametrize("dtype,kind", [("bf16", "plain"), ("f16", "i8"), ("bf16", "e4m3"), ("f32", "plain")])
@pytest.mark.parametrize("scale", [1.0, 0.01, 30.0])
def test_softmax_scale(dtype, kind, scale):
    """Nearly one-hot and nearly even softmaxes: with 30 the scores reach some hundreds."""
    Setup(dtype, kind, 4, 2, 64, 16, [700, 33], seed=4).check(scale)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_values_that_are_not_finite(dtype):
    """An infinity or NaN in a key or value of a sequence shows where the formula has it, and nowhere else."""
    s = Setup(dtype, "plain", 2, 1, 64, 16, [40, 40, 40, 200], seed=2)
    clean, clean_lse = s.attend()
    k, v = s.cache[:2]
    v[s.table[0, 1].item(), 0, 3, 5] = math.inf         # O column 5 of sequence 0: inf
    v[s.table[1, 2].item(), 0, 7, 9] = math.nan         # O column 9 of sequence 1: NaN
    k[s.table[2, 0].item(), 0, 0, :] = math.nan         # all of sequence 2
    o, lse = s.attend()
    assert (o[0, :, 5] == math.inf).all() and torch.isnan(o[1, :, 9]).all() and torch.isnan(o[2]).all()
    keep = torch.ones_like(o, dtype=torch.bool)
    keep[0, :, 5] = keep[1, :, 9] = keep[2] = False
    assert torch.equal(o[keep], clean[keep]) and torch.equal(lse[:, [0, 1, 3]], clean_lse[:, [0, 1, 3]])


def test_scores_of_minus_infinity():
    """Keys that score -inf weigh nothing; where all do, nothing is left and O is zero."""
    s = Setup("bf16", "plain", 1, 1, 64, 16, [40, 16], seed=6, garbage=False)
    s.q[:] = s.q.abs() + 0.1
    s.cache[0][s.table[0, 0].item(), 0, 2:5] = -math.inf
    s.cache[0][s.table[1, 0].item()] = -math.inf
    o, lse = s.attend()
    K = values64(s.cache[0], None)
    rows = [place(s.table.cpu(), 16, K.shape[0], 0, j) for j in range(40)]
    rows = [r for j, r in enumerate(rows) if j not in (2, 3, 4)]
    k = torch.stack([K[p, 0, r] for p, r in rows])
    v = torch.stack([values64(s.cache[1], None)[p, 0, r] for p, r in rows])
    w = torch.softmax(k @ s.q[0, 0].cpu().double() / 8, 0)
    assert ((o[0, 0].cpu().double() - w @ v).abs() <= 2.0 ** -8 * (w @ v).abs() + 2.0 ** -14 * (w @ v.abs())).all()
    assert (o[1] == 0).all() and lse[0, 1] == -math.inf


def test_offsets_past_32_bits():
    """Pages beyond 4 GiB of each tensor: bytes of a row's offset need more than 32 bits, elements more than 31."""
    page, hkv, d = 64, 8, 128
    n_pages = (1 << 32) // (page * hkv * d * 2) + 40
    k = torch.zeros((n_pages, hkv, page, d), dtype=torch.bfloat16, device=DEV)
    v = torch.zeros_like(k)
    table = torch.stack([torch.arange(n_pages - 8, n_pages), torch.arange(8)]).to(torch.int32).to(DEV)
    n = 8 * page - 3
    rows_k, rows_v = _rows(2 * n, hkv, d, "bf16", 8)
    seq = torch.arange(2, device=DEV, dtype=torch.int32).repeat_interleave(n)
    pos = torch.arange(n, device=DEV).repeat(2)
    binding.paged_cache_write(rows_k, rows_v, (k, v, None, None), table, pos, seq)
    assert torch.equal(k[-8:].transpose(1, 2).reshape(-1, hkv, d)[:n], rows_k[:n])
    assert torch.equal(v[:8].transpose(1, 2).reshape(-1, hkv, d)[:n], rows_v[n:])
    assert not k[8:-8].any() and not v[8:-8].any()
    out = binding.paged_cache_read((k, v, None, None), table, pos, seq)
    assert torch.equal(out[0], rows_k) and torch.equal(out[1], rows_v)
    q = torch.randn(2, 16, d, device=DEV).bfloat16()
    o, lse = binding.paged_attn_fwd(q, (k, v, None, None), table, torch.tensor([n, n], dtype=torch.int32, device=DEV))
    near = (torch.cat([k[-8:], k[:8]]), torch.cat([v[-8:], v[:8]]), None, None)
    small = torch.arange(16, dtype=torch.int32).view(2, 8).to(DEV)
    check_attention(o, lse, attend64(q, near, small, torch.tensor([n, n])), "bf16", n)


def test_more_rows_than_a_launch_has_room_for():
    """2^28 rows of one element: a launch ends at 2^26 of them."""
    n, hkv, page = 1 << 22, 64, 64
    k = torch.arange(n * hkv, device=DEV).remainder(251).to(torch.bfloat16).view(n, hkv, 1)
    v = -k
    cache = binding.paged_cache(n // page, page, hkv, 1, torch.bfloat16, DEV)
    table = torch.arange(n // page, dtype=torch.int32, device=DEV).flip(0)[None]
    pos, seq = torch.arange(n, device=DEV), torch.zeros(n, dtype=torch.int32, device=DEV)
    binding.paged_cache_write(k, v, cache, table, pos, seq)
    assert torch.equal(cache.k.flip(0).transpose(1, 2).reshape(n, hkv, 1), k)
    out = binding.paged_cache_read(cache, table, pos, seq)
    assert torch.equal(out[0], k) and torch.equal(out[1], v)


def test_more_sequences_than_cuts():
    """Thousands of short sequences, some empty, and a long one among them, in a table that would let all be long."""
    lens = [(31 * b) % 41 for b in range(4099)]
    lens[4000] = 3100
    Setup("f16", "e4m3", 3, 1, 8, 16, lens, seed=17, width=200, garbage=False).check()


@pytest.mark.parametrize("page", [16, 5])
@pytest.mark.parametrize("kind", ["i8", "e4m3"])
def test_poisoned_rows(kind, page):
    """A cached row that was not finite (scale NaN) makes its sequence's and KV head's results NaN, and no others'."""
    s = Setup("bf16", kind, 4, 2, 64, page, [50, 50, 700], seed=8, width=300)
    clean, clean_lse = s.attend()
    s.cache[2][s.table[0, 1].item(), 0, 3] = math.nan    # K, heads 0 and 1 of sequence 0
    s.cache[3][s.table[2, 60].item(), 1, 4] = math.nan   # V, heads 2 and 3 of sequence 2
    o, lse = s.attend()
    bad = torch.zeros_like(o, dtype=torch.bool)
    bad[0, :2] = bad[2, 2:] = True
    assert torch.isnan(o[bad]).all() and torch.equal(o[~bad], clean[~bad])
    assert torch.isnan(lse[:2, 0]).all() and torch.equal(lse[2:, 0], clean_lse[2:, 0]) and torch.equal(lse[:, 1:], clean_lse[:, 1:])


def test_calls_at_once():
    """On two streams and from two threads, each with workspaces of its own."""
    import threading
    sets = [Setup("bf16", kind, 8, 2, 128, 16, [5000, 7, 900], seed=40 + i, garbage=False) for i, kind in enumerate(("plain", "i8"))]
    want = [s.attend() for s in sets]
    got = [[], []]
    torch.cuda.synchronize()

    def work(i):
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            for _ in range(20):
                got[i].append(sets[i].attend())
        stream.synchronize()

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    [t.start() for t in threads]
    [t.join() for t in threads]
    for i in range(2):
        assert len(got[i]) == 20 and all(torch.equal(o, want[i][0]) and torch.equal(lse, want[i][1]) for o, lse in got[i])


def test_shared_pages_and_given_outputs():
    """Two sequences with the same prefix pages; outputs and workspace that the caller brings, full of NaN before."""
    s = Setup("bf16", "e4m3", 8, 2, 128, 16, [1000, 100], seed=12)
    s.table[1, :6] = s.table[0, :6]
    o = torch.full_like(s.q, math.nan)
    lse = torch.full((8, 2), math.nan, device=DEV)
    ws = binding.paged_attn_workspace(s.q, s.cache, s.table).fill_(math.nan)
    got = s.attend(out=o, lse=lse, workspace=ws)
    assert got[0] is o and got[1] is lse
    check_attention(o, lse, attend64(s.q, s.cache, s.table, s.lens), "bf16", 1000)
    again = s.attend()
    assert torch.equal(again[0], o) and torch.equal(again[1], lse)


# ---- together ------------------------------------------------------------------------------------------


@pytest.mark.parametrize("kind", ["plain", "i8", "e4m3"])
def test_prompts_and_decoding_steps(kind):
    """What generation does: packed prompts with padding behind them through rotary embedding, attention and cache, then single
    tokens.  Every step's O is the last row that the forward gives over the whole sequence with the same keys and values."""
    hq, hkv, d, page, steps = 8, 2, 64, 16, 4
    lens = [50, 3, 129, 16]
    B = len(lens)
    g = torch.Generator().manual_seed(77)
    rnd = lambda *s: torch.randn(s, generator=g).bfloat16().to(DEV)  # noqa: E731
    full = [(rnd(n + steps, hq, d), rnd(n + steps, hkv, d), rnd(n + steps, hkv, d)) for n in lens]
    cat = lambda i: torch.cat([full[b][i][:n] for b, n in enumerate(lens)] + [rnd(5, hq if i == 0 else hkv, d)])  # noqa: E731
    pos = torch.from_numpy(wl.position_ids_from_lengths([lens + [5]])).to(DEV)
    q, k, v = (binding.rope_apply(cat(0), pos), binding.rope_apply(cat(1), pos), cat(2))
    seg = binding.pack_to_cu_seqlens(pos)
    prompt_o, _ = binding.varlen_attn_fwd(q, k, v, seg)
    cache = binding.paged_cache(64, page, hkv, d, cache_dtype("bf16", kind), DEV)
    table = torch.randperm(64, generator=g)[:B * 12].view(B, 12).to(torch.int32).to(DEV)
    binding.paged_cache_write(k, v, cache, table, pos, seg.seg_id)

    def whole(b, n):
        """Rows of sequence b as they are cached."""
        return binding.paged_cache_read(cache, table, torch.arange(n, device=DEV), torch.full((n,), b, dtype=torch.int32, device=DEV))

    at = 0
    for b, n in enumerate(lens):
        if kind == "plain":
            kk, vv = whole(b, n)
            assert torch.equal(kk, k[at:at + n]) and torch.equal(vv, v[at:at + n])
        at += n
    now = torch.tensor(lens, dtype=torch.int32, device=DEV)
    for step in range(steps):
        new = [torch.stack([full[b][i][n + step] for b, n in enumerate(lens)]) for i in range(3)]
        qn, kn = binding.rope_apply(new[0], now), binding.rope_apply(new[1], now)
        binding.paged_cache_write(kn, new[2], cache, table, now)
        now += 1
        o, lse = binding.paged_attn_fwd(qn, cache, table, now)
        check_attention(o, lse, attend64(qn, cache, table, now), "bf16", 140)
        for b, n in enumerate(lens):
            m = n + step + 1
            kk, vv = whole(b, m)
            qq = binding.rope_apply(full[b][0][:m].contiguous(), torch.arange(m, device=DEV))
            one = binding.pack_to_cu_seqlens(torch.arange(m, device=DEV)[None])
            ref, ref_lse = binding.varlen_attn_fwd(qq, kk, vv, one)
            # both within the forward's bar of the formula (max-abs 2e-2); rows out of an 8-bit cache are rounded to bf16 for
            # the forward, at most 2^-8 of each product of a score and of each value
            assert (ref[-1].float() - o[b].float()).abs().max() <= 2e-2 + (0 if kind == "plain" else 2.0 ** -8 * 4)
            assert (ref_lse[:, -1] - lse[:, b]).abs().max() <= (1e-3 if kind == "plain" else 2.0 ** -8 * 4)


def test_other_stream_and_captured_graph():
    """On a stream of its own, and captured: replays see the lengths, pages and rows of their own time."""
    s = Setup("bf16", "plain", 8, 2, 128, 16, [700, 20, 0, 33], seed=3, garbage=False, width=80, spare=40)
    k, v = _rows(4, 2, 128, "bf16", 1)
    cache = tuple(x if x is None else x.clone() for x in s.cache)
    side = torch.cuda.Stream()

    def step():
        binding.paged_cache_write(k, v, cache, s.table, s.lens)
        return binding.paged_attn_fwd(s.q, cache, s.table, s.lens + 1)

    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        o, lse = step()
    torch.cuda.current_stream().wait_stream(side)
    check_attention(o, lse, attend64(s.q, cache, s.table, s.lens + 1), "bf16", 701)
    graph = torch.cuda.CUDAGraph()
    other = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o, lse = step()
    with torch.cuda.graph(other):     # a second one with workspaces of its own
        o2, lse2 = binding.paged_attn_fwd(s.q, cache, s.table, s.lens)
    for it in range(4):
        s.lens += torch.tensor([1, 16, 0, 97], dtype=torch.int32, device=DEV)
        s.table[2, 0] = 5 if it % 2 else -1
        k.copy_(torch.randn_like(k))
        s.q.copy_(torch.randn_like(s.q))
        graph.replay()
        other.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in (o, lse, o2, lse2)]
        want = (*step(), *binding.paged_attn_fwd(s.q, cache, s.table, s.lens))
        for a, b in zip(got, want):
            assert torch.equal(a, b)
        torch.cuda.synchronize()


def test_results_do_not_change_from_call_to_call():
    s = Setup("bf16", "i8", 32, 8, 128, 16, [9000, 3, 1200], seed=21, garbage=False)
    first = s.attend()
    for _ in range(5):
        again = s.attend()
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


@pytest.mark.parametrize("kind", ["plain", "i8", "e4m3"])
def test_cpp_marshalling_takes_the_plain_calls(kind, monkeypatch):
    """The calls of a decoding step marshal in C++ and give what the ctypes calls give; what differs goes through Python."""
    s = Setup("bf16", kind, 8, 2, 64, 16, [40, 300, 0], seed=31, garbage=False, width=24, spare=8)
    k, v = _rows(3, 2, 64, "bf16", 7)
    native, taken = binding._native, []
    assert native is not None

    class Spy:
        def __getattr__(self, name):
            def call(*args):
                got = getattr(native, name)(*args)
                taken.append((name, type(got).__name__))
                return got
            return call

    def step(cache):
        binding.paged_cache_write(k, v, cache, s.table, s.lens)
        rows = binding.paged_cache_read(cache, s.table, s.lens, torch.arange(3, dtype=torch.int32, device=DEV), dtype=torch.bfloat16)
        return (*rows, *binding.paged_attn_fwd(s.q, cache, s.table, s.lens + 1), *(x for x in cache if x is not None))

    monkeypatch.setattr(binding, "_native", Spy())
    caches = [tuple(x if x is None else x.clone() for x in s.cache) for _ in range(3)]
    got = step(binding.PagedCache(*caches[0]))
    assert taken == [("cache_write", "int"), ("cache_read", "tuple"), ("paged", "tuple")]
    del taken[:]
    lists = step(list(caches[1]))       # no tuple
    assert [t for _, t in taken] == ["NoneType"] * 3
    monkeypatch.setattr(binding, "_native", None)
    for a, b, c in zip(got, step(caches[2]), lists):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)) and torch.equal(a.view(torch.uint8), c.view(torch.uint8))
    # errors are the same with and without it
    for n in (native, None):
        monkeypatch.setattr(binding, "_native", n)
        with pytest.raises(ValueError, match="multiple"):
            binding.paged_attn_fwd(torch.zeros(3, 5, 64, device=DEV, dtype=torch.bfloat16), s.cache, s.table, s.lens)
        with pytest.raises(TypeError):
            binding.paged_attn_fwd(s.q, s.cache, s.table, s.lens.long())
        with pytest.raises(binding.VarlenAttnError, match="unsupported"):
            wide = tuple(torch.zeros(4, 1, 16, 264, device=DEV, dtype=torch.bfloat16) for _ in "kv") + (None, None)
            binding.paged_attn_fwd(torch.zeros(3, 1, 264, device=DEV, dtype=torch.bfloat16), wide, s.table, s.lens)
