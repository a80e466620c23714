"""Plain implementations in 64 bits of the key-value cache's operators, and inputs for their tests."""
import torch

from paper_2407_09105_amd import binding

DEV = "cuda:0"
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
CACHES = {"i8": torch.int8, "e4m3": torch.float8_e4m3fn}
TOPS = {"i8": 127, "e4m3": 448}


def cache_dtype(dtype, cache):
    return DTYPES[dtype] if cache == "plain" else CACHES[cache]


def quantise64(x, cache):
    """Rows x [..., d] (float64) -> (whole steps or e4m3 values as float64, scale float64 [...])."""
    top = TOPS[cache]
    amax = x.abs().amax(-1, keepdim=True)
    t = torch.where(amax > 0, x * top / torch.where(amax > 0, amax, 1.0), 0.0)
    if cache == "i8":
        return torch.round(t), (amax / top)[..., 0]
    step = torch.exp2(torch.floor(torch.log2(t.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(t / step) * step, (amax / top)[..., 0]


def place(table, page, n_pages, seq, pos):
    """(page, row) of a token in Python integers, or None."""
    if not 0 <= seq < table.shape[0] or not 0 <= pos < table.shape[1] * page:
        return None
    at = int(table[seq, pos // page])
    return (at, pos % page) if 0 <= at < n_pages else None


def values64(pages, scale):
    """What the elements of k or v stand for, float64 on the CPU."""
    y = pages.cpu().float().double()
    return y if scale is None else y * scale.cpu().double()[..., None]


def attend64(q, cache, table, lens, scale=None):
    """(O, LSE, sum_j p_j |v_j|, sum_j of the products' magnitudes at the worst key) of paged attention, float64 on the CPU."""
    q, table, lens = q.cpu().double(), table.cpu(), lens.cpu()
    K, V = values64(cache[0], cache[2]), values64(cache[1], cache[3])
    n_pages, hkv, page, d = K.shape
    B, hq, _ = q.shape
    G, scale = hq // hkv, d ** -0.5 if scale is None else scale
    O, A = torch.zeros(B, hq, d, dtype=torch.float64), torch.zeros(B, hq, d, dtype=torch.float64)
    LSE, worst = torch.full((hq, B), -float("inf"), dtype=torch.float64), torch.zeros(B, hq, dtype=torch.float64)
    for b in range(B):
        at = [place(table, page, n_pages, b, j) for j in range(min(int(lens[b]), table.shape[1] * page))]
        at = [a for a in at if a is not None]
        if not at:
            continue
        p, r = torch.tensor([a[0] for a in at]), torch.tensor([a[1] for a in at])
        for h in range(hq):
            k, v = K[p, h // G, r], V[p, h // G, r]
            s = (k @ q[b, h]) * scale
            w = torch.softmax(s, 0)
            O[b, h], A[b, h], LSE[h, b] = w @ v, w @ v.abs(), torch.logsumexp(s, 0)
            worst[b, h] = ((k.abs() @ q[b, h].abs()) * scale).max()
    return O, LSE, A, worst


def check_attention(o, lse, ref, dtype, n):
    """Scores: d products and sums in fp32, off by at most d 2^-24 of the products' magnitudes (and the 8-bit scale's product by
    2^-24).  P: that, twice (its own and the sum's), and 2^-20 for exponentials; for 16-bit operands P goes through the matrix units
    in two parts, 2^-16 of itself off.  Sums over n keys in fp32: chains of n / 128 + 64 additions.  O is rounded once."""
    O, LSE, A, worst = ref
    d = O.shape[-1]
    t = DTYPES[dtype]
    ds = (d + 4) * 2.0 ** -24 * worst
    rel = 2 * ds + 2.0 ** -20 + (n / 128 + 64) * 2.0 ** -24 + (0 if dtype == "f32" else 2.0 ** -15)
    tol = torch.finfo(t).eps / 2 * O.abs() + A * rel[..., None] + torch.finfo(t).tiny
    err = (o.cpu().double() - O).abs()
    assert not torch.isnan(err).any()
    assert (err <= tol).all(), (float((err - tol).max()), float((err / tol).max()))
    # the same error of a score, rounding of the sum's logarithm and of the result
    empty = LSE == -float("inf")
    got = lse.cpu().double()
    assert torch.equal(got == -float("inf"), empty)
    ltol = (ds + 2.0 ** -20 + (n / 128 + 64) * 2.0 ** -24).t() + 2.0 ** -22 * LSE.abs()
    assert ((got - LSE).abs()[~empty] <= ltol[~empty]).all()


class Setup:
    """Sequences of the given lengths, in pages dealt at random out of a cache with some to spare, rows N(0, 1) everywhere."""

    def __init__(self, dtype, cache, hq, hkv, d, page, lens, seed=0, spare=2, width=None, garbage=True):
        g = torch.Generator().manual_seed(seed)
        self.page, self.d, self.dtype = page, d, dtype
        counts = [-(-n // page) for n in lens]
        n_pages = sum(counts) + spare
        order = torch.randperm(n_pages, generator=g).to(torch.int32)
        self.table = torch.full((len(lens), width or max(counts + [1]) + 1), -1, dtype=torch.int32)
        at = 0
        for b, c in enumerate(counts):
            self.table[b, :c] = order[at:at + c]
            at += c
        self.lens = torch.tensor(lens, dtype=torch.int32)
        rnd = lambda *s: torch.randn(s, generator=g, dtype=torch.float64).to(DTYPES[dtype])  # noqa: E731
        self.q = rnd(len(lens), hq, d).to(DEV)
        k, v, ks, vs = rnd(n_pages, hkv, page, d), rnd(n_pages, hkv, page, d), None, None
        if cache != "plain":
            (k, ks), (v, vs) = quantise64(k.double(), cache), quantise64(v.double(), cache)
            k, v, ks, vs = k.float().to(CACHES[cache]), v.float().to(CACHES[cache]), ks.float(), vs.float()
        if garbage:  # what lies behind the sequences, and in pages that are nobody's, holds NaN
            used = torch.zeros(n_pages, page, dtype=torch.bool)
            for b, n in enumerate(lens):
                for j in range(n):
                    used[self.table[b, j // page], j % page] = True
            dead = (~used)[:, None, :].expand(n_pages, hkv, page)
            for x in (k, v):
                if cache == "e4m3":
                    x.view(torch.uint8)[dead] = 0x7f
                elif cache == "i8":
                    x[dead] = -128
                else:
                    x[dead] = float("nan")
            for x in (ks, vs):
                if x is not None:
                    x[dead] = float("nan")
        self.cache = tuple(None if x is None else x.to(DEV) for x in (k, v, ks, vs))
        self.table, self.lens = self.table.to(DEV), self.lens.to(DEV)

    def attend(self, scale=0.0, **kw):
        return binding.paged_attn_fwd(self.q, self.cache, self.table, self.lens, scale, **kw)

    def check(self, scale=None):
        o, lse = self.attend(scale or 0.0)
        check_attention(o, lse, attend64(self.q, self.cache, self.table, self.lens, scale), self.dtype, max(int(self.lens.max()), 1))
        return o, lse
