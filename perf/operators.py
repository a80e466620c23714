"""Timed cases of the key-value cache: rows written into it (quantised or not), read back, and one new token of every sequence
attending to it.

Kinds of pass:
  write     : K and V of a packed stream of prompts go into their sequences' pages; cache of the rows' own type;
  roundtrip : the same into an 8-bit cache, and all rows read back (a prompt's K and V handed on as they are cached);
  read      : the rows of every sequence out of the cache, one packed stream;
  attend    : one query token of every sequence against its cached keys and values;
  step      : K and V of one new token of every sequence written, then attended to, what a layer does in a decoding step.

A case fixes the multiset of sequence lengths (drawn from its length law with its own `lengths_seed`), so that its work is known;
their order, the pages they own and every tensor come from the seed given to `prepare`.
"""
import math
import random

import torch

own = False  # run() makes the framework's calls instead of computing the plain form

DEV = "cuda:0"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
EIGHT_BITS = {"i8": (torch.int8, 127.0), "e4m3": (torch.float8_e4m3fn, 448.0)}  # element type, largest value

# ---- the cases --------------------------------------------------------------------------------------


def _case(kind, seqs, lens, hq, hkv, d, page, dtype, cache="same", lengths_seed=1, pad=0):
    """lens: "fixed L", "uniform lo hi" or "lognormal median sigma lo hi"; cache: "same", "i8" or "e4m3"; pad: tokens behind the
    last sequence of a written stream, which belong to none."""
    return {"kind": kind, "seqs": seqs, "lens": lens, "hq": hq, "hkv": hkv, "d": d, "page": page, "dtype": dtype, "cache": cache,
            "lengths_seed": lengths_seed, "pad": pad}


def listed():
    cases = {
        # the smallest call: one sequence that has just begun, a small layer; latency and launches
        "attend_1x37": _case("attend", 1, "fixed 37", 8, 2, 64, 16, "bf16"),
        # one sequence with a long document behind it: the whole chip has to share it
        "attend_1x131072": _case("attend", 1, "fixed 131072", 32, 8, 128, 64, "bf16"),
        # a batch being served: prompts of very different lengths, small pages
        "attend_64_ragged": _case("attend", 64, "lognormal 2048 1.0 1 16384", 32, 8, 128, 16, "bf16"),
        # a large batch on an 8-bit cache: the largest attention
        "attend_e4m3_128": _case("attend", 128, "uniform 1024 8192", 40, 8, 128, 64, "bf16", "e4m3"),
        # fp16, one KV head for all query heads, pages of one token, some sequences still empty, 8-bit integers
        "attend_i8_mqa_33": _case("attend", 33, "uniform 0 3001", 16, 1, 64, 1, "f16", "i8"),
        # every head its own keys, head dim 256
        "attend_d256_16": _case("attend", 16, "uniform 500 4000", 16, 16, 256, 32, "bf16"),
        # a layer re-run in fp32 to check a 16-bit model's numbers: odd head dim, odd pages
        "attend_fp32_3": _case("attend", 3, "uniform 1 1000", 8, 2, 60, 24, "f32"),
        # a decoding step of 48 sequences: new rows written, then attended to
        "step_48": _case("step", 48, "lognormal 700 0.8 1 4096", 32, 8, 128, 16, "bf16"),
        # the same with an 8-bit cache, no power of two in sight; the new rows also come back as they are cached
        "step_i8_20": _case("step", 20, "uniform 1 2500", 36, 4, 80, 48, "f16", "i8"),
        # prompts of a packed row into their pages, with the row's padding behind them
        "write_16384": _case("write", 24, "lognormal 512 0.8 32 4096", 32, 8, 128, 16, "bf16", pad=37),
        # as many KV heads as query heads, quantised on the way in, read back: the largest write and read
        "roundtrip_i8_65536": _case("roundtrip", 32, "fixed 2048", 32, 32, 128, 64, "bf16", "i8"),
        # cached 8-bit floats of a few prompts handed on as fp16
        "read_e4m3_9": _case("read", 9, "uniform 1 2000", 24, 8, 96, 32, "f16", "e4m3"),
    }
    return [{"name": name, **case} for name, case in cases.items()]


# head layouts (query heads, KV heads, head_dim) of decoder layers with a few billion parameters
HEADS = [(32, 32, 128), (32, 8, 128), (40, 8, 128), (36, 4, 128), (32, 32, 64), (16, 1, 64), (32, 32, 80), (24, 8, 96), (16, 16, 256)]
PAGES = [1, 8, 16, 16, 24, 32, 48, 64, 128, 256]
LARGEST = 128 * 8192 * 8 * 128  # cached elements of K, all sequences as long as the longest


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = {c["name"]: work(c)["bytes"] for c in listed()}
    while True:
        kind = rng.choice(["attend", "attend", "attend", "step", "step", "write", "roundtrip", "read"])
        hq, hkv, d = rng.choice(HEADS)
        dtype, cache = rng.choice(["bf16", "bf16", "f16"]), rng.choice(["same", "i8", "e4m3"])
        if rng.random() < 0.15:  # a check in fp32: small layers, head dims that nothing divides
            heads, dtype, d = rng.choice([2, 4, 8]), "f32", rng.choice([16, 20, 33, 60, 64, 100])
            hq, hkv = heads, heads // rng.choice([1, 2])
        if kind == "write":
            cache = "same"
        elif kind == "roundtrip" and cache == "same":
            continue
        seqs, longest = _log_uniform(rng, 1, 256), _log_uniform(rng, 32, 131072)
        least = 0 if kind == "attend" else 1
        lens = rng.choice(["fixed %d" % longest, "uniform %d %d" % (least, longest),
                           "lognormal %d 1.0 %d %d" % (max(1, longest // 8), least, longest)])
        pad = rng.choice([0, 0, 1, 63]) if kind in ("write", "roundtrip") else 0
        c = _case(kind, seqs, lens, hq, hkv, d, rng.choice(PAGES), dtype, cache, rng.randrange(1, 1 << 20), pad)
        if kind in ("attend", "step"):
            fits = seqs * longest * hkv * d <= LARGEST and work(c)["bytes"] <= most["attend_e4m3_128"]
        else:
            fits = seqs * longest <= 1 << 20 and work(c)["bytes"] <= most["roundtrip_i8_65536"]
        if fits and longest // c["page"] <= 1 << 15:
            return c


# ---- inputs -----------------------------------------------------------------------------------------


def lengths(case):
    """Cached tokens of every sequence, those that this pass writes included, in the order they were drawn."""
    law, *args = case["lens"].split()
    args = [float(a) for a in args]
    rng = random.Random(case["lengths_seed"])
    if law == "fixed":
        return [int(args[0])] * case["seqs"]
    if law == "uniform":
        return [rng.randint(int(args[0]), int(args[1])) for _ in range(case["seqs"])]
    median, sigma, lo, hi = args
    return [int(min(hi, max(lo, rng.lognormvariate(math.log(median), sigma)))) for _ in range(case["seqs"])]


def _quantised(x, kind):
    """Rows of x [..., d] (float32) in 8 bits, and their scales [...]."""
    dtype, top = EIGHT_BITS[kind]
    amax = x.abs().amax(-1)
    q = x * top / torch.where(amax > 0, amax, 1.0)[..., None]
    return (q.round() if kind == "i8" else q).to(dtype), amax / top


def prepare(case, seed):
    lens = lengths(case)
    random.Random(seed).shuffle(lens)
    gen = torch.Generator(device=DEV).manual_seed(seed)
    dt, page, hkv, d = DTYPES[case["dtype"]], case["page"], case["hkv"], case["d"]
    normal = lambda *shape: torch.randn(shape, generator=gen, device=DEV, dtype=torch.float32).to(dt)  # noqa: E731
    pages = [-(-n // page) for n in lens]
    n_pages, width = sum(pages) + 3, max(max(pages), 1) + 2   # some pages are nobody's, some of the table's columns unused
    free = torch.randperm(n_pages, generator=gen, device=DEV)[:sum(pages)].to(torch.int32)
    of, used = torch.tensor(pages, device=DEV), torch.arange(width, device=DEV)
    table = torch.full((len(lens), width), -1, dtype=torch.int32, device=DEV)
    table[used < of[:, None]] = free
    state = {"case": case, "table": table, "lens": torch.tensor(lens, dtype=torch.int32, device=DEV)}
    k, v, scales = normal(n_pages, hkv, page, d), normal(n_pages, hkv, page, d), (None, None)
    if case["cache"] != "same":
        (k, ks), (v, vs) = _quantised(k.float(), case["cache"]), _quantised(v.float(), case["cache"])
        scales = (ks, vs)
    state["cache"] = (k, v, *scales)
    kind = case["kind"]
    if kind in ("attend", "step"):
        state["q"] = normal(len(lens), case["hq"], d)
    if kind == "step":
        state["positions"], state["seq_ids"] = state["lens"].long() - 1, None
    elif kind != "attend":  # a packed stream: example after example, then the padding as one more
        each = torch.tensor(lens + [case["pad"]], device=DEV)
        start = each.cumsum(0) - each
        seq = torch.repeat_interleave(torch.arange(len(lens) + 1, device=DEV), each)
        state["positions"], state["seq_ids"] = torch.arange(len(seq), device=DEV) - start[seq], seq.to(torch.int32)
    if kind in ("write", "roundtrip", "step"):
        state["k"], state["v"] = normal(len(state["positions"]), hkv, d), normal(len(state["positions"]), hkv, d)
    return state


# ---- one pass ---------------------------------------------------------------------------------------


def run(state):
    case, cache, table = state["case"], state["cache"], state["table"]
    kind, same = case["kind"], case["cache"] == "same"
    write, read, attend = _calls() if own else (_write, _read, _attend)
    out = {}
    if kind in ("write", "roundtrip", "step"):
        write(state["k"], state["v"], cache, table, state["positions"], state["seq_ids"])
    if kind in ("attend", "step"):
        out["o"], out["lse"] = attend(state["q"], cache, table, state["lens"])
    if kind != "attend" and same and kind != "read":
        out["k"], out["v"] = cache[:2]   # the pages themselves, whole
    elif kind != "attend":
        out["k"], out["v"] = read(cache, table, state["positions"], state["seq_ids"], DTYPES[case["dtype"]])
    if kind == "roundtrip":
        out["k_scale"], out["v_scale"] = cache[2:]
    return out


def _calls():
    from paper_2407_09105_amd import binding
    return binding.paged_cache_write, binding.paged_cache_read, binding.paged_attn_fwd


def _places(cache, table, positions, seq_ids):
    """(token has a place, its page, its row there)"""
    page = cache[0].shape[2]
    seq = torch.arange(len(positions), device=DEV) if seq_ids is None else seq_ids.long()
    ok = (seq < table.shape[0]) & (positions < table.shape[1] * page)
    at = table[torch.where(ok, seq, 0), torch.where(ok, positions // page, 0)].long()
    return ok & (at >= 0), at, positions % page


def _write(k, v, cache, table, positions, seq_ids):
    ok, at, row = _places(cache, table, positions, seq_ids)
    t = torch.where(ok, torch.arange(len(ok), device=DEV), 0)   # the padding writes the first token, which has a place, once more
    at, row, k, v = at[t], row[t], k[t], v[t]
    if cache[2] is None:
        cache[0][at, :, row], cache[1][at, :, row] = k, v
        return
    kind = "i8" if cache[0].dtype == torch.int8 else "e4m3"
    (qk, ks), (qv, vs) = _quantised(k.float(), kind), _quantised(v.float(), kind)
    cache[0].view(torch.int8)[at, :, row], cache[1].view(torch.int8)[at, :, row] = qk.view(torch.int8), qv.view(torch.int8)
    cache[2][at, :, row], cache[3][at, :, row] = ks, vs


def _rows(x, scale, at, row):
    y = x.view(torch.int8)[at, :, row].view(x.dtype).float() if scale is not None else x[at, :, row].float()
    return y if scale is None else y * scale[at, :, row][..., None]


def _read(cache, table, positions, seq_ids, dtype):
    ok, at, row = _places(cache, table, positions, seq_ids)
    at = torch.where(ok, at, 0)
    there = ok[:, None, None]
    return (torch.where(there, _rows(cache[0], cache[2], at, row), 0.0).to(dtype),
            torch.where(there, _rows(cache[1], cache[3], at, row), 0.0).to(dtype))


def _context(x, scale, table):
    """[B, Hkv, width * page, d] in float32: every row that the table names."""
    at = table.clamp(min=0).long()
    y = x.view(torch.int8)[at].view(x.dtype).float() if scale is not None else x[at].float()   # [B, width, Hkv, page, d]
    if scale is not None:
        y *= scale[at][..., None]
    return y.transpose(1, 2).reshape(y.shape[0], y.shape[2], -1, y.shape[-1])


def _attend(q, cache, table, lens):
    B, hq, d = q.shape
    hkv, page = cache[0].shape[1:3]
    k, v = _context(cache[0], cache[2], table), _context(cache[1], cache[3], table)
    s = q.float().view(B, hkv, hq // hkv, d) @ k.transpose(2, 3) / math.sqrt(d)
    there = (torch.arange(k.shape[2], device=DEV) < lens[:, None]) & (table >= 0).repeat_interleave(page, 1)
    s = s.masked_fill(~there[:, None, None], -math.inf)
    m = s.amax(-1, keepdim=True)
    p = torch.exp(s - torch.where(m == -math.inf, 0.0, m))
    l = p.sum(-1, keepdim=True)
    o = p @ v / torch.where(l == 0, 1.0, l)
    return o.view(B, hq, d).to(q.dtype), (m + torch.log(l)).view(B, hq).t().contiguous()


# ---- what a pass cannot do without, and what is right -------------------------------------------------


def work(case):
    """Bytes: every cached row of a sequence and every given row read or written once, with scales, ids and the table's used entries.
    Flops: 4 d for each pair of a query head and a cached token; 8-bit conversions are not counted."""
    lens, hq, hkv, d, kind = lengths(case), case["hq"], case["hkv"], case["d"], case["kind"]
    e = 4 if case["dtype"] == "f32" else 2
    cached = 2 * hkv * (d * e if case["cache"] == "same" else d + 4)   # of one token, K and V
    plain = 2 * hkv * d * e
    total, seqs = sum(lens), len(lens)
    table = 4 * sum(-(-n // case["page"]) for n in lens)
    attend = {"bytes": total * cached + table + seqs * (4 + hq * (2 * d * e + 4)), "flops": 4 * d * hq * total}
    moved = {"write": total * (cached + plain + 12), "read": total * (cached + plain + 12), "roundtrip": 2 * total * (cached + plain + 12)}
    if kind == "attend":
        return attend
    if kind == "step":
        back = 0 if case["cache"] == "same" else seqs * (cached + plain)
        return {"bytes": attend["bytes"] + seqs * (cached + plain + 8) + back, "flops": attend["flops"]}
    return {"bytes": moved[kind] + table, "flops": 0}


def _in_64(x, scale):
    y = x.double()
    return y if scale is None else y * scale.double()[..., None]


def _quantised_in_64(x, kind):
    """(value that each element is stored as, scale) of rows x in float64."""
    top = EIGHT_BITS[kind][1]
    amax = x.abs().amax(-1, keepdim=True)
    scale = amax / top
    t = torch.where(amax > 0, x * top / amax, 0.0)  # exact where it lies halfway between two steps
    if kind == "e4m3":  # four significant bits, steps of 2^-9 at least
        step = torch.exp2(torch.floor(torch.log2(t.abs().clamp(min=2.0 ** -6))) - 3)
        return torch.round(t / step) * step * scale, scale[..., 0]
    return torch.round(t) * scale, scale[..., 0]


def exact(case, seed):
    state = prepare(case, seed)
    kind, table, lens = case["kind"], state["table"], state["lens"].tolist()
    eight = case["cache"] != "same"
    k, v, ks, vs = state["cache"]
    page, out = case["page"], {}
    K, V = (_in_64(k, ks), _in_64(v, vs)) if kind != "roundtrip" else (torch.zeros(k.shape, dtype=torch.float64, device=DEV) for _ in "kv")
    scales = {"k_scale": ks, "v_scale": vs}
    if "k" in state:
        seq = state["seq_ids"] if state["seq_ids"] is not None else torch.arange(len(lens), device=DEV)
        n = int((seq < len(lens)).sum())        # the padding comes last
        pos = state["positions"][:n]
        at, row = table[seq[:n].long(), pos // page].long(), pos % page
        for name, to in (("k", K), ("v", V)):
            x = state[name][:n].double()
            if eight:
                x, s = _quantised_in_64(x, case["cache"])
                if kind == "roundtrip":
                    scales[name + "_scale"] = scales[name + "_scale"].double()
                    scales[name + "_scale"][at, :, row] = s
            to[at, :, row] = x
    if kind in ("attend", "step"):
        B, hq, d = state["q"].shape
        hkv = case["hkv"]
        o = torch.zeros((B, hq, d), dtype=torch.float64, device=DEV)
        lse = torch.full((hq, B), -math.inf, dtype=torch.float64, device=DEV)
        for b, n in enumerate(lens):
            if n:
                mine = table[b, :-(-n // page)].long()
                kb = K[mine].transpose(0, 1).reshape(hkv, -1, d)[:, :n].contiguous()
                vb = V[mine].transpose(0, 1).reshape(hkv, -1, d)[:, :n].contiguous()
                s = (kb @ state["q"][b].double().view(hkv, -1, d).transpose(1, 2).contiguous()).transpose(1, 2).contiguous() / math.sqrt(d)
                lse[:, b] = torch.logsumexp(s, -1).view(-1)
                o[b] = (torch.softmax(s, -1) @ vb).view(hq, d)
        out["o"], out["lse"] = o, lse
    if kind in ("write", "step") and not eight:
        out["k"], out["v"] = K, V
    elif kind != "attend":
        seq = state["seq_ids"] if state["seq_ids"] is not None else torch.arange(len(lens), device=DEV)
        there = seq < len(lens)
        at = table[torch.where(there, seq, 0).long(), torch.where(there, state["positions"] // page, 0)].long()
        for name, x in (("k", K), ("v", V)):
            out[name] = x[at, :, state["positions"] % page] * there[:, None, None]
    if kind == "roundtrip":
        out.update(scales)
    return out
