"""The key-value cache's entry points refuse on the host what they cannot run (nothing is launched by any call in this file)."""
import ctypes as C
import os

import pytest
import torch

from paper_2407_09105_amd import binding


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(binding.LIB_PATH):
        pytest.skip("library is not built")
    return binding.lib()


P = 0x10000  # never dereferenced: every call with it fails validation or has nothing to do


def _cache(**kw):
    c = binding.VaKvCache(P, P, P, P, 10, 16, 2, 64, binding.CACHE_PLAIN, 3, 4, 4, P)
    for name, value in kw.items():
        setattr(c, name, value)
    return c


BAD_CACHES = [
    (2, dict(n_pages=0)), (2, dict(page_size=0)), (2, dict(hkv=-1)), (2, dict(d=0)), (2, dict(n_seqs=-1)), (2, dict(max_pages=-1)),
    (2, dict(table_stride=3)), (2, dict(table_stride=-4)), (2, dict(n_pages=1 << 26)), (2, dict(n_pages=2 ** 31 - 1, hkv=65535)),
    (2, dict(max_pages=1 << 27, table_stride=1 << 27)), (2, dict(max_pages=2 ** 31 - 1023, page_size=1, table_stride=1 << 31)), (2, dict(page_size=1 << 20)), (3, dict(d=257)), (3, dict(format=3)), (3, dict(n_seqs=65536)),
    (3, dict(hkv=65536)), (1, dict(k=None)), (1, dict(v=None)), (1, dict(page_table=None)),
    (1, dict(format=binding.CACHE_I8, k_scale=None)), (1, dict(format=binding.CACHE_E4M3, v_scale=None))]


@pytest.mark.parametrize("status,change", BAD_CACHES)
def test_caches_that_are_refused(L, status, change):
    c = C.byref(_cache(**change))
    for f in (L.va_cache_write, L.va_cache_read):
        assert f(P, P, binding.VA_BF16, c, P, P, binding.VA_I32, 8, None) == status
    assert L.va_paged_attn_fwd(P, P, P, binding.VA_BF16, c, 65535 if change.get("hkv") == 65536 else 4, P, 0.0, P, 1 << 40, None) == status


def test_row_arguments(L):
    for f in (L.va_cache_write, L.va_cache_read):
        ok = [P, P, binding.VA_BF16, C.byref(_cache()), P, P, binding.VA_I32, 8, None]

        def with_(i, value):
            return f(*ok[:i], value, *ok[i + 1:])

        assert with_(0, None) == with_(1, None) == with_(3, None) == with_(5, None) == 1
        assert with_(2, 9) == with_(6, 9) == 3 and with_(7, -1) == 2
        assert with_(7, 0) == 0                     # nothing to do


def test_attention_arguments(L):
    f = L.va_paged_attn_fwd
    ok = [P, P, P, binding.VA_BF16, C.byref(_cache()), 4, P, 0.0, P, 1 << 40, None]

    def with_(i, value):
        return f(*ok[:i], value, *ok[i + 1:])

    assert with_(0, None) == with_(1, None) == with_(2, None) == with_(4, None) == with_(6, None) == 1
    assert with_(3, 7) == 3 and with_(5, 3) == 2 and with_(5, 0) == 2 and with_(5, 65536) == 3
    assert with_(4, C.byref(_cache(n_seqs=0))) == 0
    assert with_(4, C.byref(_cache(n_pages=1, hkv=129, n_seqs=65535))) == 2              # 4 heads of 129
    assert f(*ok[:4], C.byref(_cache(n_pages=1, hkv=129, n_seqs=65535)), 129, *ok[6:]) == 3   # too many workgroups
    # one long sequence: shared by many workgroups, which need room
    long = _cache(n_pages=10000, n_seqs=1, max_pages=10000, table_stride=10000)
    need = L.va_paged_attn_workspace_bytes(1, 10000, 16, 4, 2, 64)
    assert need > 0 and need % 256 == 0
    ok[4] = C.byref(long)
    assert with_(9, need - 1) == 4 and with_(8, None) == 1 and with_(8, P + 4) == 4


def test_workspace_sizes(L):
    f = L.va_paged_attn_workspace_bytes
    assert f(0, 4, 16, 4, 2, 64) == f(3, 0, 16, 4, 2, 64) == f(3, 4, 16, 4, 2, 0) == f(3, 4, -1, 4, 2, 64) == 0
    assert f(5, 4, 16, 4, 2, 64) == 0                                # short contexts are not cut
    assert f(5, 1000, 16, 1, 2, 64) == f(5, 1000, 16, 3, 2, 64) == 0  # refused calls need none
    assert f(2 ** 31 - 1, 2 ** 31 - 1, 2 ** 31 - 1, 4, 2, 64) == f(5, 1 << 20, 1 << 20, 4, 2, 64) == 0
    assert f(65535, 1 << 10, 1 << 10, 64, 8, 128) < 8 << 30          # and none takes the card's memory


@pytest.mark.filterwarnings("ignore:Accessing the data pointer")
def test_python_refusals(L, monkeypatch):
    """Tensors without memory behind them: a call that passes the binding's checks ends at the library's, which refuses null
    pointers."""
    from torch._subclasses.fake_tensor import FakeTensorMode
    monkeypatch.setattr(binding, "_stream", lambda: 0)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    with FakeTensorMode():
        of = lambda *shape, dtype=torch.bfloat16, device="cuda:0": torch.empty(shape, device=device, dtype=dtype)  # noqa: E731
        cache = (of(10, 2, 16, 64), of(10, 2, 16, 64), None, None)
        i8 = (of(10, 2, 16, 64, dtype=torch.int8), of(10, 2, 16, 64, dtype=torch.int8), of(10, 2, 16, dtype=torch.float32),
              of(10, 2, 16, dtype=torch.float32))
        table, lens, q = of(3, 4, dtype=torch.int32), of(3, dtype=torch.int32), of(3, 4, 64)
        k, pos, seq = of(8, 2, 64), of(8, dtype=torch.int64), of(8, dtype=torch.int32)

        def write(k=k, v=None, cache=cache, table=table, pos=pos, seq=seq):
            binding.paged_cache_write(k, k if v is None else v, cache, table, pos, seq)

        def read(cache=cache, table=table, pos=pos, seq=seq, **kw):
            binding.paged_cache_read(cache, table, pos, seq, **kw)

        def attend(q=q, cache=cache, table=table, lens=lens, **kw):
            binding.paged_attn_fwd(q, cache, table, lens, **kw)

        for call in (write, read, attend):
            for good in (cache, i8):
                with pytest.raises(binding.VarlenAttnError, match="null pointer"):
                    call(cache=good)
            bad = [cache[:2] + (None,), (cache[0], of(10, 2, 16, 32), None, None), (of(10, 2, 64), of(10, 2, 64), None, None),
                   (cache[0].transpose(1, 2), cache[1].transpose(1, 2), None, None), i8[:2] + (None, None),
                   i8[:3] + (of(10, 2, 15, dtype=torch.float32),), i8[:3] + (of(10, 2, 16),)]
            for c in bad:
                with pytest.raises(ValueError):
                    call(cache=c)
            for dtype in (torch.float64, torch.uint8):
                with pytest.raises(TypeError):
                    call(cache=(of(10, 2, 16, 64, dtype=dtype), of(10, 2, 16, 64, dtype=dtype), None, None))
            for t in (of(3, 4, dtype=torch.int64), of(12, dtype=torch.int32), of(4, 3, dtype=torch.int32).t(),
                      of(1, 4, dtype=torch.int32).expand(3, 4), of(3, 4, dtype=torch.int32, device="cpu")):
                with pytest.raises(ValueError):
                    call(table=t)
            with pytest.raises(ValueError, match="current device"):
                call(table=of(3, 4, dtype=torch.int32, device="cuda:1"))
            with pytest.raises(binding.VarlenAttnError, match="null pointer"):
                call(table=of(3, 9, dtype=torch.int32)[:, 2:6])    # a part of a wider table will do
        with pytest.raises(TypeError):
            write(cache=(of(10, 2, 16, 64, dtype=torch.float16), of(10, 2, 16, 64, dtype=torch.float16), None, None))
        with pytest.raises(TypeError):
            attend(q=of(3, 4, 64, dtype=torch.float16))
        with pytest.raises(TypeError):
            read(dtype=torch.float16)
        with pytest.raises(TypeError):
            read(cache=i8, dtype=torch.int8)
        for kw in (dict(v=of(7, 2, 64)), dict(v=of(8, 2, 64, dtype=torch.float16)), dict(k=of(8, 3, 64)), dict(k=of(8, 128)),
                   dict(k=of(8, 64, 2).transpose(1, 2)), dict(pos=of(7, dtype=torch.int64)), dict(pos=of(8, dtype=torch.int16)),
                   dict(seq=of(8, dtype=torch.int64)), dict(seq=of(9, dtype=torch.int32)), dict(pos=of(8, dtype=torch.int64, device="cpu")),
                   dict(seq=of(8, dtype=torch.int32, device="cuda:1"))):
            with pytest.raises(ValueError):
                write(**kw)
        for kw in (dict(q=of(2, 4, 64)), dict(q=of(3, 5, 64)), dict(q=of(3, 4, 32)), dict(q=of(3, 256)), dict(q=of(3, 64, 4).transpose(1, 2)),
                   dict(lens=of(2, dtype=torch.int32)), dict(lens=of(3, 1, dtype=torch.int32)), dict(out=of(3, 4, 32)),
                   dict(lse=of(3, 4, dtype=torch.float32)), dict(lse=of(4, 3)), dict(workspace=of(8))):
            with pytest.raises(ValueError):
                attend(**kw)
        with pytest.raises(TypeError):
            attend(lens=of(3, dtype=torch.int64))
        with pytest.raises(ValueError):
            read(out=(of(8, 2, 64), of(7, 2, 64)))
        with pytest.raises(TypeError):
            read(out=(of(8, 2, 64), of(8, 2, 64)), dtype=torch.float32)


def test_paged_cache_on_the_cpu_is_refused(L):
    cache = binding.paged_cache(4, 16, 2, 64, torch.int8, "cpu")
    assert cache.k.dtype == torch.int8 and cache.k.shape == (4, 2, 16, 64) and cache.v_scale.shape == (4, 2, 16)
    assert binding.paged_cache(4, 16, 2, 64, torch.bfloat16, "cpu").k_scale is None
    with pytest.raises(TypeError):
        binding.paged_cache(4, 16, 2, 64, torch.float64, "cpu")
    with pytest.raises(ValueError, match="GPU"):
        binding.paged_attn_fwd(torch.zeros(1, 2, 64), cache, torch.zeros(1, 1, dtype=torch.int32), torch.ones(1, dtype=torch.int32))


def test_sizes_past_32_bits_are_refused(L, monkeypatch):
    """(ctypes would pass on their lower halves)"""
    from torch._subclasses.fake_tensor import FakeTensorMode
    monkeypatch.setattr(binding, "_stream", lambda: 0)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    with FakeTensorMode():
        of = lambda *shape, dtype=torch.bfloat16: torch.empty(shape, device="cuda:0", dtype=dtype)  # noqa: E731
        for many in (2 ** 31, 2 ** 32 + 1):
            table, pos = of(3, 4, dtype=torch.int32), of(8, dtype=torch.int64)
            for pages in ((many, 1, 1, 1), (1, many, 1, 1), (1, 1, many, 1), (1, 1, 1, many)):
                cache = (of(*pages), of(*pages), None, None)
                with pytest.raises(ValueError, match="32 bits"):
                    binding.paged_attn_fwd(of(3, pages[1], pages[3]), cache, table, of(3, dtype=torch.int32))
                with pytest.raises(ValueError, match="32 bits"):
                    binding.paged_cache_read(cache, table, pos)
            cache = (of(10, 1, 16, 1), of(10, 1, 16, 1), None, None)
            for table in (of(3, many, dtype=torch.int32), of(many, 4, dtype=torch.int32)):
                with pytest.raises(ValueError, match="32 bits"):
                    binding.paged_cache_read(cache, table, pos)
            with pytest.raises(ValueError, match="more tokens"):
                binding.paged_cache_write(of(many, 1, 1), of(many, 1, 1), cache, of(3, 4, dtype=torch.int32), of(many, dtype=torch.int64))
            with pytest.raises(ValueError, match="more tokens"):
                binding.paged_cache_read(cache, of(3, 4, dtype=torch.int32), of(many, dtype=torch.int64))
