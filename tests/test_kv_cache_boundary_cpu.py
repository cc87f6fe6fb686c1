"""What the 8-bit key/value cache's entry points refuse, through the C ABI and through the binding, without a GPU: every call
below is refused on the host or only computes a size."""
import ctypes

import pytest
import torch


@pytest.fixture(scope="module")
def nb():
    from paper_2601_12150_amd import binding
    return binding


P = [ctypes.c_void_p(0x10000 * (i + 1)) for i in range(16)]


def good(nb, base=0x1000000, capacity=256, **kw):
    c = nb.ns_kv_cache(2, 4, 128, capacity, 64, nb.NS_CODE_I8, 4 * capacity * 128, capacity * 128, 128, base, base + 0x100000, base + 0x200000, base + 0x300000)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def desc(nb, **kw):
    d = nb.ns_kv_attn_desc(8, 3, nb.NS_BF16, 1, 0.1, 8 * 3 * 128, 3 * 128, 128, 8 * 3 * 128, 3 * 128, 128)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


BAD_CACHE = [("batch", 0, 1), ("heads_kv", 0, 1), ("head_dim", 0, 1), ("capacity", -64, 1), ("block", 0, 1), ("code", 2, 1), ("capacity", 250, 1),
             ("stride_t", 64, 1), ("stride_t", 136, 1), ("stride_h", -16, 1), ("stride_b", 8, 1), ("head_dim", 96, 2), ("block", 16, 2), ("block", 256, 2),
             ("batch", 65536, 2), ("heads_kv", 1025, 2), ("stride_t", (1 << 25) + 16, 2)]


def calls(nb):
    """name -> a call that takes a cache (and keyword arguments) and is in order but for them."""
    L = nb.lib
    ref = ctypes.byref

    def append(c, tokens=5, dtype=nb.NS_BF16, k=P[0], v=P[1], sb=4 * 5 * 128, sh=5 * 128, st=128, start=P[2], counts=None):
        return L.kv_cache_append(None if c is None else ref(c), tokens, dtype, k, v, sb, sh, st, start, counts, None)

    def read(c, lengths=P[0], first=0, tokens=10, dtype=nb.NS_F32, k=P[1], v=P[2]):
        return L.kv_cache_read(None if c is None else ref(c), lengths, first, tokens, dtype, k, v, None)

    def attn(c, d=None, q=P[0], lengths=P[1], counts=None, out=P[2], lse=None, w_in=None, w_out=None, ws=None, ws_bytes=0):
        return L.kv_cache_attn(None if c is None else ref(c), ref(desc(nb) if d is None else d), q, lengths, counts, out, lse, w_in, w_out, ws, ws_bytes, None)

    def evict(c, to=None, w=P[0], lengths=P[1], keep=100, n_global=1, n_recent=2, kept=P[2], w_out=P[3], left=P[4], ws=None, ws_bytes=0):
        return L.kv_cache_evict(None if c is None else ref(c), ref(good(nb, 0x5000000, 128) if to is None else to), w, lengths, keep, n_global, n_recent,
                                kept, w_out, left, ws, ws_bytes, None)

    return dict(append=append, read=read, attn=attn, evict=evict)


@pytest.mark.parametrize("name", ["append", "read", "attn", "evict"])
@pytest.mark.parametrize("field,value,code", BAD_CACHE)
def test_caches_are_checked(nb, name, field, value, code):
    assert calls(nb)[name](good(nb, **{field: value})) == code and nb.lib.ns_last_error()


@pytest.mark.parametrize("name", ["append", "read", "attn", "evict"])
def test_the_caches_memory_is_checked(nb, name):
    f = calls(nb)[name]
    assert f(None) == nb.NS_ERR_INVALID_ARG
    for field in ("k", "v", "k_scale", "v_scale"):
        assert f(good(nb, **{field: None})) == nb.NS_ERR_INVALID_ARG
    assert f(good(nb, k=0x1000008)) == nb.NS_ERR_INVALID_ARG and f(good(nb, v_scale=0x1000002)) == nb.NS_ERR_INVALID_ARG
    assert f(good(nb, v=0x1000000)) == nb.NS_ERR_INVALID_ARG                       # keys and values in one place
    assert f(good(nb, capacity=(1 << 30) + 64)) == nb.NS_ERR_UNSUPPORTED


def test_append_refusals(nb):
    f, c = calls(nb)["append"], good(nb)
    for kw in (dict(tokens=0), dict(dtype=7), dict(k=None), dict(v=ctypes.c_void_p(0x10008)), dict(start=None), dict(start=ctypes.c_void_p(0x10002)),
               dict(counts=ctypes.c_void_p(0x10001)), dict(st=127), dict(sh=4), dict(sb=-128), dict(k=ctypes.c_void_p(c.k)), dict(v=ctypes.c_void_p(c.k))):
        assert f(c, **kw) == nb.NS_ERR_INVALID_ARG, kw
    # sequences or heads that share rows are read, not written
    for kw in (dict(stride_b=0), dict(stride_h=0)):
        assert f(good(nb, **kw)) == nb.NS_ERR_INVALID_ARG, kw


def test_read_refusals(nb):
    f, c = calls(nb)["read"], good(nb)
    for kw in (dict(lengths=None), dict(first=-1), dict(tokens=0), dict(tokens=257), dict(first=250, tokens=7), dict(first=2 ** 31 - 1), dict(dtype=2),
               dict(k=None), dict(k=P[2]), dict(v=ctypes.c_void_p(c.k)), dict(v=ctypes.c_void_p(0x10004))):
        assert f(c, **kw) == nb.NS_ERR_INVALID_ARG, kw


def test_attention_refusals(nb):
    f, c = calls(nb)["attn"], good(nb)
    bad = [(dict(heads=0), 1), (dict(tokens=0), 1), (dict(heads=6), 1), (dict(dtype=5), 1), (dict(scale=float("nan")), 1), (dict(scale=float("inf")), 1),
           (dict(q_stride_t=64), 1), (dict(q_stride_h=1), 1), (dict(out_stride_b=-128), 1), (dict(out_stride_t=4), 1), (dict(out_stride_h=0), 1),
           (dict(out_stride_b=0), 1), (dict(heads=1028), 2), (dict(tokens=1 << 22), 2)]
    for kw, code in bad:
        d = desc(nb, **kw)
        assert f(c, d) == code, kw
        assert nb.lib.kv_cache_attn_workspace_bytes(ctypes.byref(c), ctypes.byref(d), 1) == 0
    for kw in (dict(q=None), dict(out=None), dict(lengths=None), dict(q=ctypes.c_void_p(0x10004)), dict(out=P[0]), dict(out=ctypes.c_void_p(c.k)),
               dict(w_in=P[5]), dict(lse=ctypes.c_void_p(0x10001)), dict(w_out=ctypes.c_void_p(0x10002))):
        assert f(c, **kw) == nb.NS_ERR_INVALID_ARG, kw
    need = nb.lib.kv_cache_attn_workspace_bytes(ctypes.byref(c), ctypes.byref(desc(nb)), 1)
    assert need > 0
    for kw in (dict(ws=None, ws_bytes=0), dict(ws=ctypes.c_void_p(0x10010), ws_bytes=need), dict(ws=P[6], ws_bytes=need - 1)):
        assert f(c, w_out=P[5], **kw) == nb.NS_ERR_WORKSPACE, kw


def test_evict_refusals(nb):
    f, c = calls(nb)["evict"], good(nb)
    other = dict(batch=3, heads_kv=2, head_dim=64, block=32, code=nb.NS_CODE_E4M3)
    for k, v in other.items():
        assert f(c, to=good(nb, 0x5000000, 128, **{k: v})) == nb.NS_ERR_INVALID_ARG, k
    same = good(nb, 0x5000000, 128)
    for kw in (dict(keep=0), dict(keep=257), dict(keep=129), dict(n_global=-1), dict(n_recent=-1), dict(n_global=99, n_recent=2), dict(n_global=2 ** 31 - 1, n_recent=5),
               dict(w=None), dict(kept=None), dict(w_out=None), dict(left=None), dict(w_out=P[0]), dict(left=P[1]), dict(kept=ctypes.c_void_p(0x10001)),
               dict(to=good(nb, 0x5000000, 128, k=c.k)), dict(to=good(nb, 0x5000000, 128, v=c.k)), dict(to=good(nb, 0x5000000, 128, v_scale=c.v_scale)),
               dict(to=good(nb, 0x5000000, 128, stride_h=0))):
        assert f(c, **{"to": same, **kw}) == nb.NS_ERR_INVALID_ARG, kw
    need = nb.lib.kv_cache_evict_workspace_bytes(ctypes.byref(good(nb, capacity=1 << 20)), 100)
    if need:
        assert f(good(nb, capacity=1 << 20, stride_h=1 << 27, stride_b=1 << 30)) == nb.NS_ERR_WORKSPACE
    assert nb.lib.kv_cache_evict_workspace_bytes(ctypes.byref(c), 0) == 0


def test_the_binding_checks_its_tensors(nb):
    """Wrong shapes, types and devices; the tensors lie in host memory, which is refused last."""
    B, H, N, D = 2, 2, 128, 64
    cache = nb.kv_cache_empty(B, H, N, D, 64, torch.int8, "cpu")
    f8 = nb.kv_cache_empty(B, H, N, D, 32, torch.float8_e4m3fn, "cpu")
    assert f8.k.dtype == torch.float8_e4m3fn and f8.k_scale.shape == (B, H, 4)
    x, q, n = torch.zeros((B, H, 3, D)), torch.zeros((B, 2 * H, 3, D)), torch.zeros(B, dtype=torch.int32)
    w = torch.zeros((B, H, N))
    with pytest.raises(ValueError):
        nb.kv_cache_empty(1, 1, 100, 64, 64, device="cpu")
    for bad in ((cache.k,), cache[:3], [*cache], (cache.k, cache.v, cache.k_scale, 3), None):
        with pytest.raises(TypeError):
            nb.kv_cache_append(bad, x, x, n)
    with pytest.raises(TypeError):
        nb.kv_cache_append(cache._replace(k=cache.k.float(), v=cache.v.float()), x, x, n)
    for bad in (cache._replace(k=cache.k[:, :, :64]), cache._replace(k=cache.k.transpose(2, 3), v=cache.v.transpose(2, 3)), cache._replace(v_scale=cache.v_scale[:1]),
                cache._replace(k_scale=cache.k_scale.double()), cache._replace(k_scale=torch.ones((B, H, 3)), v_scale=torch.ones((B, H, 3))),
                cache._replace(v=f8.v)):
        with pytest.raises(ValueError):
            nb.kv_cache_read(bad, n)
    for args in ((x[:, :1], x[:, :1], n), (x, x[:, :, :2], n), (x[..., :32], x[..., :32], n), (x, x.bfloat16(), n), (x, x, n.long()), (x, x, n[:1]),
                 (x, x, n, n.float())):
        with pytest.raises(ValueError):
            nb.kv_cache_append(cache, *args)
    with pytest.raises(TypeError):
        nb.kv_cache_append(cache, x.half(), x.half(), n)
    for args, kw in (((q[:1], n), {}), ((q[..., :32], n), {}), ((q, n[:1]), {}), ((q, n), dict(counts=n.long())), ((q, n), dict(weights=w[:, :, :64])),
                     ((q, n), dict(weights_out=w.double())), ((q, n), dict(out=q[:, :2])), ((q, n), dict(out=q.bfloat16()))):
        with pytest.raises(ValueError):
            nb.kv_cache_attn(cache, *args, **kw)
    to = nb.kv_cache_empty(B, H, 64, D, 64, torch.int8, "cpu")
    for args in ((w[:, :1], n, 10), (w, n.long(), 10), (w.double(), n, 10)):
        with pytest.raises(ValueError):
            nb.kv_cache_evict(cache, to, *args)
    with pytest.raises(ValueError):
        nb.kv_cache_evict(cache, to, w, n, 2 ** 40)
    with pytest.raises(TypeError):
        nb.kv_cache_read(cache, n, dtype=torch.float16)
    with pytest.raises(ValueError):
        nb.kv_cache_read(cache, n, k_out=torch.zeros((B, H, 3, D)))
    # all in order, but not on a GPU
    # before anything of such a size is allocated
    for args in ((-2 ** 31,), (-1, 5), (N,), (0, 2 ** 31 - 1), (0, 0), (5, N - 4)):
        with pytest.raises(ValueError, match="capacity"):
            nb.kv_cache_read(cache, n, *args)
    for keep in (0, -1, N + 1, 2 ** 31 - 1):
        with pytest.raises(ValueError, match="keep"):
            nb.kv_cache_evict(cache, to, w, n, keep)
    for f in (lambda: nb.kv_cache_append(cache, x, x, n), lambda: nb.kv_cache_read(cache, n), lambda: nb.kv_cache_attn(cache, q, n, want_weights=True),
              lambda: nb.kv_cache_evict(cache, to, w, n, 10)):
        with pytest.raises(ValueError, match="GPU"):
            f()
