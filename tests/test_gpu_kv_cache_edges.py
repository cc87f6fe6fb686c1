"""The 8-bit key/value cache at the edges of what its entry points take, against the float64 oracle: logits far below zero, scales of 0,
scales between whose roundings there is next to nothing.  Attention's tolerances are those of test_gpu_kv_cache.py, where they are derived;
everything else is compared for equality."""
import ctypes

import numpy as np
import pytest
import torch

import test_gpu_kv_cache as base
from oracle import kv_cache as oracle
from test_gpu_kv_cache import CODES, DTYPES, check_attention, check_same, dev, f64, i32, make, nb, rounded  # noqa: F401  (nb: the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("low", [90.0, 1000.0])
@pytest.mark.parametrize("dtype,code,D,G,T", [("bf16", "i8", 64, 2, 1), ("f32", "e4m3", 128, 4, 4), ("bf16", "e4m3", 256, 1, 1), ("bf16", "i8", 64, 2, 200),
                                              ("bf16", "e4m3", 128, 2, 200), ("f32", "i8", 64, 1, 150), ("f32", "i8", 256, 2, 90)])
def test_attention_where_all_logits_are_low(nb, dtype, code, D, G, T, low):
    """Logits that are all far below zero, where 2 to the power of their negative is beyond fp32, in every row but each third one."""
    B, H, block, N = 2, 2, 32, 672
    rng = np.random.default_rng(D + T)
    cache, host = make(nb, rng, B, H, N, D, block, code, [N, 333])
    for i in (0, 2):
        host[i][..., 0] = 104.0                                  # (a code of both kinds)
        host[i + 1][:] = 2.0 ** -6
    put = lambda a, like: torch.from_numpy(a).float().to(like.dtype).cuda()  # noqa: E731
    cache = nb.kv_cache(put(host[0], cache.k), put(host[2], cache.v), put(host[1], cache.k_scale), put(host[3], cache.v_scale))
    q = rng.standard_normal((B, H * G, T, D)) * 0.1
    q[:, :, np.arange(T) % 3 != 2, 0] = -low * D ** 0.5 / (104 * 2.0 ** -6)
    q = rounded(q.astype(np.float32), dtype)
    got = nb.kv_cache_attn(cache, dev(q, DTYPES[dtype]), i32([N, 333]), want_lse=True, want_weights=True)
    want = oracle.attend(q, oracle.values(host[0], host[1]), oracle.values(host[2], host[3]), [N, 333], [T] * B, float(np.float32(D ** -0.5)), True)
    assert want[1][np.isfinite(want[1])].min() < 20 - low
    check_attention(*got, want, dtype, D, N, G * T)


def test_more_heads_than_a_grid_has_threads_for_along_an_axis(nb):
    """65535 sequences of 256 heads, which share what they hold, each with a workgroup to itself."""
    B, H, N, D = 65535, 256, 32, 64
    rng = np.random.default_rng(4)
    one, _ = make(nb, rng, 1, 1, N, D, 32, "i8", [N])
    cache = nb.kv_cache(one.k.expand(B, H, -1, -1), one.v.expand(B, H, -1, -1), one.k_scale.expand(B, H, -1).contiguous(), one.v_scale.expand(B, H, -1).contiguous())
    q = torch.randn((1, 1, 1, D), device="cuda").to(torch.bfloat16)
    lengths = torch.arange(B, device="cuda", dtype=torch.int32) % 33
    got = nb.kv_cache_attn(cache, q.expand(B, H, -1, -1), lengths)
    want = torch.cat([nb.kv_cache_attn(one, q, i32([n])) for n in range(33)])[:, 0, 0]
    for b in range(0, B, 4096):
        assert torch.equal(got[b:b + 4096, :, 0], want[lengths[b:b + 4096].long()][:, None].expand(-1, H, -1))


def test_more_blocks_than_a_grid_has_threads_for_along_an_axis(nb):
    """2^29 tokens in blocks of 32 enter a cache and move to another one."""
    N, D, block = 1 << 29, 64, 32
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 150 << 30:
        pytest.skip("needs 150 GiB of free memory")
    rng = np.random.default_rng(2)
    at = [slice(0, 64), slice((1 << 28) - 64, (1 << 28) + 64), slice(N - 64, N)]
    x = torch.empty((1, 1, N, D), device="cuda", dtype=torch.bfloat16)
    for j, a in enumerate(at):
        x[:, :, a] = dev(rng.standard_normal((1, 1, a.stop - a.start, D)) * 4.0 ** j, torch.bfloat16)
    raw = [torch.empty((1, 1, N, D), device="cuda", dtype=torch.int8) for _ in range(2)]
    scale = [torch.empty((1, 1, N // block), device="cuda") for _ in range(2)]
    cache = nb.kv_cache(*raw, *scale)
    nb.kv_cache_append(cache, x, x, i32([0]))
    small = nb.kv_cache_empty(1, 1, 256, D, block)
    nb.kv_cache_append(small, *[torch.cat([x[:, :, a] for a in at], 2)] * 2, i32([0]))
    del x
    torch.cuda.empty_cache()

    def check(c):
        for i in range(4):
            per = block if i >= 2 else 1
            got = torch.cat([c[i][:, :, a.start // per:a.stop // per] for a in at], 2)
            assert torch.equal(got, small[i])

    check(cache)
    to = nb.kv_cache(*(torch.empty_like(r) for r in raw), *(torch.empty_like(s) for s in scale))
    kept, _, left = nb.kv_cache_evict(cache, to, torch.zeros((1, 1, N), device="cuda"), i32([N]), N)
    assert left.item() == N and all(kept[0, 0, a].tolist() == list(range(a.start, a.stop)) for a in at)
    check(to)
    del cache, to, raw, scale, kept
    torch.cuda.empty_cache()


@pytest.mark.parametrize("zero", ["first", "some", "all"])
@pytest.mark.parametrize("dtype,code,D,G,T", [("bf16", "i8", 64, 2, 1), ("f32", "e4m3", 128, 4, 4), ("bf16", "i8", 64, 2, 200), ("bf16", "e4m3", 128, 2, 200),
                                              ("f32", "i8", 128, 1, 150), ("bf16", "i8", 256, 1, 90), ("f32", "e4m3", 256, 2, 90)])
def test_attention_to_blocks_of_scale_0(nb, dtype, code, D, G, T, zero):
    """A caller's own quantisation gives a block of zeros the scale 0: its tokens are zeros, whatever their codes."""
    B, H, block, N = 2, 2, 32, 608
    rng = np.random.default_rng(D + T)
    cache, host = make(nb, rng, B, H, N, D, block, code, [N, 333])
    blocks = {"first": [0, 1, 2, 3], "some": [4, 5, 9], "all": list(range(N // block))}[zero]
    for i in (1, 3):
        host[i] = rng.uniform(0.001, 0.02, host[i].shape).astype(np.float32).astype(np.float64)
        host[i][:, :, blocks] = 0.0
    host[1][0, 0] = 0.01                                         # one head has zeros among its values only
    cache = cache._replace(k_scale=dev(host[1], torch.float32), v_scale=dev(host[3], torch.float32))
    host[1], host[3] = f64(cache.k_scale), f64(cache.v_scale)
    key, value = oracle.values(host[0], host[1]), oracle.values(host[2], host[3])
    q = rounded((rng.standard_normal((B, H * G, T, D)) * 3).astype(np.float32), dtype)
    got = nb.kv_cache_attn(cache, dev(q, DTYPES[dtype]), i32([N, 333]), want_lse=True, want_weights=True)
    check_attention(*got, oracle.attend(q, key, value, [N, 333], [T] * B, float(np.float32(D ** -0.5)), True), dtype, D, N, G * T)


@pytest.mark.parametrize("code", ["i8", "e4m3"])
def test_append_to_and_evict_from_blocks_of_scale_0(nb, code):
    """Zeros that enter a block of scale 0 leave it one; others give it their scale."""
    rng = np.random.default_rng(1)
    B, H, N, D, block = 1, 2, 128, 64, 32
    cache, host = make(nb, rng, B, H, N, D, block, code, [N])
    for i in (1, 3):
        host[i][:, :, [0, 2]] = 0.0
    cache = cache._replace(k_scale=dev(host[1], torch.float32), v_scale=dev(host[3], torch.float32))
    zeros, ones = np.zeros((1, H, 3, D)), np.ones((1, H, 3, D))
    for at, x, y in ((5, zeros, zeros), (70, zeros, ones)):
        nb.kv_cache_append(cache, dev(x, torch.float32), dev(y, torch.float32), i32([at]))
        for i, new in ((0, x), (2, y)):
            if not new.any():
                host[i][:, :, at:at + 3] = 0.0                   # (the scale stays 0)
            else:
                oracle.append(host[i], host[i + 1], new, [at], [3], code)
    check_same(cache, host)
    assert all(torch.isfinite(c.float()).all() for c in cache[:2])
    w = rng.uniform(0, 1, (B, H, N)).astype(np.float32)
    to = nb.kv_cache_empty(B, H, 64, D, block, CODES[code])
    nb.kv_cache_evict(cache, to, dev(w), i32([N]), 50)
    for h in range(H):
        kept = oracle.select(w[0, h], N, 50, 1, 0)
        for codes, scale, i in ((to.k, to.k_scale, 0), (to.v, to.v_scale, 2)):
            ref, ref_scale = oracle.move(host[i][0, h], host[i + 1][0, h], kept, block, code)
            assert np.array_equal(f64(codes[0, h]), ref) and np.array_equal(f64(scale[0, h]), ref_scale)


def scale_beside_a_tie(code, tie):
    """A scale of 24 bits whose product with `code` (1 to 15) is next to `tie` (an odd number of 5 bits: half way between two of e4m3's) times
    2^23, nearer than fp32 can tell: (scale below 2, of the tie's own unit; the product's distance in units of 2^-23)."""
    for off in (1, -1, 2, -2, 3, -3, 5, -5, 7, -7):
        if (tie * 2 ** 23 + off) % code == 0:
            m = (tie * 2 ** 23 + off) // code
            while m >= 2 ** 24 and m % 2 == 0:
                m //= 2
            if 2 ** 23 <= m < 2 ** 24 and abs(off) * 2.0 ** -23 < tie * 2.0 ** -24:
                return m * 2.0 ** -23
    return None


def near_ties():
    """(code, scale): products that are no ties but round to one in fp32."""
    found = []
    for code in range(8, 16):
        for tie in range(17, 32, 2):
            s = scale_beside_a_tie(code, tie)
            if s is not None and float(np.float32(code * s)) != code * s and float(np.float32(code * s) * 2.0 ** 23) % 2 ** 19 == 0:
                found.append((code, s))
    return found


def test_moved_codes_are_rounded_once(nb):
    """Values of the caller's own scales that are no ties, but of which fp32 makes one: the nearest code is told by what fp32 drops."""
    pairs = near_ties()
    assert len(pairs) >= 8
    block, D, N = 32, 64, 32 * len(pairs)
    codes, scale = np.zeros((1, 1, N, D)), np.zeros((1, 1, len(pairs)))
    for j, (c, s) in enumerate(pairs):
        codes[0, 0, j * block:(j + 1) * block] = np.random.default_rng(j).integers(-c, c + 1, (block, D))
        codes[0, 0, j * block:j * block + 2] = np.array([[c], [-c]])
        scale[0, 0, j] = s
    put = torch.from_numpy(codes).float().to(torch.float8_e4m3fn).cuda()
    cache = nb.kv_cache(put, put.clone(), dev(scale, torch.float32), dev(scale, torch.float32))
    to = nb.kv_cache_empty(1, 1, N, D, block, torch.float8_e4m3fn)
    nb.kv_cache_evict(cache, to, torch.zeros((1, 1, N), device="cuda"), i32([N]), N)
    ref, ref_scale = oracle.move(codes[0, 0], scale[0, 0], np.arange(N), block, "e4m3")
    assert np.array_equal(f64(to.k_scale[0, 0]), ref_scale) and np.array_equal(f64(to.k[0, 0]), ref) and np.array_equal(f64(to.v[0, 0]), ref)
    # one token that needs a larger scale: what the block held is rounded again
    host = [codes, scale, codes.copy(), scale.copy()]
    for j in range(len(pairs)):
        x = np.full((1, 1, 1, D), 2.0 ** 11)
        nb.kv_cache_append(cache, dev(x, torch.float32), dev(x, torch.float32), i32([j * block + block - 1]))
        for i in (0, 2):
            oracle.append(host[i], host[i + 1], x, [j * block + block - 1], [1], "e4m3")
    check_same(cache, host)


@pytest.mark.parametrize("code,limit", [("i8", 127), ("e4m3", 448)])
def test_scales_beside_their_limits(nb, code, limit):
    """A block's largest value is beside the limit of a scale by less than fp32 can tell: the smallest scale that holds it is still meant."""
    found = []
    for c in range(1, 128 if code == "i8" else 16):
        m = round(limit * 2.0 ** 23 / c)
        for m in (m, m + 1):
            while m >= 2 ** 24:
                m //= 2
            while m < 2 ** 23:
                m *= 2
            s = m * 2.0 ** -23
            ratio = c * s / limit
            while ratio > 1.5:
                ratio /= 2
            while ratio < 0.75:
                ratio *= 2
            if 1 < ratio < 1 + 2.0 ** -24 or 1 - 2.0 ** -24 < ratio < 1:
                found.append((c, s))
    assert len(found) >= 4
    block, D, N = 32, 64, 32 * len(found)
    codes, scale = np.zeros((1, 1, N, D)), np.zeros((1, 1, len(found)))
    for j, (c, s) in enumerate(found):
        codes[0, 0, j * block + 3, 5] = -c
        scale[0, 0, j] = s
    put = torch.from_numpy(codes).float().to(CODES[code]).cuda()
    cache = nb.kv_cache(put, put.clone(), dev(scale, torch.float32), dev(scale, torch.float32))
    to = nb.kv_cache_empty(1, 1, N, D, block, CODES[code])
    nb.kv_cache_evict(cache, to, torch.zeros((1, 1, N), device="cuda"), i32([N]), N)
    ref, ref_scale = oracle.move(codes[0, 0], scale[0, 0], np.arange(N), block, code)
    assert np.array_equal(f64(to.k_scale[0, 0]), ref_scale) and np.array_equal(f64(to.k[0, 0]), ref)
    # a new token of just that size, and the floats next to it, in a block of such a scale
    for c, s in found:
        for x in (np.float32(limit * s), np.nextafter(np.float32(limit * s), np.float32(0)), np.nextafter(np.float32(limit * s), np.float32(1e9))):
            host = [np.zeros((1, 1, block, D)), np.full((1, 1, 1), s)]
            one = nb.kv_cache_empty(1, 1, block, D, block, CODES[code])
            one.k_scale.fill_(s), one.v_scale.fill_(s)
            new = np.full((1, 1, 1, D), float(x))
            nb.kv_cache_append(one, dev(new, torch.float32), dev(new, torch.float32), i32([4]))
            oracle.append(*host, new, [4], [1], code)
            assert one.k_scale.item() == host[1].item() and np.array_equal(f64(one.k), host[0])


@pytest.mark.parametrize("T", [1, 12, 70])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attention_of_the_largest_scales(nb, dtype, T):
    """A scale near the end of fp32's range, whose product with log2 e is beyond it, and queries as small as that takes."""
    D, N = 64, 256
    rng = np.random.default_rng(9)
    cache, host = make(nb, rng, 1, 1, N, D, 64, "i8", [N])
    q = rounded((rng.standard_normal((1, 2, T, D)) * 2.0 ** -131).astype(np.float32), dtype)
    scale = float(np.float32(3e38))
    got = nb.kv_cache_attn(cache, dev(q, DTYPES[dtype]), i32([N]), scale=scale, want_lse=True, want_weights=True)
    want = oracle.attend(q, oracle.values(host[0], host[1]), oracle.values(host[2], host[3]), [N], [T], scale, True)
    check_attention(*got, want, dtype, D, N, 2 * T)


def select(w, length, keep, n_global, n_recent):
    """oracle.select for weights without NaN, by a stable sort."""
    if length <= keep:
        return np.arange(length)
    order = np.argsort(-w[n_global:length - n_recent].astype(np.float64), kind="stable")[:keep - n_global - n_recent] + n_global
    return np.sort(np.concatenate([np.arange(n_global), order, np.arange(length - n_recent, length)]))


@pytest.mark.parametrize("N,lengths", [(1 << 19, [1 << 19, 524000]), ((1 << 19) + 64, [(1 << 19) + 64, 500001, 8193]), (1700032, [1700001, 300000])])
@pytest.mark.parametrize("kind", ["spread", "few"])
def test_evict_of_very_long_sequences(nb, kind, N, lengths):
    """Sequences of more pieces than there are workgroups for, up to and beyond the first such length."""
    B, H, D, block, keep = len(lengths), 2, 64, 64, 40000
    rng = np.random.default_rng(N)
    w = rng.uniform(0, 1, (B, H, N)).astype(np.float32) if kind == "spread" else rng.integers(0, 9, (B, H, N)).astype(np.float32)
    k = torch.arange(N, device="cuda", dtype=torch.int32)[:, None].bitwise_right_shift(torch.arange(D, device="cuda", dtype=torch.int32) % 24) % 100
    k = k.to(torch.int8).expand(B, H, N, D)                        # codes that tell tokens apart
    scale = torch.ones((B, H, N // block), device="cuda")
    v = torch.empty((N, D), device="cuda", dtype=torch.int8).copy_(k[0, 0]).neg_().expand(B, H, N, D)
    to = nb.kv_cache_empty(B, H, -(-keep // block) * block, D, block)
    kept, w_out, left = nb.kv_cache_evict(nb.kv_cache(k, v, scale, scale.clone()), to, dev(w), i32(lengths), keep, n_global=5, n_recent=300)
    assert left.tolist() == [min(n, keep) for n in lengths]
    kept, w_out = kept.cpu().numpy(), w_out.cpu().numpy()
    for b in range(B):
        for h in range(H):
            want = select(w[b, h], lengths[b], keep, 5, 300)
            n = len(want)
            assert np.array_equal(kept[b, h, :n], want) and (kept[b, h, n:] == -1).all()
            assert np.array_equal(w_out[b, h, :n], w[b, h, want]) and not w_out[b, h, n:].any()
            at = torch.from_numpy(want).cuda()
            values = oracle.values(f64(to.k[b:b + 1, h:h + 1]), f64(to.k_scale[b:b + 1, h:h + 1]))[0, 0, :n]
            assert np.array_equal(values, f64(k[b, h][at])) and np.array_equal(f64(to.v[b, h]), -f64(to.k[b, h]))


# ---- kernels' variants that the sizes of test_gpu_kv_cache.py do not reach


@pytest.mark.parametrize("kind", ["spread", "few", "odd"])
@pytest.mark.parametrize("code,B,H,D,block,N,M,keep,n_global,n_recent,lengths", [
    ("i8", 2, 1, 64, 64, 8256, 4096, 4000, 1, 0, [8193, 8256]),            # more than 8192 tokens in one workgroup's registers
    ("e4m3", 4, 1, 64, 32, 16384, 8192, 8192, 4, 100, [16384, 16383, 8193, 8192]),     # as many as it takes
    ("i8", 3, 1, 64, 32, 16416, 8192, 8001, 4, 100, [16416, 16384, 8192]),   # and more
    ("e4m3", 2, 2, 128, 128, 640, 384, 300, 1, 0, [640, 401]),             # blocks of 16384 codes
    ("i8", 2, 1, 256, 64, 640, 320, 257, 0, 5, [640, 300]),
    ("e4m3", 1, 2, 256, 128, 1280, 640, 600, 3, 70, [1280]),               # and of 32768
    ("i8", 2, 1, 256, 128, 1280, 640, 513, 3, 70, [1279, 513]),
])
def test_evict_of_other_sizes(nb, code, kind, B, H, D, block, N, M, keep, n_global, n_recent, lengths):
    base.test_evict(nb, code, kind, B, H, D, block, N, M, keep, n_global, n_recent, lengths)


@pytest.mark.parametrize("dtype,code,B,H,G,D,block,N,T,lengths,causal", [
    ("bf16", "i8", 16, 16, 1, 256, 64, 256, 40, None, True),               # 256 channels' weights without rows to share out
    ("bf16", "e4m3", 8, 16, 1, 256, 32, 544, 40, None, False),
    ("f32", "e4m3", 16, 16, 1, 256, 32, 160, 40, None, True),
    ("bf16", "i8", 1, 1, 1, 64, 32, 32, 70, [32], True),                   # many rows of a single block, and of one and a half tiles
    ("f32", "e4m3", 2, 1, 1, 128, 32, 32, 40, [31, 32], False),
    ("bf16", "e4m3", 1, 1, 1, 256, 32, 32, 40, [32], True),
    ("f32", "i8", 1, 1, 2, 256, 32, 96, 40, [95], True),
    ("bf16", "i8", 1, 2, 1, 128, 32, 96, 70, [96], True),
])
def test_attention_of_other_sizes(nb, dtype, code, B, H, G, D, block, N, T, lengths, causal):
    lengths = [N, 0, 1, N - 1, *np.random.default_rng(B).integers(0, N + 1, B).tolist()][:B] if lengths is None else lengths
    base.attention_case(nb, dtype, code, B, H, G, D, block, N, T, lengths, None, causal)


@pytest.mark.parametrize("D,T,N", [(64, 1, 96), (128, 3, 1024), (64, 90, 640), (256, 33, 512)])
def test_nothing_is_written_beside_the_log_sums(nb, D, T, N):
    """lse is asked of the C ABI, between guard bands; what it holds is what the binding returns."""
    B, H, G, block = 2, 2, 2, 32
    rng = np.random.default_rng(D)
    lengths = [N, N // 2]
    cache, _ = make(nb, rng, B, H, N, D, block, "i8", lengths)
    q = torch.randn((B, H * G, T, D), device="cuda", dtype=torch.bfloat16)
    bands, n = base.Bands(), i32(lengths)
    out, lse = bands((B, H * G, T, D), torch.bfloat16), bands((B, H * G, T), torch.float32)
    d = nb.ns_kv_attn_desc(H * G, T, nb.NS_BF16, 1, D ** -0.5, *q.stride()[:3], *out.stride()[:3])
    c = nb.ns_kv_cache(B, H, D, N, block, nb.NS_CODE_I8, *cache.k.stride()[:3], *(t.data_ptr() for t in cache))
    need = nb.lib.kv_cache_attn_workspace_bytes(ctypes.byref(c), ctypes.byref(d), 0)
    ws = bands((need,), torch.uint8)
    torch.cuda.synchronize()
    assert nb.lib.kv_cache_attn(ctypes.byref(c), ctypes.byref(d), q.data_ptr(), n.data_ptr(), None, out.data_ptr(), lse.data_ptr(), None, None,
                                ws.data_ptr() if need else None, need, None) == nb.NS_OK
    bands.check()
    want = nb.kv_cache_attn(cache, q, n, want_lse=True)
    assert torch.equal(out, want[0]) and torch.equal(lse, want[1])


@pytest.mark.parametrize("T", [1, 70])
@pytest.mark.parametrize("dtype,code,D,N", [("bf16", "i8", 64, 32), ("f32", "e4m3", 128, 64), ("bf16", "e4m3", 128, 2048), ("f32", "i8", 256, 64), ("bf16", "i8", 256, 2048)])
def test_log_sums_of_few_keys_with_small_logits(nb, dtype, code, D, N, T):
    """Rows of one channel, whose logits are single products: z is off by the scaling's four roundings.  One key's log-sum is its logit and
    its weight is 1; that of n equal keys is log n more, its weights 1 / n.  Roundings behind z: the sum's (a whole number, exact), the
    logarithm's and the two that put z and it together, 2^-24 each of the larger one (the instruction's: 2^-23); the weight's exponent twice
    that, its exponential 2^-23.  bf16 calls of many rows in caches of more than 512 tokens have exponents that are 11 higher, in steps of 2^-20: half of one for the weight, and
    one for the sum's logarithm, times log 2, are 2^-20 more of the log-sum and twice that of the weights.  In the fp32 calls out is the value to the weight's two parts (2^-23) and the normalisation (2^-23)."""
    n = 5 if T == 1 else 3
    B, H, block = n, 1, 32
    codes = torch.zeros((B, H, N, D)).to(CODES[code])
    codes[..., 0] = torch.full((B, H, N), 96.0).to(CODES[code])
    codes = codes.cuda()
    scale = torch.full((B, H, N // block), 2.0 ** -9, device="cuda")
    cache = nb.kv_cache(codes, codes.clone(), scale, scale.clone())
    q = np.zeros((B, H, T, D))
    q[..., 0] = np.random.default_rng(D).uniform(-9, 9, (B, H, T))
    q = rounded(q.astype(np.float32), dtype)
    lengths = list(range(1, n + 1))
    out, lse, weights = nb.kv_cache_attn(cache, dev(q, DTYPES[dtype]), i32(lengths), scale=0.1, causal=False, want_lse=True, want_weights=True)
    z = float(np.float32(0.1)) * q[..., 0] * 96 * 2.0 ** -9
    many = np.array(lengths)[:, None, None]
    want, size = z + np.log(many), np.maximum(np.abs(z), np.log(many))
    more = 2.0 ** -20 if dtype == "bf16" and T == 70 and N > 512 else 0.0
    assert (np.abs(f64(lse) - want) <= more + 4 * 2.0 ** -24 * np.abs(z) + 4 * 2.0 ** -24 * np.maximum(size, np.abs(want))).all()
    step = 2 * (8 * 2.0 ** -24 * np.maximum(size, np.abs(want))).max() + 2.0 ** -23 + 2 * more
    for b in range(B):
        assert np.abs(f64(weights)[b, 0, :lengths[b]] * lengths[b] / T - 1).max() <= step + T * 2.0 ** -24
        assert not f64(weights)[b, 0, lengths[b]:].any()
    half = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    assert np.abs(f64(out)[..., 0] / (96 * 2.0 ** -9) - 1).max() <= 2.0 ** -22 + half and not f64(out)[..., 1:].any()


@pytest.mark.parametrize("code", ["i8", "e4m3"])
def test_from_the_backbone_into_the_cache(nb, code):
    """What a reader behind the backbone calls: the stack prunes, linear maps make keys and values of the tokens it kept, these enter a cache
    as views of the map's output, queries attend across them with weights, and the tokens with the least weight leave.  The oracle of the cache
    starts from what the maps wrote."""
    from paper_2601_12150_amd import synth
    from test_gpu_vit_block import dev_weights
    B, g, heads, dim, keep_k, H, G, D, block, T = 2, 16, 8, 512, 150, 2, 2, 128, 32, 40
    rng = np.random.default_rng(30)
    x = dev(synth.round_to_bf16(rng.standard_normal((B, 1 + g * g, dim)).astype(np.float32)), torch.bfloat16)
    tokens, kept = nb.vit_forward(x, [dev_weights(synth.make_block_weights(dim, dim, seed=40 + i)) for i in range(2)], g, g, 8, heads, prune_after=1, keep_k=keep_k)
    n = 1 + keep_k
    w = dev(synth.round_to_bf16((rng.standard_normal((2 * H * D, dim)) * dim ** -0.5).astype(np.float32)), torch.bfloat16)
    kv = nb.linear_forward(tokens.view(B * n, dim), w, torch.zeros(2 * H * D, device="cuda")).view(B, n, 2, H, D)
    k, v = (kv[:, :, i].transpose(1, 2) for i in range(2))
    N = 192
    cache = nb.kv_cache_empty(B, H, N, D, block, CODES[code])
    nb.kv_cache_append(cache, k, v, i32([0] * B))
    host = [np.zeros((B, H, N, D)), np.ones((B, H, N // block)), np.zeros((B, H, N, D)), np.ones((B, H, N // block))]
    for i, t in ((0, k), (2, v)):
        oracle.append(host[i], host[i + 1], f64(t), [0] * B, [n] * B, code)
    check_same(cache, host)
    q = dev(rounded(rng.standard_normal((B, H * G, T, D)).astype(np.float32), "bf16"), torch.bfloat16)
    out, lse, weights = nb.kv_cache_attn(cache, q, i32([n] * B), causal=False, want_lse=True, want_weights=True)
    want = oracle.attend(f64(q), oracle.values(host[0], host[1]), oracle.values(host[2], host[3]), [n] * B, [T] * B, float(np.float32(D ** -0.5)), False)
    check_attention(out, lse, weights, want, "bf16", D, N, G * T)
    to = nb.kv_cache_empty(B, H, 96, D, block, CODES[code])
    chosen, moved, left = nb.kv_cache_evict(cache, to, weights, i32([n] * B), 90)
    assert left.tolist() == [90] * B and (chosen[:, :, 0] == 0).all()              # (the CLS token stays)
    for b in range(B):
        for h in range(H):
            at = oracle.select(weights[b, h].cpu().numpy(), n, 90, 1, 0)
            assert np.array_equal(chosen[b, h].cpu().numpy(), at) and torch.equal(moved[b, h, :90], weights[b, h][chosen[b, h].long()])
            # the patches that they are, in the image
            patches = kept[b][chosen[b, h, 1:].long() - 1]
            assert (patches[1:] > patches[:-1]).all()
            for codes, scale, i in ((to.k, to.k_scale, 0), (to.v, to.v_scale, 2)):
                ref, ref_scale = oracle.move(host[i][b, h], host[i + 1][b, h], at, block, code)
                assert np.array_equal(f64(codes[b, h]), ref) and np.array_equal(f64(scale[b, h]), ref_scale)
