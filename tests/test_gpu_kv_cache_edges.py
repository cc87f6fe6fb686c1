"""The 8-bit key/value cache at the edges of what its entry points take, against the float64 oracle: logits far below zero, scales of 0,
scales between whose roundings there is next to nothing.  Attention's tolerances are those of test_gpu_kv_cache.py, where they are derived;
everything else is compared for equality."""
import ctypes

import numpy as np
import pytest
import torch

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
