"""The 8-bit key/value cache at the limits of what its entry points take, without a GPU."""
import ctypes
import os
import subprocess

import pytest

from paper_2601_12150_amd import build as hip_build


@pytest.mark.skipif(not os.path.exists(hip_build.HIPCC), reason="needs hipcc")
def test_shares_of_as_many_tiles_as_there_may_be(tmp_path):
    """Every workgroup's share of the tiles covers them all, without one that is not needed, up to the last number that is let through."""
    src = tmp_path / "shares.hip"
    src.write_text('#include "%s"\n' % os.path.join(hip_build.CSRC, "ns_kv.h") + """
constexpr bool good(int tiles, int workgroups) {
  const long long share = ns::kv_share(tiles, workgroups);
  return share >= 1 && share * workgroups >= tiles && (tiles == 0 || (share - 1) * workgroups < tiles);
}
constexpr bool all_good() {
  for (int workgroups : {1, 255, 256, 512, 1024})
    for (int tiles : {0, 1, 511, 512, 513, 1 << 30, 0x7fffffff - 511, 0x7fffffff - 1, 0x7fffffff})
      if (!good(tiles, workgroups)) return false;
  return true;
}
static_assert(all_good(), "shares");
""")
    r = subprocess.run([hip_build.HIPCC, "--offload-host-only", "-fsyntax-only", "-std=c++17", str(src)], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert r.returncode == 0, r.stdout[-2000:]


def test_the_selections_scratch_does_not_grow_without_end():
    """Its histograms are read by every workgroup of the sequence and head: their number has an end."""
    from paper_2601_12150_amd import binding as nb
    need = []
    for capacity in [1 << n for n in range(10, 31)]:
        c = nb.ns_kv_cache(3, 2, 64, capacity, 64, nb.NS_CODE_I8, 2 * capacity * 64, capacity * 64, 64, 0x10000, 0x20000, 0x30000, 0x40000)
        need.append(nb.lib.kv_cache_evict_workspace_bytes(ctypes.byref(c), 64))
    assert need[0] == 0 and need[10] > 0 and max(need) <= 6 * (2 << 20)


def test_an_evictions_workspace_is_checked():
    """A cache of 2^20 tokens needs one."""
    from paper_2601_12150_amd import binding as nb
    P = [ctypes.c_void_p(0x10000 * (i + 1)) for i in range(8)]
    c, to = (nb.ns_kv_cache(1, 2, 64, n, 64, nb.NS_CODE_I8, 2 * n * 64, n * 64, 64) for n in (1 << 20, 128))
    for i, x in enumerate((c, to)):
        x.k, x.v, x.k_scale, x.v_scale = (0x10000000 * (4 * i + j + 1) for j in range(4))
    need = nb.lib.kv_cache_evict_workspace_bytes(ctypes.byref(c), 100)
    assert need > 0

    def evict(ws, size):
        return nb.lib.kv_cache_evict(ctypes.byref(c), ctypes.byref(to), P[0], P[1], 100, 1, 2, P[2], P[3], P[4], ws, size, None)

    for ws, size in ((None, 0), (None, need), (P[5], need - 1), (P[5], 0), (ctypes.c_void_p(0x60010), need)):
        assert evict(ws, size) == nb.NS_ERR_WORKSPACE, (ws, size)
