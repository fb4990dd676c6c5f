"""Rotary positions with several axes, the pages of a pool and the 4-bit cache, as far as it goes without a GPU: refusals before any launch,
the validation under host sanitizers, and what pins the oracle."""
import ctypes
import os
import shutil
import subprocess

import numpy as np
import pytest
import torch

from oracle import cache_oracle, pages_oracle
from paper_2407_08608_amd import binding
from test_cache_host import _BAD_CACHES, _CACHE, P, ROOT, SAN, _attend, _longs, _read, _write

FP4 = binding.FA_FP4_E2M1


@pytest.mark.parametrize("bwd", [False, True])
@pytest.mark.parametrize("kw,status", [
    (dict(q=None), 1), (dict(qo=None), 1), (dict(f=None), 1), (dict(ko=None), 1), (dict(axis=None), 1), (dict(pos=None), 1), (dict(dtype=-1), 3),
    (dict(dtype=FP4), 3), (dict(dtype=binding.FA_FP8_E4M3), 4), (dict(axes=0), 2), (dict(axes=-1), 2), (dict(B=0), 2), (dict(H_kv=0), 2), (dict(rot=80), 2),
    (dict(amp=0.0), 2), (dict(il=2), 2), (dict(d=96, rot=32), 4), (dict(rot=24), 4), (dict(axis=P + 2), 5), (dict(pos=P + 1), 5), (dict(f=P + 4), 5),
    (dict(k=P + 8), 5), (dict(qs=_longs(0, 512, 65)), 5), (dict(kos=_longs(0, 32, 64)), 2)])
def test_rope_axes_refuses_before_any_launch(bwd, kw, status):
    a = dict(q=P, qs=None, k=P, ks=None, qo=P, qos=None, ko=P, kos=None, f=P, axis=P, pos=P, axes=3, B=1, H=4, H_kv=2, N=8, d=64, rot=64, amp=1.0, il=0,
             dtype=binding.FA_BF16)
    assert set(kw) <= set(a)
    a.update(kw)
    L = binding.lib()
    assert (L.fa_rope_axes_bwd if bwd else L.fa_rope_axes)(*a.values(), None) == status


_FOUR = dict(ks=P, vs=P, cache=FP4)


@pytest.mark.parametrize("call", [_write, _read, _attend])
@pytest.mark.parametrize("kw,status", [(dict(ks=None), 1), (dict(vs=None), 1), (dict(ks=P + 2), 5), (dict(vs=P + 1), 5), (dict(kp=P + 8), 5), (dict(page=24), 4),
                                       (dict(d=96), 4), (dict(max_pages=0), 2)])
def test_a_4_bit_cache_is_refused_before_any_launch(call, kw, status):
    assert call(**dict(_FOUR, **kw)) == status


def test_a_4_bit_cache_with_other_types():
    assert _write(**_FOUR, dense=FP4) == 3 and _read(**_FOUR, dense=FP4) == 3 and _write(**_FOUR, dense=binding.FA_FP8_E4M3) == 4
    W = binding.fa_fwd_cache_workspace_bytes
    assert W(2, 4, 2, 1, 128, 100000, FP4) > 0 and W(2, 4, 2, 1, 128, 100000, 5) == 0
    assert _attend(**_FOUR, ws=None, ws_bytes=0, max_len=100000) == 6


def _copy(**kw):
    a = dict(kp=P, vp=P, ks=None, vs=None, src=P, dst=P, n=3, H_kv=2, d=64, page=16, n_pages=9, cache=binding.FA_BF16)
    assert set(kw) <= set(a)
    a.update(kw)
    return binding.lib().fa_cache_copy(*a.values(), None)


@pytest.mark.parametrize("kw,status", [x for x in _BAD_CACHES if not {"table", "lens", "B", "max_pages"} & set(x[0])] + [
    (dict(src=None), 1), (dict(dst=None), 1), (dict(n=0), 2), (dict(n=-1), 2), (dict(src=P + 2), 5), (dict(dst=P + 1), 5), (dict(_FOUR, vs=None), 1)])
def test_copy_refuses_before_any_launch(kw, status):
    assert _copy(**kw) == status


def _fork(**kw):
    a = dict(table=P, lens=P, parents=P, held=P, new=2 * P, new_lens=3 * P, src=P, dst=P, missing=P, ws=P, bytes=1 << 20, B=3, B_new=4, page=16, n_pages=9, max_pages=5)
    assert set(kw) <= set(a)
    a.update(kw)
    return binding.lib().fa_cache_fork(*a.values(), None)


def _extend(**kw):
    a = dict(table=P, lens=P, counts=P, held=P, missing=P, ws=P, bytes=1 << 20, B=3, T=4, page=16, n_pages=9, max_pages=5)
    assert set(kw) <= set(a)
    a.update(kw)
    return binding.lib().fa_cache_extend(*a.values(), None)


def _compact(**kw):
    a = dict(table=P, held=P, new=P, src=P, dst=P, top=P, ws=P, bytes=1 << 20, B=3, moves=4, n_pages=9, max_pages=5)
    assert set(kw) <= set(a)
    a.update(kw)
    return binding.lib().fa_cache_compact(*a.values(), None)


@pytest.mark.parametrize("call,kw,status", [
    (c, kw, s) for c, ptrs in ((_fork, ("table", "lens", "parents", "new", "new_lens", "src", "dst", "missing")), (_extend, ("table", "lens", "missing")),
                               (_compact, ("table", "new", "src", "dst", "top"))) for kw, s in
    [({p: None}, 1) for p in ptrs] + [({p: P + 2}, 5) for p in ptrs + ("held",)] +
    [(dict(B=0), 2), (dict(n_pages=0), 2), (dict(max_pages=0), 2), (dict(B=1 << 16, max_pages=1 << 15), 2), (dict(ws=None, n_pages=5000), 6), (dict(bytes=3, n_pages=5000), 6), (dict(ws=P + 8, n_pages=5000), 5)]
] + [(_fork, dict(B_new=0), 2), (_fork, dict(B_new=-1), 2), (_fork, dict(page=0), 2), (_fork, dict(page=1 << 16, max_pages=1 << 15), 2), (_fork, dict(new=P), 2), (_fork, dict(new_lens=P), 2),
     (_fork, dict(B_new=1 << 16, max_pages=1 << 15), 2), (_extend, dict(T=0), 2), (_extend, dict(page=-1), 2), (_extend, dict(B=3, T=1 << 30), 2),
     (_extend, dict(counts=P + 1), 5), (_compact, dict(moves=0), 2), (_compact, dict(moves=-5), 2)])
def test_pages_refuse_before_any_launch(call, kw, status):
    assert call(**kw) == status


def test_workspace_of_pages():
    W = binding.fa_cache_pages_workspace_bytes
    assert W(0, 9) == 0 and W(3, 0) == 0 and W(3, 9) == 0 and W(1024, 4096) == 0 and W(1025, 9) >= 4 * 27 and W(3, 4097) >= 4 * 3 * 4097
    for B, n_pages in ((2000, 9), (4, 100000)):
        need = W(B, n_pages)
        assert _fork(B_new=B, n_pages=n_pages, bytes=need - 1) == 6 and _extend(B=B, n_pages=n_pages, bytes=need - 1) == 6
        assert _compact(B=B, n_pages=n_pages, bytes=need - 1) == 6


def test_the_binding_refuses_tensors_that_are_not_on_a_device():
    i, x = torch.zeros((2, 3), dtype=torch.int32), torch.zeros((4, 1, 16, 32), dtype=torch.uint8)
    s, q = torch.zeros((4, 1, 16, 2), dtype=torch.uint8), torch.zeros((2, 1, 1, 64), dtype=torch.bfloat16)
    for call in (lambda: binding.fa_cache_fork(i, i[:, 0], i[0], 16, 4), lambda: binding.fa_cache_extend(i, i[:, 0], 1, 16, 4), lambda: binding.fa_cache_compact(i, 4),
                 lambda: binding.fa_cache_copy(x, x, i[0], i[0], k_scales=s, v_scales=s), lambda: binding.fa_cache_read(x, x, i, i[:, 0], 3, k_scales=s, v_scales=s),
                 lambda: binding.fa_fwd_cache(q, x, x, i, i[:, 0], 0.1, k_scales=s, v_scales=s), lambda: binding.fa_rope_axes(q, s, i[0], i[None]),
                 lambda: binding.fa_rope_axes_bwd(q, s, i[0], i[0])):
        with pytest.raises((ValueError, RuntimeError)):
            call()


def test_argument_validation_under_host_sanitizers(tmp_path):
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if not (os.path.exists(hipcc) or shutil.which(hipcc)):
        pytest.skip("hipcc not available")
    exe = str(tmp_path / "pages_api_san")
    cmd = [hipcc, "--offload-arch=gfx950", "-std=c++17", "-O1", "-g", "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined", "-Xarch_host",
           "-fno-sanitize-recover=all", os.path.join(ROOT, "paper_2407_08608_amd", "csrc", "fa_pages_api.hip"), os.path.join(SAN, "pages_api_driver.cpp"), "-o", exe,
           "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined"]
    subprocess.run(cmd, check=True, stderr=subprocess.DEVNULL)
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:exitcode=23", UBSAN_OPTIONS="halt_on_error=1:exitcode=24")
    r = subprocess.run([exe], env=env, capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stdout + r.stderr
    assert "pages api sanitizer run: 0 failures" in r.stdout


# ---- the oracle: closed forms and invariants


def test_oracle_axes_of_equal_positions_are_one_axis():
    g = np.random.default_rng(1)
    x, pos = g.standard_normal((2, 3, 5, 64)), g.integers(-5, 1000, (2, 5))
    f, _ = cache_oracle.frequencies(32, 10000.0)
    for interleaved in (False, True):
        for back in (False, True):
            y = cache_oracle.rope_axes(x, f, g.integers(0, 3, 16), np.stack([pos] * 3), 32, interleaved, 1.5, back)
            np.testing.assert_allclose(y, cache_oracle.rope(x, f, pos, 32, interleaved, 1.5, back), atol=1e-12)
    y = cache_oracle.rope_axes(x, f, [0, 1] * 8, np.stack([pos, 0 * pos]), 32, True)
    np.testing.assert_array_equal(y.reshape(2, 3, 5, 32, 2)[..., 1:16:2, :], x.reshape(2, 3, 5, 32, 2)[..., 1:16:2, :])  # pairs of the axis that stands still


def test_oracle_e2m1():
    assert cache_oracle.e2m1_decode(np.arange(16)).tolist() == [0, .5, 1, 1.5, 2, 3, 4, 6, 0, -.5, -1, -1.5, -2, -3, -4, -6]
    np.testing.assert_array_equal(cache_oracle.e2m1_encode(cache_oracle.e2m1_decode(np.arange(16))), np.arange(16))
    # from the middle to the even code, and to no other from next to it
    middle = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0])
    assert cache_oracle.e2m1_encode(middle).tolist() == [0, 2, 2, 4, 4, 6, 6]
    assert cache_oracle.e2m1_encode(np.nextafter(middle, 9)).tolist() == [1, 2, 3, 4, 5, 6, 7] and cache_oracle.e2m1_encode(np.nextafter(middle, 0)).tolist() == [0, 1, 2, 3, 4, 5, 6]
    g = np.random.default_rng(2)
    x = (g.standard_normal((50, 96)) * 2.0 ** g.integers(-60, 60, (50, 1))).astype(np.float32)
    x[3, :32] = 0
    codes, scales = cache_oracle.quantise_groups(x)
    assert codes.shape == (50, 48) and scales.shape == (50, 3) and scales[3, 0] == 27
    back = cache_oracle.group_values(codes, scales)
    a = np.repeat(np.abs(x.astype(np.float64)).reshape(50, 3, 32).max(-1), 32, axis=-1)
    assert (np.abs(back - x) <= a * (1 / 3.5) + 1e-300).all()  # half of the widest step, 2 s, and a > 3.5 s
    assert (np.repeat(2.0 ** (scales - 127.0), 32, axis=-1) * 7 >= a).all() and (a[a > 0] > 3.5 * np.repeat(2.0 ** (scales - 127.0), 32, axis=-1)[a > 0]).all()
    again = cache_oracle.quantise_groups(back.astype(np.float32))
    np.testing.assert_array_equal(cache_oracle.group_values(*again), back)  # values of the cache are kept as they are


def test_oracle_pages():
    # a page of 4 tokens; two sequences that share page 5; the first has 6 tokens, the second 9
    table, lens = [[5, 2, -1], [5, 7, 0]], [6, 9]
    rows, n, src, dst, missing = pages_oracle.fork(table, lens, [0, 0, 1, -1], None, 4, 10)
    assert rows == [[5, 2, -1], [5, 1, -1], [5, 7, 0], [-1] * 3] and n == [6, 6, 9, 0] and (src, dst, missing) == ([-1, 2, -1, -1], [-1, 1, -1, -1], 0)
    assert pages_oracle.fork(table, lens, [0, 0, 0], None, 4, 6)[0][2] == [5, 1, -1]  # (page 7 is none of 6; pages 0 and 1 are free)
    held = [1, 1, 0, 1, 1, 0]
    assert pages_oracle.fork(table, lens, [0, 0], held, 4, 6)[2:] == ([-1, -1], [-1, -1], 1)
    assert pages_oracle.extend(table, lens, [3, 4], None, 4, 10) == ([[5, 2, 1], [5, 7, 0]], 1)
    assert pages_oracle.compact(table, None, 10, 5) == ([[3, 2, -1], [3, 1, 0]], [7, 5, -1, -1, -1], [1, 3, -1, -1, -1], 4)
    assert pages_oracle.compact(table, [0] * 7 + [1, 0, 0], 10, 5) == ([[1, 2, -1], [1, 7, 0]], [5] + [-1] * 4, [1] + [-1] * 4, 8)
    assert pages_oracle.compact(table, None, 10, 1)[1:] == ([7], [1], 6)
    assert pages_oracle.compact([[-1]], None, 3, 1) == ([[-1]], [-1], [-1], 0)
