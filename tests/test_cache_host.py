"""Rotary positions, the paged cache and attention over it, as far as it goes without a GPU: refusals before any launch, the
frequencies, the tree words, and the fp64 oracle itself."""
import ctypes
import math
import os
import shutil
import subprocess

import numpy as np
import pytest
import torch

import oracle
from oracle import cache_oracle, fp8_oracle
from paper_2407_08608_amd import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SAN = os.path.join(ROOT, "tests", "sanitize")
P = 0x1000  # an aligned address that nothing reads: validation fails first
NAN = float("nan")


def _longs(*x):
    return (ctypes.c_longlong * 3)(*x)


def _rope(bwd=False, **kw):
    a = dict(q=P, qs=None, k=P, ks=None, qo=P, qos=None, ko=P, kos=None, f=P, pos=P, B=1, H=4, H_kv=2, N=8, d=64, rot=64, amp=1.0, il=0,
             dtype=binding.FA_BF16)
    assert set(kw) <= set(a)
    a.update(kw)
    L = binding.lib()
    return (L.fa_rope_bwd if bwd else L.fa_rope)(*a.values(), None)


@pytest.mark.parametrize("bwd", [False, True])
@pytest.mark.parametrize("kw,status", [
    (dict(q=None), 1), (dict(qo=None), 1), (dict(f=None), 1), (dict(ko=None), 1),
    (dict(dtype=-1), 3), (dict(dtype=4), 3), (dict(dtype=binding.FA_FP8_E4M3), 4),
    (dict(B=0), 2), (dict(H=0), 2), (dict(H_kv=0), 2), (dict(N=0), 2), (dict(d=0), 2), (dict(rot=0), 2), (dict(rot=80), 2),
    (dict(amp=0.0), 2), (dict(amp=NAN), 2), (dict(amp=float("inf")), 2), (dict(il=2), 2), (dict(B=1 << 16, N=1 << 16), 2),
    (dict(H=0x7fffffff), 2), (dict(d=96, rot=32), 4), (dict(rot=24), 4), (dict(rot=8), 4),
    (dict(q=P + 8), 5), (dict(k=P + 8), 5), (dict(qo=P + 2), 5), (dict(ko=P + 8), 5), (dict(f=P + 4), 5), (dict(pos=P + 2), 5),
    (dict(qs=_longs(0, 0, -64), N=2), 2), (dict(qs=_longs(0, 512, 65)), 5), (dict(ks=_longs(0, 511, 64)), 5),
    (dict(qos=_longs(0, 512, 0)), 2), (dict(kos=_longs(0, 32, 64)), 2), (dict(dtype=binding.FA_F32, qs=_longs(0, 512, 66)), 5),
])
def test_rope_refuses_before_any_launch(bwd, kw, status):
    assert _rope(bwd, **kw) == status


_CACHE = dict(kp=P, vp=P, ks=None, vs=None, table=P, lens=P)
_CODES = dict(ks=P, vs=P, cache=binding.FA_FP8_E4M3)
# what is refused in each of the three calls on a cache, and with which status
_BAD_CACHES = [(dict(kp=None), 1), (dict(vp=None), 1), (dict(table=None), 1), (dict(lens=None), 1), (dict(_CODES, ks=None), 1),
               (dict(_CODES, vs=None), 1), (dict(ks=P), 3), (dict(vs=P), 3), (dict(cache=7), 3), (dict(cache=-1), 3),
               (dict(cache=binding.FA_F32), 4), (dict(B=0), 2), (dict(H_kv=0), 2), (dict(d=0), 2), (dict(page=0), 2), (dict(n_pages=0), 2),
               (dict(max_pages=0), 2), (dict(page=-16), 2), (dict(page=1 << 16, max_pages=1 << 15), 2), (dict(page=24), 4), (dict(page=8), 4),
               (dict(d=96), 4), (dict(page=1 << 24, d=64), 4), (dict(kp=P + 8), 5), (dict(vp=P + 2), 5), (dict(_CODES, ks=P + 2), 5),
               (dict(_CODES, vs=P + 1), 5), (dict(table=P + 2), 5), (dict(lens=P + 1), 5)]


def _write(**kw):
    a = dict(k=P, kst=None, v=P, vst=None, **_CACHE, counts=P, B=2, H_kv=2, T=3, d=64, page=16, n_pages=9, max_pages=4,
             dense=binding.FA_BF16, cache=binding.FA_BF16)
    assert set(kw) <= set(a)
    a.update(kw)
    return binding.lib().fa_cache_write(*a.values(), None)


def _read(**kw):
    a = dict(**_CACHE, k=P, v=P, B=2, H_kv=2, N=3, d=64, page=16, n_pages=9, max_pages=4, cache=binding.FA_BF16, dense=binding.FA_BF16)
    assert set(kw) <= set(a)
    a.update(kw)
    return binding.lib().fa_cache_read(*a.values(), None)


def _attend(**kw):
    a = dict(q=P, qst=None, **_CACHE, counts=P, tree=P, batches=2, o=P, ost=None, lse=P, ws=P, ws_bytes=1 << 40, B=2, H=4, H_kv=2, T=3, d=64,
             page=16, n_pages=9, max_pages=4, max_len=0, scale=0.125, dense=binding.FA_BF16, cache=binding.FA_BF16)
    assert set(kw) <= set(a)
    a.update(kw)
    return binding.lib().fa_fwd_cache(*a.values(), None)


@pytest.mark.parametrize("kw,status", _BAD_CACHES)
@pytest.mark.parametrize("call", [_write, _read, _attend])
def test_calls_on_a_cache_refuse_before_any_launch(call, kw, status):
    assert call(**kw) == status


@pytest.mark.parametrize("call,kw,status", [
    (_write, dict(k=None), 1), (_write, dict(v=None), 1), (_write, dict(T=0), 2), (_write, dict(T=1 << 30), 2), (_write, dict(dense=9), 3),
    (_write, dict(dense=binding.FA_FP8_E4M3), 4), (_write, dict(dense=binding.FA_F16), 4), (_write, dict(k=P + 8), 5),
    (_write, dict(counts=P + 2), 5), (_write, dict(kst=_longs(512, 192, 60)), 5), (_write, dict(vst=_longs(-8, 192, 64)), 2),
    (_read, dict(k=None), 1), (_read, dict(v=None), 1), (_read, dict(N=0), 2), (_read, dict(N=1 << 30), 2), (_read, dict(dense=-1), 3),
    (_read, dict(dense=binding.FA_FP8_E4M3), 4), (_read, dict(dense=binding.FA_F16), 4), (_read, dict(v=P + 4), 5),
    (_attend, dict(q=None), 1), (_attend, dict(o=None), 1), (_attend, dict(lse=None), 1), (_attend, dict(H=5), 2), (_attend, dict(H=0), 2),
    (_attend, dict(T=0), 2), (_attend, dict(T=257), 8), (_attend, dict(max_len=-1), 2), (_attend, dict(scale=0.0), 2),
    (_attend, dict(scale=NAN), 2), (_attend, dict(batches=3), 2), (_attend, dict(batches=0), 2), (_attend, dict(dense=binding.FA_F32), 4),
    (_attend, dict(dense=binding.FA_F16), 4), (_attend, dict(_CODES, dense=binding.FA_FP8_E4M3), 4), (_attend, dict(dense=5), 3),
    (_attend, dict(q=P + 2), 5), (_attend, dict(o=P + 8), 5), (_attend, dict(lse=P + 2), 5), (_attend, dict(tree=P + 2), 5),
    (_attend, dict(counts=P + 1), 5), (_attend, dict(qst=_longs(0, 100, 64)), 5), (_attend, dict(ost=_longs(0, 512, 64)), 2),
    (_attend, dict(B=1 << 14, H=1 << 12, T=64, batches=1), 2),
])
def test_each_call_refuses_what_is_its_own(call, kw, status):
    assert call(**kw) == status


def test_attention_over_a_cache_refuses_a_missing_or_small_workspace():
    B, H, H_kv, T, d, page, max_pages = 1, 4, 1, 1, 128, 64, 1024
    need = binding.fa_fwd_cache_workspace_bytes(B, H, H_kv, T, d, page * max_pages)
    call = lambda ws, n: _attend(B=B, H=H, H_kv=H_kv, T=T, d=d, page=page, max_pages=max_pages, tree=None, ws=ws, ws_bytes=n)  # noqa: E731
    if need:
        assert call(None, need) == 6 and call(P, need - 1) == 6 and call(P + 8, need) == 5
    for bad in (dict(B=0), dict(H=3), dict(H_kv=0), dict(T=0), dict(T=257), dict(d=96), dict(max_len=0), dict(code=binding.FA_F32)):
        a = dict(B=1, H=4, H_kv=2, T=1, d=64, max_len=100, code=binding.FA_BF16)
        a.update(bad)
        assert binding.fa_fwd_cache_workspace_bytes(*a.values()) == 0


@pytest.mark.parametrize("scaling,name,factor,trained", [
    (binding.FA_ROPE_PLAIN, "plain", 1.0, 0), (binding.FA_ROPE_LINEAR, "linear", 4.0, 0), (binding.FA_ROPE_NTK, "ntk", 8.0, 0),
    (binding.FA_ROPE_BY_PARTS, "by_parts", 4.0, 4096), (binding.FA_ROPE_BY_PARTS, "by_parts", 1.0, 2048)])
@pytest.mark.parametrize("rot,base", [(128, 10000.0), (64, 500000.0), (16, 10000.0)])
def test_frequencies_follow_the_formulas(scaling, name, factor, trained, rot, base):
    f, amplitude = binding.fa_rope_frequencies(rot, base, scaling, factor, trained, device="cpu")
    want, a = cache_oracle.frequencies(rot, base, name, factor, trained)
    assert f.dtype == torch.float64 and f.shape == (rot // 2,)
    np.testing.assert_allclose(f.numpy(), want, rtol=1e-13)  # pow and exp of 64 bits, exponents up to 13
    assert amplitude == pytest.approx(a, rel=2 ** -24)
    assert f[0] == (1.0 if name != "linear" else 1 / factor)  # the fastest pair, which by parts keeps
    if name == "by_parts" and factor > 1:  # the slowest is interpolated
        assert f[-1] == pytest.approx(base ** (-(rot - 2) / rot) / factor, rel=1e-12) or rot == 16


@pytest.mark.parametrize("a", [dict(rot=0), dict(rot=-2), dict(rot=7), dict(base=1.0), dict(base=NAN), dict(scaling=4), dict(scaling=-1),
                               dict(scaling=1, factor=0.5), dict(scaling=2, factor=NAN), dict(scaling=2, rot=2, factor=2.0),
                               dict(scaling=3, factor=2.0), dict(scaling=3, factor=2.0, trained=float("inf")),
                               dict(scaling=2, factor=1e300, base=1e300, rot=4)])
def test_frequencies_refuse_what_has_none(a):
    b = dict(rot=64, base=10000.0, scaling=0, factor=1.0, trained=0.0)
    b.update(a)
    with pytest.raises(binding.FaError) as e:
        binding.fa_rope_frequencies(*b.values(), device="cpu")
    assert e.value.status == 2
    assert binding.lib().fa_rope_frequencies(None, None, 64, 1e4, 0, 1.0, 0.0) == 1


@pytest.mark.parametrize("T", [1, 2, 31, 32, 33, 64, 100, 256])
def test_tree_words_hold_the_bits(T):
    g = torch.Generator().manual_seed(T)
    visible = torch.rand((2, T, T), generator=g) < 0.5
    words = binding.fa_tree_words(visible)
    assert words.dtype == torch.int32 and words.shape == (2, T, -(-T // 32))
    for b in range(2):
        for t in range(T):
            for u in range(T):
                assert bool((int(words[b, t, u // 32]) >> (u % 32)) & 1) == bool(visible[b, t, u])
    assert torch.equal(binding.fa_tree_words(visible[0]), words[0])


def test_the_binding_refuses_tensors_that_the_library_cannot_take():
    q = torch.zeros(1, 2, 3, 64)  # on the CPU
    pages, table, lens = torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16), torch.zeros(1, 2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    f = torch.zeros(32, dtype=torch.float64)
    for call in (lambda: binding.fa_rope(q, f), lambda: binding.fa_rope_bwd(q, f), lambda: binding.fa_rope(q[0], f),
                 lambda: binding.fa_cache_write(q, q, pages, pages, table, lens), lambda: binding.fa_cache_read(pages, pages, table, lens, 3),
                 lambda: binding.fa_cache_read(pages, pages, table, lens), lambda: binding.fa_cache_read(pages, pages, table, lens, 3, torch.int8),
                 lambda: binding.fa_fwd_cache(q, pages, pages, table, lens, 0.125), lambda: binding.fa_fwd_cache(q[0], pages, pages, table, lens, 0.125)):
        with pytest.raises((ValueError, RuntimeError)):  # (RuntimeError: no device to ask which is current)
            call()


def test_argument_validation_under_host_sanitizers(tmp_path):
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if not (os.path.exists(hipcc) or shutil.which(hipcc)):
        pytest.skip("hipcc not available")
    exe = str(tmp_path / "cache_api_san")
    cmd = [hipcc, "--offload-arch=gfx950", "-std=c++17", "-O1", "-g", "-Xarch_host", "-fsanitize=address", "-Xarch_host",
           "-fsanitize=undefined", "-Xarch_host", "-fno-sanitize-recover=all",
           os.path.join(ROOT, "paper_2407_08608_amd", "csrc", "fa_cache_api.hip"), os.path.join(SAN, "cache_api_driver.cpp"), "-o", exe,
           "-fsanitize=address", "-fsanitize=undefined"]
    subprocess.run(cmd, check=True, stderr=subprocess.DEVNULL)
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:exitcode=23", UBSAN_OPTIONS="halt_on_error=1:exitcode=24")
    r = subprocess.run([exe], env=env, capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stdout + r.stderr
    assert "cache api sanitizer run: 0 failures" in r.stdout


# ---- the oracle: closed forms and an independent way


def test_oracle_rope_is_a_rotation_that_its_transpose_undoes():
    g = np.random.default_rng(1)
    x, pos = g.standard_normal((2, 3, 5, 64)), g.integers(-5, 1000, (2, 5))
    f, _ = cache_oracle.frequencies(32, 10000.0)
    for interleaved in (False, True):
        y = cache_oracle.rope(x, f, pos, 32, interleaved)
        np.testing.assert_allclose((y ** 2).sum(-1), (x ** 2).sum(-1), rtol=1e-12)
        np.testing.assert_array_equal(y[..., 32:], x[..., 32:])
        np.testing.assert_allclose(cache_oracle.rope(y, f, pos, 32, interleaved, transposed=True), x, atol=1e-12)
        # the product of two rotated rows goes by the difference of their positions
        z = cache_oracle.rope(x, f, pos + 77, 32, interleaved)
        w = cache_oracle.rope(x, f, np.full_like(pos, 77), 32, interleaved)
        np.testing.assert_allclose((y * z).sum(-1), (cache_oracle.rope(x, f, 0 * pos, 32, interleaved) * w).sum(-1), rtol=1e-9)
    # one pair by hand: position 1, frequency 1
    e = np.zeros((1, 1, 1, 64))
    e[..., 0] = 1.0
    y = cache_oracle.rope(e, f, np.ones((1, 1)), 32, False, amplitude=2.0)
    assert y[0, 0, 0, 0] == pytest.approx(2 * math.cos(1)) and y[0, 0, 0, 16] == pytest.approx(2 * math.sin(1))


def test_oracle_rows_are_quantised_as_blocks_of_one_row():
    g = np.random.default_rng(2)
    x = g.standard_normal((1, 2, 6, 64)).astype(np.float32)
    codes, scales = cache_oracle.quantise_rows(x)
    want, s = fp8_oracle.quantize(x, None, 1)
    np.testing.assert_array_equal(codes, want)
    np.testing.assert_array_equal(scales, np.asarray(s, dtype=np.float32).reshape(scales.shape))
    x[0, 0, 0, :2], x[0, 0, 1] = (np.inf, -np.nan), 0.0
    codes, scales = cache_oracle.quantise_rows(x)
    assert fp8_oracle.e4m3_decode(codes)[0, 0, 0, 0] == 448 and np.isnan(fp8_oracle.e4m3_decode(codes)[0, 0, 0, 1])
    assert scales[0, 0, 1] == 1 and (codes[0, 0, 1] == 0).all() and np.isfinite(scales).all()


def test_oracle_attention_over_a_cache_is_dense_attention():
    # a causal sequence of 40 tokens, the last 7 of them as new ones, through pages in any order
    g = np.random.default_rng(3)
    q, k, v = (g.standard_normal((1, h, 40, 64)) for h in (4, 2, 2))
    o, lse = oracle.attention_fwd_gqa(q, k, v, 0.125, True)
    table = np.array([[4, 0, 2]])
    cache = {"block_table": table, "k_pages": np.full((5, 2, 16, 64), np.nan), "v_pages": np.full((5, 2, 16, 64), np.nan)}
    for p in range(40):
        cache["k_pages"][table[0, p // 16], :, p % 16], cache["v_pages"][table[0, p // 16], :, p % 16] = k[0, :, p], v[0, :, p]
    got = cache_oracle.attend(q[:, :, 33:], cache, [33], [7], None, 0.125)
    tree = np.tril(np.ones((1, 7, 7), dtype=bool))
    as_tree = cache_oracle.attend(q[:, :, 33:], cache, [33], [7], tree, 0.125)
    for h in range(4):
        for t in range(7):
            np.testing.assert_allclose(got[0, h, t][0], o[0, h, 33 + t], rtol=1e-10, atol=1e-12)
            assert got[0, h, t][1] == pytest.approx(lse[0, h, 33 + t], rel=1e-12)
            np.testing.assert_array_equal(got[0, h, t][0], as_tree[0, h, t][0])
    empty = cache_oracle.attend(q[:, :, :1], cache, [0], [1], np.zeros((1, 1, 1), dtype=bool), 0.125)
    assert empty[0, 0, 0][1] == -np.inf and (empty[0, 0, 0][0] == 0).all()
