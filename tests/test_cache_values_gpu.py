"""fa_fwd_cache where the values and scales of some places are nothing like the others': what a row does not see, or hardly weighs, or
what is zero, leaves the row's other weights as they are.  Every form of the kernel, in one launch and joined.

The bound of a row is the one of test_fwd_cache_gpu.py without its terms in the largest |v|: all errors are in proportion to sum w |v|.
With codes the weights (times the scale of V) go to their product in two bf16 numbers, which leaves 2^-16 of each: half a step, 2^-8, of
what half a step, 2^-8, of the weight left over; and an fp32 product, 2^-24."""
import numpy as np
import pytest
import torch

from helpers import f64
from oracle import cache_oracle
from paper_2407_08608_amd import binding, inputs
from test_fwd_cache_gpu import _HALF, _T, Case, _random_tree

pytestmark = pytest.mark.gpu

# d, H, H_kv, T: up to 16, 32 and 64 rows to a key/value head, and more
_FORMS = [(64, 8, 4, 3), (128, 4, 2, 2), (256, 4, 2, 3), (128, 8, 2, 6), (64, 8, 2, 12), (128, 8, 2, 12), (256, 8, 2, 12), (64, 4, 1, 20),
          (128, 8, 2, 40), (256, 4, 1, 30)]


def _check(c, o, lse, rows=None):
    """Every row (of new tokens `rows`) within the bound of sum w |v|; what the output's type cannot hold is infinite there"""
    q, half = f64(c.q), _HALF[c.dtype]
    want = cache_oracle.attend(q, c.host, c.lens, c.counts, c.tree, c.scale)
    o, lse, d, top_o = f64(o), f64(lse), q.shape[-1], float(torch.finfo(_T[c.dtype]).max)
    for (b, h, t), (x, L, K, V) in want.items():
        if rows is not None and t not in rows:
            continue
        s = c.scale * (K @ q[b, h, t])
        top = np.abs(s).max()
        e_s = (d + 4) * 2.0 ** -24 * c.scale * (np.abs(K) @ np.abs(q[b, h, t])).max() + 2.0 ** -23 * top
        e_w = 2 * (e_s + 2.0 ** -22 * top + 2.0 ** -21)
        size = np.exp(s - L) @ np.abs(V)
        bound = (e_w + 2.0 ** -16 + 2.0 ** -24 + len(K) * 2.0 ** -24) * size + half * np.abs(x) + (2.0 ** -25 if c.dtype == "f16" else 2.0 ** -134)
        fits = np.abs(x) + bound < top_o
        err = np.abs(o[b, h, t] - x)
        assert (err[fits] <= bound[fits]).all(), ((b, h, t), err[fits].max(), bound[fits][np.argmax((err - bound)[fits])])
        assert abs(lse[b, h, t] - L) <= e_s + 2.0 ** -22 * top + 2.0 ** -20 + 2.0 ** -23 * abs(L), ((b, h, t), lse[b, h, t], L)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d,H,H_kv,T", _FORMS)
@pytest.mark.parametrize("max_len", [0, 1 << 20])
@pytest.mark.parametrize("chain", [True, False])
def test_a_scale_that_a_row_does_not_see(dtype, d, H, H_kv, T, max_len, chain):
    tree = None if chain else _random_tree(T, 2, T)
    c = Case(700 + T, dtype, "e4m3", 2, H, H_kv, T, d, 16, [300, 21], tree=tree)
    clean = c.run(max_len=max_len)
    _check(c, *clean)
    u = T // 2
    slots = [cache_oracle.place(c.host, b, int(c.lens[b]) + u) for b in range(2)]
    for factor in (2.0 ** 12, 2.0 ** 20, 2.0 ** 30, 2.0 ** 100, -2.0 ** 30, 0.0):
        scales = c.args["v_scales"].clone()
        for page, slot in slots:
            scales[page, :, slot] *= factor
        got = c.run(v_scales=scales, max_len=max_len)
        for b in range(2):
            for t in range(T):
                if u > t if chain else not tree[b, t, u]:
                    assert torch.equal(got[0][b, :, t], clean[0][b, :, t]) and torch.equal(got[1][b, :, t], clean[1][b, :, t]), (factor, b, t)
        was, c.host["v_scales"] = c.host["v_scales"], scales.cpu().numpy()
        _check(c, *got)
        c.host["v_scales"] = was


def _written(dtype, B, H, H_kv, T, d, n, k, v, seed):
    """A Case whose cache fa_cache_write filled with k, v [B,H_kv,n+T,d]: n tokens, and T new ones behind them"""
    page = 16
    c = Case(seed, dtype, "e4m3", B, H, H_kv, T, d, page, [n] * B)
    names = ("k_pages", "v_pages", "k_scales", "v_scales")
    binding.fa_cache_write(k, v, c.args["k_pages"], c.args["v_pages"], c.args["block_table"], torch.zeros(B, dtype=torch.int32, device="cuda"),
                           k_scales=c.args["k_scales"], v_scales=c.args["v_scales"])
    c.host.update({x: c.args[x].cpu().numpy() for x in names})
    return c


@pytest.mark.parametrize("dtype,size", [("bf16", 1e-2), ("bf16", 1e-5), ("bf16", 1e-20), ("bf16", 2.0 ** -99), ("f16", 1e-2), ("f16", 1e-4)])
@pytest.mark.parametrize("d,H,H_kv,T", [(64, 8, 4, 1), (128, 16, 2, 1), (256, 4, 1, 1)] + _FORMS)
def test_a_value_of_zeros_among_small_ones(dtype, size, d, H, H_kv, T):
    # (a row of zeros is written with the scale 1)
    B, n = 2, 75
    k, v = (inputs.normal_tensor(31, x, (B, H_kv, n + T, d), "f32").cuda() for x in ("k", "v"))
    v *= size
    v[:, :, 3] = v[:, :, n] = 0
    v[1, :, 50] = 0
    c = _written(dtype, B, H, H_kv, T, d, n, k, v, 800 + T)
    for max_len in (0, 1 << 20):
        _check(c, *c.run(max_len=max_len))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d,H,H_kv,T", [(64, 8, 4, 1), (128, 16, 2, 1), (256, 4, 1, 1)] + _FORMS)
def test_large_values_that_hardly_count(dtype, d, H, H_kv, T):
    # one token of 2^18 times the others' values, with a score 20 below the largest: weight x value is 2^-11 of the others'
    B, n = 2, 200
    k, v = (inputs.normal_tensor(32, x, (B, H_kv, n + T, d), "f32").cuda() for x in ("k", "v"))
    v *= 2.0 ** -10
    v[:, :, 40] *= 2.0 ** 18
    c = _written(dtype, B, H, H_kv, T, d, n, k, v, 900 + T)
    k[:, :, 40] = 0
    for b in range(B):
        for g in range(H_kv):
            q = c.q[b, g * (H // H_kv)].double().mean(0)
            k[b, g, 40] = (-20 * d ** 0.5 / float(q @ q) * q).float().cuda()
    c = _written(dtype, B, H, H_kv, T, d, n, k, v, 900 + T)
    for max_len in (0, 1 << 20):
        _check(c, *c.run(max_len=max_len))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d,H,H_kv,T", [(64, 8, 4, 1), (128, 16, 2, 1), (256, 4, 1, 1)] + _FORMS)
def test_scales_of_either_sign(dtype, d, H, H_kv, T):
    # a cached value is code * scale, whatever the scale
    c = Case(950 + T, dtype, "e4m3", 2, H, H_kv, T, d, 16, [90, 33])
    for sign in ("negative", "mixed"):
        for x in ("k_scales", "v_scales"):
            s = np.abs(c.host[x])
            s = -s if sign == "negative" else s * np.random.default_rng(len(x) + T).choice([-1.0, 1.0], s.shape).astype(np.float32)
            if sign == "mixed" and x == "v_scales":
                s = np.where(s < 0, s * np.float32(64), s)
            c.host[x], c.args[x] = s, torch.from_numpy(s).cuda()
        for max_len in (0, 1 << 20):
            _check(c, *c.run(max_len=max_len))


@pytest.mark.parametrize("dtype,cache", [("bf16", "bf16"), ("f16", "f16"), ("bf16", "e4m3"), ("f16", "e4m3")])
@pytest.mark.parametrize("d,H,H_kv,T", [(64, 8, 4, 1), (128, 16, 2, 1), (256, 4, 1, 1)] + _FORMS)
@pytest.mark.parametrize("max_len", [0, 1 << 20])
def test_values_of_old_tokens_that_are_not_finite(dtype, cache, d, H, H_kv, T, max_len):
    # every row sees them: beside the new tokens in their tile of 32 keys (100 is 96 + 4), and far from them
    B, n = 2, 100
    c = Case(970 + T, dtype, cache, B, H, H_kv, T, d, 16, [n, n - 3], tree=_random_tree(T, B, T) if T > 1 else None)
    for b, p, col, x in ((0, 96, 3, np.nan), (0, 99, 17, np.inf), (1, 96, 40, -np.inf), (1, 5, 41, np.nan), (1, 40, 42, np.inf)):
        page, slot = cache_oracle.place(c.host, b, p)
        x = 0x7F if cache == "e4m3" else float(x)
        c.args["v_pages"][page, :, slot, col] = x
        c.host["v_pages"][page, :, slot, col] = x
    o, lse = c.run(max_len=max_len)
    o64 = f64(o)
    bad = [(0, 3), (0, 17), (1, 40), (1, 41), (1, 42)]
    for b, col in bad:
        assert not np.isfinite(o64[b, :, :, col]).any(), (b, col)
        if cache != "e4m3" and col in (17, 40):
            assert (o64[b, :, :, col] == (np.inf if col == 17 else -np.inf)).all()
    # the other columns as with zeros there
    fine = [i for i in range(d) if i not in {col for _, col in bad}]
    clean = dict(c.args, v_pages=c.args["v_pages"].clone())
    for b, p, col in ((0, 96, 3), (0, 99, 17), (1, 96, 40), (1, 5, 41), (1, 40, 42)):
        page, slot = cache_oracle.place(c.host, b, p)
        clean["v_pages"][page, :, slot, col] = 0
    want = c.run(max_len=max_len, **clean)
    assert torch.equal(o[..., fine], want[0][..., fine]) and torch.equal(lse, want[1])
