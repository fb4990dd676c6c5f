"""fa_cache_write and fa_cache_read: bit for bit what the definitions give, nothing else touched."""
import numpy as np
import pytest
import torch

from helpers import f64
from oracle import cache_oracle, fp8_oracle
from paper_2407_08608_amd import binding, inputs

pytestmark = pytest.mark.gpu

_T = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def make_cache(seed, n_pages, H_kv, page, d, cache):
    """Pages full of earlier values: (k_pages, v_pages, k_scales, v_scales)"""
    g = torch.Generator(device="cuda").manual_seed(seed)
    if cache != "e4m3":
        return tuple(torch.randn((n_pages, H_kv, page, d), generator=g, device="cuda").to(_T[cache]) for _ in range(2)) + (None, None)
    pages = tuple(torch.randint(0, 127, (n_pages, H_kv, page, d), generator=g, device="cuda", dtype=torch.uint8) for _ in range(2))
    return pages + tuple(torch.rand((n_pages, H_kv, page), generator=g, device="cuda") + 0.01 for _ in range(2))


def make_table(seed, B, max_pages, n_pages):
    return torch.from_numpy(np.random.default_rng(seed).permutation(n_pages)[:B * max_pages].reshape(B, max_pages).astype(np.int32))


def expected_write(x, pages, scales, table, lens, counts, page):
    """The pages (and scales) after x [B,H_kv,T,d] has been written, in numpy"""
    pages, scales = pages.clone(), None if scales is None else scales.clone()
    codes, s = (torch.from_numpy(a) for a in cache_oracle.quantise_rows(x.float().cpu().numpy()))
    places = {"k_pages": pages, "block_table": table.numpy()}
    for b in range(x.shape[0]):
        for t in range(min(int(counts[b]), x.shape[2])):
            at = cache_oracle.place(places, b, max(int(lens[b]), 0) + t)
            if at is None:
                continue
            if scales is None:
                pages[at[0], :, at[1]] = x[b, :, t].to(pages.dtype)
            else:
                pages[at[0], :, at[1]] = codes[b, :, t].to(pages.device)
                scales[at[0], :, at[1]] = s[b, :, t].to(pages.device)
    return pages, scales


@pytest.mark.parametrize("dense,cache", [("bf16", "bf16"), ("f16", "f16"), ("f32", "bf16"), ("f32", "f16"), ("bf16", "e4m3"), ("f16", "e4m3"),
                                         ("f32", "e4m3")])
@pytest.mark.parametrize("B,H_kv,T,d,page,max_pages", [(1, 1, 1, 64, 16, 1), (3, 2, 1, 128, 16, 5), (2, 3, 37, 256, 48, 3), (4, 5, 70, 64, 32, 4),
                                                       (2, 1, 19, 128, 16, 9)])
def test_write(dense, cache, B, H_kv, T, d, page, max_pages):
    n_pages = B * max_pages + 2
    kp, vp, ks, vs = make_cache(B + T, n_pages, H_kv, page, d, cache)
    table = make_table(T, B, max_pages, n_pages)
    room = max_pages * page - T
    rng = np.random.default_rng(d + T)
    lens = torch.from_numpy(rng.integers(0, max(room, 0) + 1, B).astype(np.int32))
    counts = torch.from_numpy(rng.integers(0, T + 1, B).astype(np.int32))
    counts[0] = T
    k, v = (inputs.heavy_tailed_tensor(3, n, (B, H_kv, T, d), dense, p_outlier=0.05).cuda() for n in ("k", "v"))
    k[0, 0, 0] = 0
    for n in (None, counts):
        have = [None if t is None else t.clone() for t in (kp, vp, ks, vs)]
        got = binding.fa_cache_write(k, v, have[0], have[1], table.cuda(), lens.cuda(), counts=None if n is None else n.cuda(), k_scales=have[2],
                                     v_scales=have[3])
        assert got[0] is have[0] and got[1] is have[1]
        full = torch.full((B,), T) if n is None else n
        for x, pages, scales, a, s in ((k, kp, ks, have[0], have[2]), (v, vp, vs, have[1], have[3])):
            want, want_s = expected_write(x, pages, scales, table, lens, full, page)
            assert torch.equal(a.view(torch.uint8), want.view(torch.uint8))
            assert s is None or torch.equal(s, want_s)


def test_write_from_strided_rows_and_past_every_end():
    B, H_kv, T, d, page, max_pages, n_pages = 4, 2, 5, 64, 16, 2, 6
    kp, vp, ks, vs = make_cache(1, n_pages, H_kv, page, d, "e4m3")
    # one sequence ends in the middle of its new tokens, one has a page that is none, one is beyond its end already, one "negative"
    table = torch.tensor([[0, 1], [-1, 6], [2, 3], [4, 2 ** 31 - 1]], dtype=torch.int32)
    lens = torch.tensor([30, 14, 32, -7], dtype=torch.int32)
    counts = torch.tensor([5, 5, 5, 9], dtype=torch.int32)
    x = inputs.normal_tensor(2, "kv", (B, T, 2, H_kv, d), "bf16").cuda()
    k, v = x[:, :, 0].transpose(1, 2), x[:, :, 1].transpose(1, 2)
    have = [t.clone() for t in (kp, vp, ks, vs)]
    binding.fa_cache_write(k, v, *have[:2], table.cuda(), lens.cuda(), counts=counts.cuda(), k_scales=have[2], v_scales=have[3])
    for t, pages, scales, a, s in ((k, kp, ks, have[0], have[2]), (v, vp, vs, have[1], have[3])):
        want, want_s = expected_write(t, pages, scales, table, lens, counts, page)
        assert torch.equal(a, want) and torch.equal(s, want_s)
    # lengths near the largest int
    lens = torch.full((B,), 2 ** 31 - 1, dtype=torch.int32)
    again = [t.clone() for t in have]
    binding.fa_cache_write(k, v, *again[:2], table.cuda(), lens.cuda(), k_scales=again[2], v_scales=again[3])
    assert all(torch.equal(a, b) for a, b in zip(again, have))


def test_special_values_in_a_quantised_row():
    d = 128
    k = torch.zeros((1, 1, 8, d), dtype=torch.float32)
    k[0, 0, 0] = torch.linspace(-3, 3, d)
    k[0, 0, 0, 5], k[0, 0, 0, 6], k[0, 0, 0, 7] = float("inf"), float("-inf"), float("nan")
    k[0, 0, 1, :3] = torch.tensor([float("inf"), float("nan"), float("-inf")])  # nothing finite but zeros
    k[0, 0, 2] = 2.0 ** -140  # below what 448 / a could take
    k[0, 0, 3, 9] = 3e38
    k[0, 0, 4] = torch.linspace(0, 2.0 ** -100, d)
    k[0, 0, 5] = -0.0
    k[0, 0, 6] = 448.0 / 449.0 * torch.linspace(-1, 1, d)
    pages = torch.zeros((1, 1, 16, d), dtype=torch.uint8, device="cuda")
    scales = torch.zeros((1, 1, 16), device="cuda")
    kp, vp, ks, vs = pages.clone(), pages.clone(), scales.clone(), scales.clone()
    zero = torch.zeros((1,), dtype=torch.int32, device="cuda")
    binding.fa_cache_write(k.cuda(), k.cuda(), kp, vp, zero[:, None], zero, k_scales=ks, v_scales=vs)
    codes, s = cache_oracle.quantise_rows(k.numpy())
    got = fp8_oracle.e4m3_decode(kp[0, 0, :8].cpu().numpy())
    np.testing.assert_array_equal(got, fp8_oracle.e4m3_decode(codes)[0, 0])
    np.testing.assert_array_equal(ks[0, 0, :8].cpu().numpy(), s[0, 0])
    assert got[0, 5] == 448 and got[0, 6] == -448 and np.isnan(got[0, 7]) and np.isfinite(s).all() and (s > 0).all()
    assert torch.equal(kp, vp) and torch.equal(ks, vs)


@pytest.mark.parametrize("cache,dense", [("bf16", "bf16"), ("f16", "f16"), ("bf16", "f32"), ("f16", "f32"), ("e4m3", "bf16"), ("e4m3", "f16"),
                                         ("e4m3", "f32")])
@pytest.mark.parametrize("B,H_kv,N,d,page,max_pages", [(1, 1, 1, 64, 16, 1), (3, 2, 70, 128, 16, 5), (2, 3, 100, 256, 48, 3), (4, 5, 33, 64, 32, 2)])
def test_read(cache, dense, B, H_kv, N, d, page, max_pages):
    n_pages = B * max_pages + 2
    kp, vp, ks, vs = make_cache(N, n_pages, H_kv, page, d, cache)
    table = make_table(N, B, max_pages, n_pages)
    table[B - 1, max_pages - 1] = -1
    lens = torch.from_numpy(np.random.default_rng(N).integers(0, max_pages * page + 5, B).astype(np.int32))
    lens[0] = min(N, max_pages * page)
    if B > 2:
        lens[1] = -3
    out = [torch.full((B, H_kv, N, d), -7.0, device="cuda", dtype=_T[dense]) for _ in range(2)]
    got = binding.fa_cache_read(kp, vp, table.cuda(), lens.cuda(), k_scales=ks, v_scales=vs, k=out[0], v=out[1])
    assert got[0] is out[0] and got[1] is out[1]
    for pages, scales, y in ((kp, ks, out[0]), (vp, vs, out[1])):
        x = pages.float() if scales is None else pages.view(torch.float8_e4m3fn).float() * scales[..., None]
        x = x.to(_T[dense])
        want = torch.full_like(y, -7.0)
        for b in range(B):
            for n in range(min(N, max(int(lens[b]), 0))):
                at = cache_oracle.place({"k_pages": pages, "block_table": table.numpy()}, b, n)
                if at is not None:
                    want[b, :, n] = x[at[0], :, at[1]]
        assert torch.equal(y, want)
    fresh = binding.fa_cache_read(kp, vp, table.cuda(), lens.cuda(), N, _T[dense], k_scales=ks, v_scales=vs)
    assert fresh[0].dtype == _T[dense]
    if table[0, 0] >= 0:  # (rows of what is no page hold whatever was in the memory)
        n = min(int(lens[0]), page)
        assert torch.equal(fresh[0][0, :, :n], out[0][0, :, :n]) and torch.equal(fresh[1][0, :, :n], out[1][0, :, :n])


def test_a_prompt_written_and_read_back_is_itself():
    # 16-bit: exactly; e4m3: half a step of a code, 2^-4 of the value, or of the smallest normal code's step, 2^-10 of a / 448, and the rounding to bf16
    B, H_kv, T, d, page = 2, 4, 1000, 128, 64
    k, v = (inputs.heavy_tailed_tensor(4, n, (B, H_kv, T, d), "bf16").cuda() for n in ("k", "v"))
    table = torch.arange(B * 16, dtype=torch.int32, device="cuda").view(B, 16)
    zero, full = torch.zeros(B, dtype=torch.int32, device="cuda"), torch.full((B,), T, dtype=torch.int32, device="cuda")
    kp, vp = (torch.empty((B * 16, H_kv, page, d), device="cuda", dtype=torch.bfloat16) for _ in range(2))
    binding.fa_cache_write(k, v, kp, vp, table, zero)
    got = binding.fa_cache_read(kp, vp, table, full, T)
    assert torch.equal(got[0], k) and torch.equal(got[1], v)
    kp, vp = (torch.empty((B * 16, H_kv, page, d), device="cuda", dtype=torch.float8_e4m3fn) for _ in range(2))
    ks, vs = (torch.empty((B * 16, H_kv, page), device="cuda") for _ in range(2))
    binding.fa_cache_write(k, v, kp, vp, table, zero, k_scales=ks, v_scales=vs)
    got = binding.fa_cache_read(kp, vp, table, full, T, k_scales=ks, v_scales=vs)
    for x, y in zip((k, v), got):
        x, y = f64(x), f64(y)
        a = np.abs(x).max(-1, keepdims=True)
        assert (np.abs(y - x) <= np.maximum(2.0 ** -4 * np.abs(x), 2.0 ** -10 * a / 448) * (1 + 2 ** -7) + 2.0 ** -8 * np.abs(x)).all()


def test_slots_past_32_bits():
    # 4.3 GB of codes to a tensor: the last page lies beyond 2^32 bytes
    H_kv, page, d = 8, 1024, 256
    n_pages = 2 ** 32 // (H_kv * page * d) + 3
    kp = torch.zeros((n_pages, H_kv, page, d), dtype=torch.uint8, device="cuda")
    vp, ks, vs = torch.zeros_like(kp), torch.zeros((n_pages, H_kv, page), device="cuda"), torch.zeros((n_pages, H_kv, page), device="cuda")
    k, v = (inputs.normal_tensor(5, n, (1, H_kv, 3, d), "bf16").cuda() for n in ("k", "v"))
    table = torch.tensor([[0, n_pages - 1]], dtype=torch.int32, device="cuda")
    lens = torch.tensor([page + 5], dtype=torch.int32, device="cuda")
    binding.fa_cache_write(k, v, kp, vp, table, lens, k_scales=ks, v_scales=vs)
    codes, scales = cache_oracle.quantise_rows(k.float().cpu().numpy())
    np.testing.assert_array_equal(kp[-1, :, 5:8].cpu().numpy(), codes[0])
    assert int((kp != 0).sum()) == int((codes != 0).sum())
    y = binding.fa_cache_read(kp, vp, table, lens + 3, page + 8, torch.float32, k_scales=ks, v_scales=vs)
    want = torch.from_numpy(fp8_oracle.e4m3_decode(codes).astype(np.float32) * scales[..., None])
    assert torch.equal(y[0][:, :, page + 5:].cpu(), want)


def test_the_binding_refuses_what_does_not_fit():
    kp, vp, ks, vs = make_cache(1, 4, 2, 16, 64, "e4m3")
    b16 = kp.to(torch.bfloat16)
    k = torch.zeros((2, 2, 3, 64), device="cuda", dtype=torch.bfloat16)
    table, lens = torch.zeros((2, 2), dtype=torch.int32, device="cuda"), torch.zeros((2,), dtype=torch.int32, device="cuda")
    ok = dict(k=k, v=k, k_pages=kp, v_pages=vp, block_table=table, lens=lens, counts=lens, k_scales=ks, v_scales=vs)
    binding.fa_cache_write(**ok)
    for kw in (dict(v=k[:, :1]), dict(v=k.float()), dict(k=k.double(), v=k.double()), dict(k_pages=kp[:2]), dict(v_pages=b16), dict(k_scales=None),
               dict(k_scales=ks[:2]), dict(k_pages=b16, v_pages=b16), dict(block_table=table.long()), dict(block_table=table[0]),
               dict(lens=lens[:1]), dict(counts=lens.float()), dict(k_pages=kp.transpose(1, 2)), dict(k_pages=kp[..., :32]), dict(lens=lens.cpu()),
               dict(k_pages=kp.int(), v_pages=vp.int())):
        with pytest.raises(ValueError):
            binding.fa_cache_write(**dict(ok, **kw))
    ok = dict(k_pages=kp, v_pages=vp, block_table=table, lens=lens, N=3, k_scales=ks, v_scales=vs)
    binding.fa_cache_read(**ok)
    for kw in (dict(N=None), dict(dtype=torch.int32), dict(k=k.transpose(0, 1)), dict(k=k.float(), v=k), dict(k=k, N=4), dict(v_scales=None)):
        with pytest.raises(ValueError):
            binding.fa_cache_read(**dict(ok, **kw))
    with pytest.raises(binding.FaError):
        binding.fa_cache_read(**dict(ok, N=0))
    with pytest.raises(binding.FaError):  # bf16 pages as fp16
        binding.fa_cache_read(b16, b16, table, lens, 3, torch.float16)
