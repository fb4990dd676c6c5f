"""The native and the Python way through the binding of rotary positions with several axes, pages and the 4-bit cache: the same results,
refusals and errors."""
import pytest
import torch

from paper_2407_08608_amd import binding
from test_binding import _both, _same_error

needs_native = pytest.mark.skipif(binding._native is None, reason="the native part has not been built")


def _ints(*x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _same(native, python):
    assert type(native) is tuple and type(python) is tuple and len(native) == len(python), (native, python)
    for a, b in zip(native, python):
        assert (a is None) == (b is None)
        if a is not None:
            assert type(a) is torch.Tensor and a.dtype == b.dtype and a.device == b.device and a.shape == b.shape and a.stride() == b.stride()
            assert torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))


def test_arguments_that_no_way_takes(monkeypatch):
    x, i = torch.zeros(1, 2, 16, 64), torch.zeros(1, dtype=torch.int32)
    for bad in (x, x[0], None, "q", 3):
        for call in (lambda: binding.fa_rope_axes(bad, x, i, i), lambda: binding.fa_rope_axes_bwd(x, x, bad, i), lambda: binding.fa_cache_fork(bad, i, i, 16, 4),
                     lambda: binding.fa_cache_fork(i[None], i, bad, 16, 4), lambda: binding.fa_cache_fork(i[None], i, i, 16, 4, held=bad),
                     lambda: binding.fa_cache_extend(bad, i, 1, 16, 4), lambda: binding.fa_cache_compact(bad, 4), lambda: binding.fa_cache_copy(bad, x, i, i),
                     lambda: binding.fa_cache_copy(x, x, bad, i), lambda: binding.fa_cache_copy(x.byte(), x.byte(), i, i, k_scales=bad, v_scales=x.byte())):
            _same_error(*_both(monkeypatch, call))


@pytest.mark.gpu
@needs_native
def test_both_ways_give_the_same(monkeypatch):
    g = torch.Generator(device="cuda").manual_seed(3)
    q, k = (torch.randn((2, h, 5, 64), generator=g, device="cuda").bfloat16() for h in (4, 2))
    f, _ = binding.fa_rope_frequencies(64)
    axis, at = (torch.arange(32, device="cuda") % 3).int(), torch.arange(30, dtype=torch.int32, device="cuda").view(3, 2, 5)
    table, lens, parents, held = _ints([3, 5, 1, -1], [2, 0, 4, 6]), _ints(40, 17), _ints(0, 1, 0, -1, 1), _ints(*([0] * 7 + [1, 0, 0, 0]))
    codes = [torch.randint(0, 256, (11, 2, 16, 32), generator=g, device="cuda", dtype=torch.uint8) for _ in range(2)]
    powers = [torch.randint(120, 130, (11, 2, 16, 2), generator=g, device="cuda", dtype=torch.uint8) for _ in range(2)]
    typed = [t.view(torch.float4_e2m1fn_x2) for t in codes], [t.view(torch.float8_e8m0fnu) for t in powers]
    space = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")

    def copied(pages, scales):
        have = [t.clone() for t in pages + scales]
        binding.fa_cache_copy(have[0], have[1], _ints(3, -1, 5), _ints(8, 9, 10), k_scales=have[2], v_scales=have[3])
        return tuple(have)

    def written(pages, scales):
        have = [t.clone() for t in pages + scales]
        binding.fa_cache_write(k, k, have[0], have[1], table, lens, k_scales=have[2], v_scales=have[3])
        return tuple(have)

    calls = [lambda: binding.fa_rope_axes(q, f, axis, at, k=k), lambda: binding.fa_rope_axes_bwd(q, f, axis, at, interleaved=True, amplitude=1.5),
             lambda: binding.fa_rope_axes(q.transpose(1, 2).contiguous().transpose(1, 2), f[:16].contiguous(), axis[:16].contiguous(), at, rot_dim=32),
             lambda: binding.fa_cache_fork(table, lens, parents, 16, 11), lambda: binding.fa_cache_fork(table, lens, parents, 16, 9000, held=torch.zeros(9000, dtype=torch.int32, device="cuda")),
             lambda: binding.fa_cache_fork(table, lens, parents, 16, 11, held=held, src=_ints(*[7] * 5), missing=_ints(3), workspace=space),
             lambda: binding.fa_cache_extend(table.clone(), lens, 20, 16, 11, held=held), lambda: binding.fa_cache_extend(table.clone(), lens, 20, 16, 11, counts=_ints(9, 20), missing=_ints(3)),
             lambda: binding.fa_cache_compact(table, 11), lambda: binding.fa_cache_compact(table, 9000, moves=3, workspace=space), lambda: binding.fa_cache_compact(table, 11, held=held, dst=_ints(1, 2), moves=2)]
    for pages, scales in ((codes, powers), typed):
        s = dict(k_scales=scales[0], v_scales=scales[1])
        calls += [lambda p=pages, s=scales: copied(p, s), lambda p=pages, s=scales: written(p, s), lambda p=pages, s=s: binding.fa_cache_read(p[0], p[1], table, lens, 16, **s),
                  lambda p=pages, s=s: binding.fa_fwd_cache(q, p[0], p[1], table, lens, 0.125, **s)]
    for call in calls:
        _same(*_both(monkeypatch, call))


@pytest.mark.gpu
def test_both_ways_refuse_the_same(monkeypatch):
    q, f = torch.zeros((2, 4, 5, 64), dtype=torch.bfloat16, device="cuda"), torch.zeros(32, dtype=torch.float64, device="cuda")
    axis, at = torch.zeros(32, dtype=torch.int32, device="cuda"), torch.zeros((3, 2, 5), dtype=torch.int32, device="cuda")
    t, lens, p = _ints([0, 1], [2, 3]), _ints(1, 2), _ints(0, 1, 1)
    c, s = torch.zeros((4, 1, 16, 32), dtype=torch.uint8, device="cuda"), torch.zeros((4, 1, 16, 2), dtype=torch.uint8, device="cuda")
    A, F = binding.fa_rope_axes, binding.fa_cache_fork
    for call in (lambda: A(q, f, axis[:3], at), lambda: A(q, f, axis, at[0]), lambda: A(q, f, axis.long(), at), lambda: A(q, f, axis, at[:, :1]), lambda: A(q, f, axis, at[:0]),
                 lambda: A(q, f, axis.cpu(), at), lambda: A(q, f, axis, at, rot_dim="x"), lambda: A(q, f, axis, at, amplitude=-1.0), lambda: A(q, f, axis, at, k=q.float()),
                 lambda: F(t, lens, p, 16, 9, held=p), lambda: F(t, lens, p, "x", 9), lambda: F(t, lens, p, -1, 9), lambda: F(t, lens[:1], p, 16, 9), lambda: F(t[0], lens, p, 16, 9),
                 lambda: F(t, lens, p, 16, 9, new_lens=lens), lambda: F(t, lens, p, 16, 9, workspace=t), lambda: F(t, lens, p, 16, 5000, workspace=c.view(-1)),
                 lambda: binding.fa_cache_extend(t, lens, 1, 16, 9, counts=p), lambda: binding.fa_cache_extend(t, lens, -1, 16, 9), lambda: binding.fa_cache_extend(t, lens, "1", "x", 9),
                 lambda: binding.fa_cache_extend(t, lens, 1, 16, 9, missing=p), lambda: binding.fa_cache_compact(t, -1), lambda: binding.fa_cache_compact(t, 9, moves=0),
                 lambda: binding.fa_cache_compact(t, 9, src=lens), lambda: binding.fa_cache_compact(t, 9, top=lens), lambda: binding.fa_cache_copy(c, c, p, p, k_scales=s),
                 lambda: binding.fa_cache_copy(c, c, p, p, k_scales=s, v_scales=s.float()), lambda: binding.fa_cache_copy(c, c, p, lens, k_scales=s, v_scales=s),
                 lambda: binding.fa_cache_copy(c[:, :, :8].contiguous(), c[:, :, :8].contiguous(), p, p, k_scales=s[:, :, :8].contiguous(), v_scales=s[:, :, :8].contiguous())):
        a, b = _both(monkeypatch, call)
        assert isinstance(a, Exception) and isinstance(b, Exception), (a, b)
        _same_error(a, b)
