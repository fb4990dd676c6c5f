"""The native and the Python way through the binding of rotary positions, the cache and attention over it: the same results,
refusals and errors."""
import pytest
import torch
from torch.utils._python_dispatch import TorchDispatchMode

from paper_2407_08608_amd import binding
from test_binding import _both, _device_typed, _same_error

needs_native = pytest.mark.skipif(binding._native is None, reason="the native part has not been built")


def _fake_calls():
    # plain tensors that say they are on the device, over no memory: for calls that end before any is touched
    q, k = _device_typed(1, 4, 16, 64), _device_typed(1, 2, 16, 64)
    f = _device_typed(32, dtype=torch.float64)
    pages, codes, scales = _device_typed(3, 2, 16, 64), _device_typed(3, 2, 16, 64, dtype=torch.uint8), _device_typed(3, 2, 16, dtype=torch.float32)
    table, lens = _device_typed(1, 2, dtype=torch.int32), _device_typed(1, dtype=torch.int32)
    return [lambda: binding.fa_rope(q, f, k=k), lambda: binding.fa_rope_bwd(q, f),
            lambda: binding.fa_fwd_cache(q, pages, pages, table, lens, 0.125),
            lambda: binding.fa_fwd_cache(q, codes, codes, table, lens, 0.125, k_scales=scales, v_scales=scales)]


def _as_if_on_a_device(monkeypatch):
    monkeypatch.setattr(binding, "_stream", lambda: 0)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)


def test_an_exception_of_a_dispatch_mode_reaches_the_caller(monkeypatch):
    class Refuse(TorchDispatchMode):
        def __torch_dispatch__(self, func, types, args=(), kwargs=None):
            raise LookupError(f"no {func}")

    binding.lib()
    _as_if_on_a_device(monkeypatch)
    for call in _fake_calls():
        with Refuse():
            a, b = _both(monkeypatch, call)
        assert type(a) is LookupError
        _same_error(a, b)


def test_arguments_that_no_way_takes(monkeypatch):
    x, i = torch.zeros(1, 2, 16, 64), torch.zeros(1, dtype=torch.int32)
    for bad in (x, x[0], None, "q", 3):
        for call in (lambda: binding.fa_rope(bad, x), lambda: binding.fa_rope(x, bad), lambda: binding.fa_cache_write(bad, x, x, x, i, i),
                     lambda: binding.fa_cache_write(x, x, x, bad, i, i), lambda: binding.fa_cache_read(bad, x, i, i, 3),
                     lambda: binding.fa_cache_read(x, x, i, bad, "3"), lambda: binding.fa_fwd_cache(bad, x, x, i, i, 0.1),
                     lambda: binding.fa_fwd_cache(x, x, x, i, bad, "scale")):
            _same_error(*_both(monkeypatch, call))


def _step(dtype=torch.bfloat16, cache=None, B=2, H=4, H_kv=2, T=3, d=64):
    g = torch.Generator(device="cuda").manual_seed(3)
    mk = lambda *s: torch.randn(s, generator=g, device="cuda").to(dtype)  # noqa: E731
    q, k, v = mk(B, H, T, d), mk(B, H_kv, T, d), mk(B, H_kv, T, d)
    pages = [mk(9, H_kv, 16, d) for _ in range(2)]
    scales = [None, None]
    if cache is not None:
        pages = [torch.randint(0, 127, (9, H_kv, 16, d), generator=g, device="cuda", dtype=torch.uint8).view(cache) for _ in range(2)]
        scales = [torch.rand((9, H_kv, 16), generator=g, device="cuda") + 0.01 for _ in range(2)]
    table = torch.tensor([[3, 5, 1, 8], [2, 0, 4, 6]], dtype=torch.int32, device="cuda")
    return q, k, v, pages, scales, table, torch.tensor([40, 17], dtype=torch.int32, device="cuda"), torch.tensor([3, 2], dtype=torch.int32, device="cuda")


@pytest.mark.gpu
@needs_native
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("cache", [None, torch.uint8, torch.float8_e4m3fn])
def test_both_ways_give_the_same(monkeypatch, dtype, cache):
    q, k, v, pages, scales, table, lens, counts = _step(dtype, cache)
    f, _ = binding.fa_rope_frequencies(64)
    half, _ = binding.fa_rope_frequencies(32)
    positions = torch.arange(6, dtype=torch.int32, device="cuda").view(2, 3)
    words = binding.fa_tree_words(torch.ones((2, 3, 3), dtype=torch.bool, device="cuda").tril())
    strided = q.transpose(1, 2).contiguous().transpose(1, 2)
    s = dict(k_scales=scales[0], v_scales=scales[1])

    def write(**kw):
        to = [t.clone() for t in pages] + [None if t is None else t.clone() for t in scales]
        got = binding.fa_cache_write(k, v, to[0], to[1], table, lens, k_scales=to[2], v_scales=to[3], **kw)
        assert got[0] is to[0] and got[1] is to[1] and type(got) is tuple
        return tuple(t for t in to if t is not None)

    def read(**kw):
        type_ = kw.pop("type", dtype)
        x = [torch.zeros((2, 2, 40, 64), device="cuda", dtype=type_) for _ in range(2)]
        return binding.fa_cache_read(pages[0], pages[1], table, lens, k=x[0], v=x[1], **s, **kw)

    def attend(**kw):
        o, lse = torch.zeros_like(q), torch.zeros((2, 4, 3), device="cuda")
        return binding.fa_fwd_cache(kw.pop("q", q), pages[0], pages[1], table, lens, 0.125, o=o, lse=lse, **s, **kw)

    workspace = torch.empty((binding.fa_fwd_cache_workspace_bytes(2, 4, 2, 3, 64, 4096) + 16,), dtype=torch.uint8, device="cuda")
    calls = [lambda: binding.fa_rope(q, f, k=k, positions=positions), lambda: binding.fa_rope(strided, half, rot_dim=32, interleaved=True, amplitude=1.5),
             lambda: binding.fa_rope_bwd(q, f, k=k, q_out=torch.empty_like(strided)), lambda: binding.fa_rope(q.float(), f, k_out=None),
             write, lambda: write(counts=counts), lambda: read(), lambda: read(type=torch.float32), lambda: read(N=40, dtype=dtype),
             lambda: binding.fa_cache_read(pages[0], pages[1], table, lens * 0 + 5, 5, **s), attend, lambda: attend(tree=words, counts=counts, max_len=50),
             lambda: attend(tree=words[:1], max_len=4096, workspace=workspace), lambda: attend(q=strided, max_len=4096),
             lambda: binding.fa_fwd_cache(q, pages[0], pages[1], table, lens, 0.125, **s)]
    for call in calls:
        native, python = _both(monkeypatch, call)
        assert type(native) is tuple and type(python) is tuple and len(native) == len(python), (native, python)
        for a, b in zip(native, python):
            assert (a is None) == (b is None)
            if a is not None:
                assert type(a) is torch.Tensor and a.dtype == b.dtype and a.device == b.device and a.stride() == b.stride()
                assert torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))


@pytest.mark.gpu
def test_both_ways_refuse_the_same(monkeypatch):
    q, k, v, pages, scales, table, lens, counts = _step()
    codes, s = pages[0].to(torch.uint8), torch.ones((9, 2, 16), device="cuda")
    f, _ = binding.fa_rope_frequencies(64)
    small = torch.empty((16,), dtype=torch.uint8, device="cuda")
    W = lambda *a, **kw: binding.fa_cache_write(k, v, *a, **kw)  # noqa: E731
    A = lambda *a, **kw: binding.fa_fwd_cache(*a, 0.125, **kw)  # noqa: E731
    p, t = pages
    for call in (lambda: binding.fa_rope(q, f, amplitude=-1.0), lambda: binding.fa_rope(q, f, rot_dim=32), lambda: binding.fa_rope(q, f, rot_dim=-2),
                 lambda: binding.fa_rope(q, f, rot_dim="x"), lambda: binding.fa_rope(q, f[:12], rot_dim=24), lambda: binding.fa_rope(q, f, k=k[:, :, :2]),
                 lambda: binding.fa_rope(q, f, positions=lens), lambda: binding.fa_rope(q.double(), f), lambda: binding.fa_rope(q, f, q_out=q.float()),
                 lambda: binding.fa_rope(q[..., ::2], f), lambda: binding.fa_rope(q, f.cpu()), lambda: binding.fa_rope(q, f, amplitude="a"),
                 lambda: W(p, t[:3], table, lens), lambda: W(codes, codes, table, lens), lambda: W(p, t, table, lens, k_scales=s, v_scales=s),
                 lambda: W(codes, codes, table, lens, k_scales=s, v_scales=s[:2]), lambda: W(p, t, table[0], lens), lambda: W(p, t, table.long(), lens),
                 lambda: W(p, t, table, lens, counts=counts[:1]), lambda: W(p.half(), t.half(), table, lens), lambda: W(p, t, table.t().contiguous().t(), lens),
                 lambda: binding.fa_cache_read(p, t, table, lens), lambda: binding.fa_cache_read(p, t, table, lens, -1),
                 lambda: binding.fa_cache_read(p, t, table, lens, 0), lambda: binding.fa_cache_read(p, t, table, lens, 3, torch.float16),
                 lambda: binding.fa_cache_read(p, t, table, lens, 3, torch.int32), lambda: binding.fa_cache_read(p, t, table, lens, 3, "x"),
                 lambda: binding.fa_cache_read(p, t, table, lens, k=k, v=v.float()), lambda: binding.fa_cache_read(p, t, table, lens, 4, k=k),
                 lambda: A(q.float(), p, t, table, lens), lambda: A(q[:, :3], p, t, table, lens), lambda: A(q, p, t, table, lens, max_len=-1),
                 lambda: A(q, p, t, table, lens, max_len="x"), lambda: A(q, p, t, table, lens, tree=lens), lambda: A(q, p, t, table, lens, o=q.float()),
                 lambda: A(q, p, t, table, lens, max_len=100000, workspace=small), lambda: A(q, p, t, table, lens, workspace=small.view(torch.int32)),
                 lambda: A(q, p.half(), t.half(), table, lens), lambda: binding.fa_fwd_cache(q, p, t, table, lens, "scale"),
                 lambda: binding.fa_fwd_cache(q, p, t, table, lens, 0.0), lambda: A(q, p[..., :32], t[..., :32], table, lens)):
        a, b = _both(monkeypatch, call)
        assert isinstance(a, Exception) and isinstance(b, Exception), (a, b)
        _same_error(a, b)
