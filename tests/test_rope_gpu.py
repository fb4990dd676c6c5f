"""fa_rope and fa_rope_bwd against the fp64 oracle, element by element.

The bound: sines and cosines are off by at most 2.2e-7 (reduced to half a turn in fp64, then rounded: 2 pi 2^-26; sincospif: 2^-23),
a product with the amplitude, two products and a sum add 4 roundings of 2^-24 to each term, so before the last rounding
|err| <= 5e-7 A (|x_a| + |x_b|); that rounding adds half a step of the output type (and half its smallest subnormal).  The angle
itself is a product of three fp64 numbers, the oracle's of two: 4 * 2^-53 |position| rad more between them (frequencies up to 1)."""
import numpy as np
import pytest
import torch

from helpers import f64
from oracle import cache_oracle
from paper_2407_08608_amd import binding, inputs

pytestmark = pytest.mark.gpu

_T = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_TINY = {"f32": 0.0, "bf16": 0.0, "f16": 2.0 ** -25}


def _check(x, y, inv_freq, positions, rot, interleaved, amplitude, transposed, dtype):
    x, y = f64(x), f64(y)
    want = cache_oracle.rope(x, f64(inv_freq), positions, rot, interleaved, amplitude, transposed)
    size = np.abs(x[..., :rot])
    pair = size[..., 0::2] + size[..., 1::2] if interleaved else size[..., :rot // 2] + size[..., rot // 2:]
    pair = np.repeat(pair, 2, axis=-1) if interleaved else np.concatenate((pair, pair), axis=-1)
    bound = (5e-7 + 2.0 ** -51 * np.abs(np.asarray(positions, dtype=np.float64))[:, None, :, None]) * amplitude * pair
    bound += torch.finfo(_T[dtype]).eps / 2 * (np.abs(want[..., :rot]) + bound) + _TINY[dtype]
    np.testing.assert_array_less(np.abs(y - want)[..., :rot], bound + 1e-300)
    np.testing.assert_array_equal(y[..., rot:], x[..., rot:])


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("B,H,H_kv,N,d,rot", [(1, 1, 1, 1, 64, 64), (3, 5, 1, 7, 128, 128), (2, 8, 2, 33, 256, 256), (2, 3, 3, 65, 128, 32),
                                              (1, 20, 4, 300, 64, 48), (2, 2, 1, 17, 256, 16), (70, 2, 2, 1, 128, 112)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_rope_and_its_gradient(dtype, B, H, H_kv, N, d, rot, interleaved):
    q, k = (inputs.normal_tensor(11, n, (B, h, N, d), dtype).cuda() for n, h in (("q", H), ("k", H_kv)))
    f, amplitude = binding.fa_rope_frequencies(rot, 10000.0, binding.FA_ROPE_BY_PARTS, 4.0, 4096)
    rng = np.random.default_rng(B * N + d)
    at = rng.integers(-50, 200000, (B, N)).astype(np.int32)
    at[0, 0] = 2 ** 31 - 1
    for positions in (None, at):
        place = np.broadcast_to(np.arange(N), (B, N)) if positions is None else positions
        t = None if positions is None else torch.from_numpy(positions).cuda()
        for call, transposed in ((binding.fa_rope, False), (binding.fa_rope_bwd, True)):
            y = call(q, f, k=k, positions=t, rot_dim=rot, interleaved=interleaved, amplitude=amplitude)
            for x, got in zip((q, k), y):
                assert got.is_contiguous() and got.dtype == x.dtype
                _check(x, got, f, place, rot, interleaved, amplitude, transposed, dtype)


def test_gradient_is_the_derivative():
    # y is linear in x, so a difference over any step is the derivative: <dy, rope(x + e) - rope(x)> = <rope_bwd(dy), e>
    q = inputs.normal_tensor(1, "q", (2, 3, 9, 64), "f32").cuda()
    e, dy = (inputs.normal_tensor(s, "q", (2, 3, 9, 64), "f32").cuda() for s in (2, 3))
    for interleaved in (False, True):
        f, _ = binding.fa_rope_frequencies(32)
        turn = lambda x: binding.fa_rope(x, f, rot_dim=32, interleaved=interleaved, amplitude=1.25)[0].double()  # noqa: E731,B023
        back = binding.fa_rope_bwd(dy, f, rot_dim=32, interleaved=interleaved, amplitude=1.25)[0].double()
        left, right = (dy.double() * (turn(q + e) - turn(q))).sum(), (back * e.double()).sum()
        # about 8 roundings of 2^-24 relative to each of the 3456 terms, which have random signs: 3456^0.5 * 8 * 2^-24 * 5
        assert abs(float(left - right)) < 2e-4


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_strided_rows_in_and_out_and_in_place(dtype):
    B, H, H_kv, N, d, rot = 2, 6, 2, 37, 128, 64
    f, _ = binding.fa_rope_frequencies(rot)
    # one projection's [B, N, H + 2 H_kv, d], of which Q and K are slices
    qkv = inputs.normal_tensor(5, "qkv", (B, N, H + 2 * H_kv, d), dtype).cuda()
    q, k = qkv[:, :, :H].transpose(1, 2), qkv[:, :, H:H + H_kv].transpose(1, 2)
    want = binding.fa_rope(q.contiguous(), f, k=k.contiguous(), rot_dim=rot)
    place = np.broadcast_to(np.arange(N), (B, N))
    _check(q, want[0], f, place, rot, False, 1.0, False, dtype)
    got = binding.fa_rope(q, f, k=k, rot_dim=rot)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    # a broadcast batch and tokens in reverse head order
    same = q[:1].expand(B, H, N, d)
    assert torch.equal(binding.fa_rope(same, f, rot_dim=rot)[0][1], want[0][0])
    # in place: the projection's other columns stay as they are
    before = qkv.clone()
    got = binding.fa_rope(q, f, k=k, rot_dim=rot, q_out=q, k_out=k)
    assert got[0] is q and torch.equal(q, want[0]) and torch.equal(k, want[1])
    assert torch.equal(qkv[:, :, H + H_kv:], before[:, :, H + H_kv:])
    # into a larger tensor
    room = torch.full((B, H + 1, N + 3, d + 8), 7.0, dtype=q.dtype, device="cuda")
    binding.fa_rope(want[0], f, rot_dim=rot, q_out=room[:, 1:, 2:-1, :d])
    assert torch.equal(room[:, 1:, 2:-1, :d], binding.fa_rope(want[0], f, rot_dim=rot)[0])
    assert (room[:, 0] == 7).all() and (room[:, :, :2] == 7).all() and (room[:, :, -1:] == 7).all() and (room[..., d:] == 7).all()


def test_a_row_of_special_values_is_its_own_only():
    q = inputs.normal_tensor(6, "q", (1, 2, 5, 64), "bf16").cuda()
    f, _ = binding.fa_rope_frequencies(64)
    want = binding.fa_rope(q, f)[0]
    bad = q.clone()
    bad[0, 1, 3, 10], bad[0, 1, 3, 20] = float("inf"), float("nan")
    got = binding.fa_rope(bad, f)[0]
    row = torch.zeros_like(q, dtype=torch.bool)
    row[0, 1, 3, [10, 42, 20, 52]] = True
    assert torch.equal(got[~row], want[~row]) and not torch.isfinite(got[row]).any()


def test_many_tokens_and_heads():
    # more (token, head) groups than one launch dimension holds without walking heads, and every head the same
    f, _ = binding.fa_rope_frequencies(64)
    q = inputs.normal_tensor(8, "q", (1, 1, 5000, 64), "bf16").cuda()
    want = binding.fa_rope(q, f)[0]
    got = binding.fa_rope(q.expand(1, 70, 5000, 64), f, k=q.expand(1, 30, 5000, 64))
    assert torch.equal(got[0], want.expand(1, 70, 5000, 64)) and torch.equal(got[1], want.expand(1, 30, 5000, 64))
    # very many heads of one token
    q = inputs.normal_tensor(9, "q", (1, 1, 1, 64), "bf16").cuda()
    p = torch.tensor([[77]], dtype=torch.int32, device="cuda")
    want = binding.fa_rope(q, f, positions=p)[0]
    got = binding.fa_rope(q.expand(1, 200000, 1, 64), f, positions=p)[0]
    assert torch.equal(got, want.expand(1, 200000, 1, 64))


def test_the_binding_refuses_what_does_not_fit():
    q = torch.zeros((2, 4, 8, 64), device="cuda", dtype=torch.bfloat16)
    f, _ = binding.fa_rope_frequencies(64)
    p = torch.zeros((2, 8), dtype=torch.int32, device="cuda")
    for kw in (dict(k=q.float()), dict(k=q[:, :, :4].contiguous()), dict(positions=p.long()), dict(positions=p[:1]), dict(rot_dim=32),
               dict(q_out=q.float()), dict(q_out=q[:, :2]), dict(k=q, k_out=q[..., ::2])):
        with pytest.raises(ValueError):
            binding.fa_rope(q, f, **kw)
    for bad in (q.double(), q[..., ::2], q[0], q.cpu()):
        with pytest.raises(ValueError):
            binding.fa_rope(bad, f)
    with pytest.raises(ValueError):
        binding.fa_rope(q, f.float())
    for kw in (dict(rot_dim=24, f=12), dict(amplitude=0.0), dict(rot_dim=128, f=64)):
        n = kw.pop("f", None)
        with pytest.raises(binding.FaError):
            binding.fa_rope(q, f if n is None else torch.zeros(n, dtype=torch.float64, device="cuda"), **kw)
