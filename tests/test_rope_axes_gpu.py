"""fa_rope_axes and fa_rope_axes_bwd against the fp64 oracle, element by element, within the bound of test_rope_gpu.py: sines and cosines
off by at most 2.2e-7, 4 roundings of 2^-24 in the products and the sum, half a step of the output's type, and 4 * 2^-53 |position|."""
import numpy as np
import pytest
import torch

from helpers import f64
from oracle import cache_oracle
from paper_2407_08608_amd import binding, inputs

pytestmark = pytest.mark.gpu

_T = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def _check(x, y, f, axis, positions, rot, interleaved, amplitude, transposed, dtype):
    x, y, axis, positions = f64(x), f64(y), np.asarray(axis), np.asarray(positions)
    want = cache_oracle.rope_axes(x, f64(f), axis, positions, rot, interleaved, amplitude, transposed)
    size = np.abs(x[..., :rot])
    pair = size[..., 0::2] + size[..., 1::2] if interleaved else size[..., :rot // 2] + size[..., rot // 2:]
    bound = (5e-7 + 2.0 ** -51 * np.abs(positions.astype(np.float64)).max(axis=0))[:, None, :, None] * amplitude * pair
    bound = np.repeat(bound, 2, axis=-1) if interleaved else np.concatenate((bound, bound), axis=-1)
    bound += torch.finfo(_T[dtype]).eps / 2 * (np.abs(want[..., :rot]) + bound) + (2.0 ** -25 if dtype == "f16" else 0)
    np.testing.assert_array_less(np.abs(y - want)[..., :rot], bound + 1e-300)
    np.testing.assert_array_equal(y[..., rot:], x[..., rot:])


def _tensors(seed, B, H, H_kv, N, d, rot, axes, dtype):
    q, k = (inputs.normal_tensor(seed, n, (B, h, N, d), dtype).cuda() for n, h in (("q", H), ("k", H_kv)))
    g = np.random.default_rng(seed)
    at = g.integers(-50, 200000, (axes, B, N)).astype(np.int32)
    at[-1, 0, 0] = 2 ** 31 - 1
    return q, k, g.integers(0, axes, rot // 2).astype(np.int32), at


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("B,H,H_kv,N,d,rot,axes", [(1, 1, 1, 1, 64, 64, 1), (3, 5, 1, 7, 128, 128, 3), (2, 8, 2, 33, 256, 256, 2), (2, 3, 3, 65, 128, 32, 4),
                                                   (1, 20, 4, 300, 64, 48, 3), (2, 2, 1, 17, 256, 16, 7), (70, 2, 2, 1, 128, 112, 5)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_rotation_and_its_gradient(dtype, B, H, H_kv, N, d, rot, axes, interleaved):
    q, k, axis, at = _tensors(B * N + d, B, H, H_kv, N, d, rot, axes, dtype)
    f, amplitude = binding.fa_rope_frequencies(rot, 10000.0, binding.FA_ROPE_BY_PARTS, 4.0, 4096)
    for call, transposed in ((binding.fa_rope_axes, False), (binding.fa_rope_axes_bwd, True)):
        y = call(q, f, torch.from_numpy(axis).cuda(), torch.from_numpy(at).cuda(), k=k, rot_dim=rot, interleaved=interleaved, amplitude=amplitude)
        for x, got in zip((q, k), y):
            assert got.is_contiguous() and got.dtype == x.dtype
            _check(x, got, f, axis, at, rot, interleaved, amplitude, transposed, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_equal_positions_are_those_of_one_axis(dtype):
    q, k, axis, at = _tensors(3, 2, 4, 2, 50, 128, 128, 3, dtype)
    f, _ = binding.fa_rope_frequencies(128)
    at[:] = at[0]
    place = torch.from_numpy(at).cuda()
    got = binding.fa_rope_axes(q, f, torch.from_numpy(axis).cuda(), place, k=k)
    want = binding.fa_rope(q, f, k=k, positions=place[0].contiguous())
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_an_axis_that_there_is_not_turns_nothing():
    q, _, axis, at = _tensors(4, 2, 3, 1, 20, 64, 64, 2, "bf16")
    f, _ = binding.fa_rope_frequencies(64)
    axis[5], axis[6], axis[7] = -1, 2, 2 ** 31 - 1
    got, none = binding.fa_rope_axes(q, f, torch.from_numpy(axis).cuda(), torch.from_numpy(at).cuda(), amplitude=1.5)
    assert none is None
    _check(q, got, f, axis, at, 64, False, 1.5, False, "bf16")
    assert torch.equal(got[..., 5:8], q[..., 5:8] * 1.5)


def test_gradient_is_the_derivative():
    # y is linear in x, so a difference over any step is the derivative: <dy, rope(x + e) - rope(x)> = <rope_bwd(dy), e>
    q, _, axis, at = _tensors(5, 2, 3, 1, 9, 64, 32, 3, "f32")
    e, dy = (inputs.normal_tensor(s, "q", (2, 3, 9, 64), "f32").cuda() for s in (2, 3))
    f, _ = binding.fa_rope_frequencies(32)
    axis, at = torch.from_numpy(axis).cuda(), torch.from_numpy(at).cuda()
    for interleaved in (False, True):
        kw = dict(rot_dim=32, interleaved=interleaved, amplitude=1.25)
        turn = lambda x: binding.fa_rope_axes(x, f, axis, at, **kw)[0].double()  # noqa: E731,B023
        back = binding.fa_rope_axes_bwd(dy, f, axis, at, **kw)[0].double()
        left, right = (dy.double() * (turn(q + e) - turn(q))).sum().item(), (back * e.double()).sum().item()
        # each of 3456 elements is off by some 1e-6 of a few units before the products are summed
        assert abs(left - right) <= 3456 * 8e-6, (left, right)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_projection_layout_in_place_and_on_another_stream(dtype):
    B, H, H_kv, N, d = 2, 4, 2, 37, 128
    q, k, axis, at = _tensors(6, B, H, H_kv, N, d, 64, 3, dtype)
    f, _ = binding.fa_rope_frequencies(64)
    axis, at = torch.from_numpy(axis).cuda(), torch.from_numpy(at).cuda()
    want = binding.fa_rope_axes(q, f, axis, at, k=k, rot_dim=64)
    row = torch.empty((B, N, (H + 2 * H_kv) * d), dtype=q.dtype, device="cuda")  # Q, K and V of a token side by side
    sq = row[..., :H * d].view(B, N, H, d).transpose(1, 2)
    sk = row[..., H * d:(H + H_kv) * d].view(B, N, H_kv, d).transpose(1, 2)
    sq.copy_(q)
    sk.copy_(k)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = binding.fa_rope_axes(sq, f, axis, at, k=sk, rot_dim=64)
        binding.fa_rope_axes(sq, f, axis, at, k=sk, rot_dim=64, q_out=sq, k_out=sk)
    torch.cuda.current_stream().wait_stream(side)
    for a, b, c in zip(got, (sq, sk), want):
        assert torch.equal(a, c) and torch.equal(b, c)


def test_large_inputs_are_streamed_to_the_same_values():
    q, _, axis, at = _tensors(7, 1, 40, 1, 8192, 128, 128, 3, "bf16")  # 80 MiB
    f, _ = binding.fa_rope_frequencies(128)
    axis, at = torch.from_numpy(axis).cuda(), torch.from_numpy(at).cuda()
    got = binding.fa_rope_axes(q, f, axis, at)[0]
    parts = torch.cat([binding.fa_rope_axes(q[:, h:h + 5].contiguous(), f, axis, at)[0] for h in range(0, 40, 5)], 1)
    assert torch.equal(got, parts)
