"""A cache of e2m1 codes: written and read bit for bit as the definitions say, and attention over it against the fp64 oracle, element by
element.  Whatever a row must not see holds NaN scales over random codes.

The bound of a row, with s_j its scores, w_j = p_j / sum p its weights, eps half a step of a type (bf16 2^-8, fp16 2^-11), and every cached
value a bf16 number as it is:
  scores    products are exact in fp32 and d of them are summed; with fp16 Q K is in units, powers of two, of its row's largest scale:
            e_s = (2 d + 4) 2^-24 scale max_j sum |q k_j|
  weights   the argument of the exponential, in units of log 2, is rounded at |s| and |m|: 2^-22 max |s|; the exponential itself 2^-21;
            numerator and sum both: e_w = 2 (e_s + 2^-22 max |s| + 2^-21)
  O         (e_w + eps_p + n 2^-24) sum w |v| + eps_o |O|; eps_p: probabilities as two bf16 numbers 2^-16, as one (bf16 Q with more than 16
            rows to a key/value head) 2^-8.  And 2 n 2^-126 (1 + max |v|): fp32 and bf16 have no normal numbers below 2^-126, and what is
            below may count as zero: a probability p, or what its first bf16 number leaves out (off by 2^-126 |v| at most, each), and a
            product p v (2^-126), for each of n keys.  sum p, which all is divided by, is at least 1: the reference of a row is a score
            of its own.
  L         e_s + 2^-22 max |s| + 2^-20 + 2^-23 |L|"""
import numpy as np
import pytest
import torch

from helpers import f64
from oracle import cache_oracle
from paper_2407_08608_amd import binding, inputs
from test_cache_gpu import make_table
from test_fwd_cache_gpu import _random_tree

pytestmark = pytest.mark.gpu

_T = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_HALF = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11}


def _empty_cache(seed, n_pages, H_kv, page, d):
    """Pages full of earlier codes: [k_pages, v_pages, k_scales, v_scales]"""
    g = torch.Generator(device="cuda").manual_seed(seed)
    return [torch.randint(0, 256, (n_pages, H_kv, page, n), generator=g, device="cuda", dtype=torch.uint8) for n in (d // 2, d // 2, d // 32, d // 32)]


@pytest.mark.parametrize("dense", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("B,H_kv,T,d,page,max_pages", [(1, 1, 1, 64, 16, 1), (3, 2, 1, 128, 16, 5), (2, 3, 37, 256, 48, 3), (4, 5, 70, 64, 32, 4),
                                                       (2, 1, 19, 128, 16, 9)])
def test_write(dense, B, H_kv, T, d, page, max_pages):
    n_pages = B * max_pages + 2
    cache = _empty_cache(B + T, n_pages, H_kv, page, d)
    table = make_table(T, B, max_pages, n_pages)
    rng = np.random.default_rng(d + T)
    lens = torch.from_numpy(rng.integers(0, max(max_pages * page - T, 0) + 1, B).astype(np.int32))
    counts = torch.from_numpy(rng.integers(0, T + 1, B).astype(np.int32))
    counts[0] = T
    k, v = (inputs.heavy_tailed_tensor(3, n, (B, H_kv, T, d), dense, p_outlier=0.05).cuda() for n in ("k", "v"))
    k[0, 0, 0, :32] = 0
    k[0, 0, 0, 32:64] = float("inf")
    k[0, 0, 0, 33], k[-1, -1, -1, 5], k[-1, -1, -1, 6] = 1.5, float("-inf"), -0.0
    v[-1, -1, -1, 40], v[0, 0, 0, 3] = float("nan"), torch.finfo(_T[dense]).max
    v[0, 0, 0, 32:64] = torch.finfo(_T[dense]).tiny
    # the values in the middle of two codes, and at the border of two scales
    border = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0], device="cuda")
    v[0, -1, -1, :32] = torch.cat((border, -border, border / 2, -border / 4))
    v[0, -1, -1, 32:64] = 3.5
    if dense == "f16":  # multiples of the smallest number there is
        k[0, -1, -1, :32] = torch.arange(32, device="cuda") * 2.0 ** -24
        k[0, -1, -1, 32:64] = -2.0 ** -24
    for n in (None, counts):
        have = [t.clone() for t in cache]
        got = binding.fa_cache_write(k, v, have[0], have[1], table.cuda(), lens.cuda(), counts=None if n is None else n.cuda(), k_scales=have[2], v_scales=have[3])
        assert got[0] is have[0] and got[1] is have[1]
        for x, pages, scales, a, s in ((k, cache[0], cache[2], have[0], have[2]), (v, cache[1], cache[3], have[1], have[3])):
            codes, powers = (torch.from_numpy(y) for y in cache_oracle.quantise_groups(x.float().cpu().numpy()))
            want, want_s, a, s = pages.cpu(), scales.cpu(), a.cpu(), s.cpu()
            for b in range(B):
                for t in range(T if n is None else int(n[b])):
                    at = cache_oracle.place({"k_pages": pages, "block_table": table.numpy()}, b, int(lens[b]) + t)
                    if at is not None:
                        want[at[0], :, at[1]], want_s[at[0], :, at[1]] = codes[b, :, t], powers[b, :, t]
            nan = torch.repeat_interleave((want_s == 255) & (s == 255), 16, -1)  # (of a NaN scale any codes)
            assert torch.equal(s, want_s) and torch.equal(torch.where(nan, 0, a), torch.where(nan, 0, want))


@pytest.mark.parametrize("dtypes", [(torch.uint8, torch.uint8), (torch.float4_e2m1fn_x2, torch.float8_e8m0fnu), (torch.uint8, torch.float8_e8m0fnu)])
@pytest.mark.parametrize("out", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_read_of_every_code_and_scale(out, d, dtypes):
    H_kv, page, n_pages = 2, 32, 9
    cache = _empty_cache(d, n_pages, H_kv, page, d)
    flat = cache[2].view(-1)  # every scale, over every code somewhere
    flat[:256] = torch.arange(256, dtype=torch.uint8, device="cuda")
    table, lens = torch.tensor([[0, 3, 1], [8, -1, 2]], dtype=torch.int32), torch.tensor([70, 96], dtype=torch.int32)
    typed = [t.view(dtypes[i // 2]) for i, t in enumerate(cache)]
    k, v = (torch.full((2, H_kv, 96, d), 7.0, device="cuda", dtype=_T[out]) for _ in range(2))
    binding.fa_cache_read(typed[0], typed[1], table.cuda(), lens.cuda(), k_scales=typed[2], v_scales=typed[3], k=k, v=v)
    host = {"k_pages": cache[0].cpu().numpy(), "block_table": table.numpy()}
    for x, pages, scales in ((k, cache[0], cache[2]), (v, cache[1], cache[3])):
        with np.errstate(over="ignore"):  # a code of the largest scales is past fp32, as in any type
            values = torch.from_numpy(cache_oracle.group_values(pages.cpu().numpy(), scales.cpu().numpy()).astype(np.float32)).to(_T[out])
        for b in range(2):
            for p in range(96):
                at = cache_oracle.place(host, b, p) if p < int(lens[b]) else None
                want = values[at[0], :, at[1]] if at is not None else torch.full((H_kv, d), 7.0, dtype=_T[out])
                assert torch.equal(torch.nan_to_num(x[b, :, p].cpu().float(), nan=5e30), torch.nan_to_num(want.float(), nan=5e30)), (b, p)


class Case:
    """A filled cache, queries, and what each row may see"""

    def __init__(self, seed, dtype, B, H, H_kv, T, d, page, lens, counts=None, tree=None, width=None, table=None, k_std=1.0, spread=3):
        self.dtype, self.scale, self.rows = dtype, d ** -0.5, H // H_kv * T
        g = np.random.default_rng(seed)
        self.lens = np.asarray(lens, dtype=np.int32)
        self.counts = np.full(B, T) if counts is None else np.asarray(counts)
        self.tree = tree
        width = -(-(int(max(self.lens)) + T) // page) if width is None else width
        n_pages = B * width + 3 if table is None else 19
        self.table = g.permutation(n_pages)[:B * width].reshape(B, width).astype(np.int32) if table is None else table
        self.host = {"block_table": self.table}
        live = np.zeros((n_pages, page), dtype=bool)
        for b in range(B):
            for p in range(max(int(self.lens[b]), 0) + min(int(self.counts[b]), T)):
                at = cache_oracle.place({"k_pages": np.empty((n_pages, 1, page, 1)), "block_table": self.table}, b, p)
                if at is not None:
                    live[at] = True
        for n in ("k", "v"):
            x = g.standard_normal((n_pages, H_kv, page, d)) * 2.0 ** g.integers(-spread, 1, (n_pages, H_kv, page, d // 32)).repeat(32, axis=-1)
            codes, powers = cache_oracle.quantise_groups((x * (k_std if n == "k" else 1.0)).astype(np.float32))
            powers[np.broadcast_to(~live[:, None], powers.shape[:3])] = 255
            self.host[n + "_pages"], self.host[n + "_scales"] = codes, powers
        self.q = inputs.normal_tensor(seed, "q", (B, H, T, d), dtype)
        self.args = {n: torch.from_numpy(x).cuda() for n, x in self.host.items()}
        self.args.update(lens=torch.from_numpy(self.lens).cuda(), scale=self.scale, counts=None if counts is None else torch.from_numpy(self.counts.astype(np.int32)).cuda(),
                         tree=None if tree is None else binding.fa_tree_words(torch.from_numpy(tree)).cuda())

    def run(self, **kw):
        return binding.fa_fwd_cache(**dict(dict(self.args, q=self.q.cuda()), **kw))

    def check(self, o, lse, rows=None):
        q = f64(self.q)
        want = cache_oracle.attend(q, self.host, self.lens, self.counts, self.tree, self.scale)
        o, lse, d, half = f64(o), f64(lse), q.shape[-1], _HALF[self.dtype]
        eps_p = 2.0 ** -16 if self.dtype == "f16" or self.rows <= 16 else 2.0 ** -8
        for (b, h, t), (x, L, K, V) in want.items():
            if rows is not None and t not in rows:
                continue
            got, got_l = o[b, h, t], lse[b, h, t]
            if len(K) == 0:
                assert (got == 0).all() and got_l == -np.inf, (b, h, t)
                continue
            s = self.scale * (K @ q[b, h, t])
            top = np.abs(s).max()
            e_s = (2 * d + 4) * 2.0 ** -24 * self.scale * (np.abs(K) @ np.abs(q[b, h, t])).max()
            e_w = 2 * (e_s + 2.0 ** -22 * top + 2.0 ** -21)
            bound = (e_w + eps_p + len(K) * 2.0 ** -24) * (np.exp(s - L) @ np.abs(V)) + half * np.abs(x) + (2.0 ** -25 if self.dtype == "f16" else 2.0 ** -134)
            bound += 2 * len(K) * 2.0 ** -126 * (1 + np.abs(V).max(axis=0))
            err = np.abs(got - x)
            fits = np.abs(x) + bound < float(torch.finfo(_T[self.dtype]).max)
            assert (err[fits] <= bound[fits]).all(), ((b, h, t), err[fits].max(), bound[fits][np.argmax((err - bound)[fits])])
            assert abs(got_l - L) <= e_s + 2.0 ** -22 * top + 2.0 ** -20 + 2.0 ** -23 * abs(L), ((b, h, t), got_l, L)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("B,H,H_kv,page,lens", [
    (1, 1, 1, 16, [0]),                      # the token itself
    (4, 4, 4, 16, [1, 15, 16, 17]),          # around a page
    (5, 8, 2, 16, [30, 31, 32, 33, 63]),     # around a tile of 32 keys, with their own key
    (3, 6, 1, 48, [127, 500, 0]),            # pages that no tile divides
    (2, 32, 2, 128, [777, 1290]),            # 16 heads to a key/value head
    (1, 40, 1, 64, [333]),                   # more rows than a tile
])
def test_one_token(dtype, d, B, H, H_kv, page, lens):
    c = Case(100 + d, dtype, B, H, H_kv, 1, d, page, lens)
    c.check(*c.run())


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d,B,H,H_kv,T,page,lens,counts", [
    (64, 2, 4, 4, 2, 16, [0, 31], None),
    (128, 3, 4, 2, 5, 16, [0, 100, 30], [5, 0, 3]),
    (64, 2, 6, 2, 33, 32, [250, 15], [33, 32]),
    (256, 2, 4, 1, 13, 16, [99, 640], [13, 1]),
    (128, 2, 4, 1, 15, 16, [99, 640], [15, 2]),
    (128, 1, 8, 2, 64, 64, [1000], None),
    (256, 1, 8, 2, 10, 64, [400], None),
    (128, 2, 2, 1, 100, 16, [5, 300], [77, 100]),
    (256, 2, 2, 1, 100, 16, [5, 300], [77, 100]),
    (64, 1, 2, 2, 256, 48, [123], None),
])
def test_chains_and_trees(dtype, d, B, H, H_kv, T, page, lens, counts):
    for tree in (None, _random_tree(T, B, T), _random_tree(T, B, T, empty=True)):
        c = Case(200 + T, dtype, B, H, H_kv, T, d, page, lens, counts, tree)
        o, lse = torch.full(c.q.shape, 7.0, dtype=c.q.dtype, device="cuda"), torch.full(c.q.shape[:3], 7.0, device="cuda")
        got = c.run(o=o, lse=lse)
        assert got[0] is o and got[1] is lse
        c.check(o, lse)
        for b in range(B):
            assert (o[b, :, c.counts[b]:] == 7).all() and (lse[b, :, c.counts[b]:] == 7).all()


# d, H, H_kv, T: up to 16, 32 and 64 rows to a key/value head, and more
_FORMS = [(64, 8, 4, 3), (128, 4, 2, 2), (256, 4, 2, 3), (128, 8, 2, 6), (64, 8, 2, 12), (128, 8, 2, 12), (256, 8, 2, 12), (64, 4, 1, 20),
          (128, 8, 2, 40), (256, 4, 1, 30)]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d,H,H_kv,T", _FORMS)
def test_pages_that_are_none_and_places_past_the_table(dtype, d, H, H_kv, T):
    page, width = 16, 4
    table = np.array([[0, -1, 2, 3], [-1, -1, -1, -1], [4, 5, 6, 19], [7, 8, 9, 10]], dtype=np.int32)  # of 19 pages
    # a hole; nothing at all; the last page is none; new tokens past the last place, and lengths that are far past it or negative
    for lens in ([60, 20, 50, 61], [10, 0, 3, 64], [2 ** 31 - 1, 5, 64, -5]):
        c = Case(7, dtype, 4, H, H_kv, T, d, page, np.minimum(lens, 64), tree=_random_tree(3, 4, T), width=width, table=table)
        o, lse = c.run(lens=torch.tensor(lens, dtype=torch.int32).cuda())
        c.check(o, lse)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d,H,H_kv,T,lens", [(128, 2, 2, 1, [70001, 40]), (64, 16, 2, 1, [33000, 9000]), (256, 8, 1, 3, [20011, 1]), (128, 4, 1, 40, [9000, 300])])
def test_long_caches_are_divided_and_joined(dtype, d, H, H_kv, T, lens):
    c = Case(300 + d, dtype, 2, H, H_kv, T, d, 64, lens, tree=_random_tree(T, 2, T) if T > 1 else None)
    o, lse = c.run()
    c.check(o, lse)
    for max_len in (1, 5000, 1 << 20):
        c.check(*c.run(max_len=max_len))
    assert torch.equal(c.run()[0], o) and torch.equal(c.run()[1], lse)  # repeatable


@pytest.mark.parametrize("dtype,d,B,H,H_kv,T,lens", [("bf16", 64, 48, 8, 8, 1, (1, 400)), ("f16", 128, 48, 16, 8, 1, (1, 400)), ("bf16", 64, 70, 4, 2, 3, (0, 700)),
                                                     ("f16", 64, 130, 2, 1, 1, (0, 900)), ("bf16", 128, 20, 16, 2, 9, (0, 600)), ("f16", 256, 66, 2, 2, 1, (3, 300))])
def test_shares_of_many_sequences(dtype, d, B, H, H_kv, T, lens):
    c = Case(400 + B, dtype, B, H, H_kv, T, d, 16, np.random.default_rng(B).integers(lens[0], lens[1] + 1, B))
    for max_len in (0, 1 << 20):
        c.check(*c.run(max_len=max_len))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d,H,H_kv,T", _FORMS)
@pytest.mark.parametrize("max_len", [0, 1 << 20])
def test_values_that_are_not_finite(dtype, d, H, H_kv, T, max_len):
    """A NaN scale of one new token's V, and K: rows that do not see it are as they were bit for bit, rows that do have NaN in its 32 columns"""
    tree = _random_tree(T, 2, T)
    c = Case(500 + T, dtype, 2, H, H_kv, T, d, 16, [300, 21], tree=tree)
    clean = c.run(max_len=max_len)
    c.check(*clean)
    u, group = T // 2, 1
    slots = [cache_oracle.place(c.host, b, int(c.lens[b]) + u) for b in range(2)]
    scales = c.args["v_scales"].clone()
    for page, slot in slots:
        scales[page, :, slot, group] = 255
    got = c.run(v_scales=scales, max_len=max_len)
    sick = torch.zeros(d, dtype=torch.bool, device="cuda")
    sick[32 * group:32 * group + 32] = True
    for b in range(2):
        for t in range(T):
            a, x = got[0][b, :, t], clean[0][b, :, t]
            assert torch.equal(got[1][b, :, t], clean[1][b, :, t])
            if tree[b, t, u]:
                assert a[:, sick].isnan().all() and torch.equal(a[:, ~sick], x[:, ~sick]), (b, t)
            else:
                assert torch.equal(a, x), (b, t)
    scales = c.args["k_scales"].clone()
    for page, slot in slots:
        scales[page, :, slot, group] = 255
    got = c.run(k_scales=scales, max_len=max_len)
    for b in range(2):
        for t in range(T):
            if tree[b, t, u]:
                assert got[0][b, :, t].isnan().all() and got[1][b, :, t].isnan().all()
            else:
                assert torch.equal(got[0][b, :, t], clean[0][b, :, t]) and torch.equal(got[1][b, :, t], clean[1][b, :, t])


@pytest.mark.parametrize("d,H,H_kv,T", _FORMS)
def test_scales_of_very_different_size(d, H, H_kv, T):
    # in bf16 every scale and value fits; scores of up to some hundred, values from 2^-60 to 2^60 in one row
    c = Case(600 + T, "bf16", 2, H, H_kv, T, d, 16, [200, 50], k_std=30.0, spread=60)
    c.check(*c.run())
    c = Case(601 + T, "f16", 2, H, H_kv, T, d, 16, [200, 50], k_std=300.0, spread=20)
    c.check(*c.run())
    # K past what fp16 holds, made up for by a small scale
    c = Case(602 + T, "f16", 2, H, H_kv, T, d, 16, [200, 50], k_std=1e6, spread=3)
    c.scale = c.args["scale"] = 1e-6 * d ** -0.5
    c.check(*c.run())


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d,H,H_kv,T", _FORMS)
def test_scales_of_zeros_are_any(dtype, d, H, H_kv, T):
    """A group of zeros, of either sign, is zero whatever its scale, and has no influence on the other groups' values"""
    c = Case(700 + T, dtype, 2, H, H_kv, T, d, 16, [200, 50])
    groups = np.random.default_rng(T).random(c.host["k_scales"].shape) < 0.3
    big = {}
    for n in ("k", "v"):
        zero = torch.from_numpy(groups).cuda()
        codes = torch.where(zero.repeat_interleave(16, -1), 0x80, c.args[n + "_pages"])
        c.args[n + "_pages"], c.host[n + "_pages"] = codes, codes.cpu().numpy()
        low = torch.where(zero & (c.args[n + "_scales"] != 255), 27, c.args[n + "_scales"]).to(torch.uint8)
        c.args[n + "_scales"], c.host[n + "_scales"] = low, low.cpu().numpy()
        big[n] = low
    want = c.run()
    c.check(*want)
    for scale in (0, 1, 254, 228, 255 - 127, 253):
        kw = {n + "_scales": torch.where(torch.from_numpy(groups).cuda() & (big[n] != 255), scale, big[n]).to(torch.uint8) for n in ("k", "v")}
        got = c.run(**kw)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]), scale


def test_rising_scores():
    # every tile of keys raises the maximum
    for dtype in ("bf16", "f16"):
        c = Case(8, dtype, 1, 4, 4, 1, 128, 16, [2000])
        ramp = torch.linspace(0, 8, 2001).floor().to(torch.uint8)
        for p in range(2001):
            page, slot = cache_oracle.place(c.host, 0, p)
            c.args["k_scales"][page, :, slot] += ramp[p].item()
        c.host["k_scales"] = c.args["k_scales"].cpu().numpy()
        c.check(*c.run())


def test_strides_another_stream_and_types():
    B, H, H_kv, T, d = 2, 8, 2, 5, 128
    c = Case(9, "bf16", B, H, H_kv, T, d, 16, [100, 40])
    want = c.run()
    q = c.q.cuda().transpose(1, 2).contiguous().transpose(1, 2)
    o = torch.empty((B, T, H, d), dtype=torch.bfloat16, device="cuda").transpose(1, 2)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = c.run(q=q, o=o)
    torch.cuda.current_stream().wait_stream(side)
    assert got[0] is o and torch.equal(o, want[0]) and torch.equal(got[1], want[1])
    typed = {n: c.args[n].view(torch.float4_e2m1fn_x2 if "pages" in n else torch.float8_e8m0fnu) for n in ("k_pages", "v_pages", "k_scales", "v_scales")}
    assert torch.equal(c.run(**typed)[0], want[0])


def test_a_captured_step_with_pages_positions_and_attention():
    """The run of a serving step, captured once: pages for the new tokens, positions with three axes, the 4-bit cache written, attention over
    it.  Replays on new inputs give what the calls give, and what the oracle says of the written cache."""
    B, H, H_kv, T, d, page, wide = 3, 8, 2, 4, 128, 16, 8
    n_pages = 30
    cache = [torch.zeros((n_pages, H_kv, page, n), dtype=torch.uint8, device="cuda") for n in (d // 2, d // 2, d // 32, d // 32)]
    table = torch.full((B, wide), -1, dtype=torch.int32, device="cuda")
    lens = torch.zeros(B, dtype=torch.int32, device="cuda")
    counts, positions = torch.zeros(B, dtype=torch.int32, device="cuda"), torch.zeros((3, B, T), dtype=torch.int32, device="cuda")
    q, k, v = (torch.zeros((B, h, T, d), dtype=torch.bfloat16, device="cuda") for h in (H, H_kv, H_kv))
    f, _ = binding.fa_rope_frequencies(d)
    axis = (torch.arange(d // 2, device="cuda") % 3).int()
    outs = [torch.zeros_like(q), torch.zeros((B, H, T), device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")]
    qr, kr = torch.zeros_like(q), torch.zeros_like(k)
    pool_space = torch.empty(max(binding.fa_cache_pages_workspace_bytes(B, n_pages), 16), dtype=torch.uint8, device="cuda")
    space = torch.empty(max(binding.fa_fwd_cache_workspace_bytes(B, H, H_kv, T, d, wide * page, binding.FA_FP4_E2M1), 16), dtype=torch.uint8, device="cuda")

    def step():
        binding.fa_cache_extend(table, lens, T, page, n_pages, counts=counts, missing=outs[2], workspace=pool_space)
        binding.fa_rope_axes(q, f, axis, positions, k=k, q_out=qr, k_out=kr)
        binding.fa_cache_write(kr, v, cache[0], cache[1], table, lens, counts=counts, k_scales=cache[2], v_scales=cache[3])
        binding.fa_fwd_cache(qr, cache[0], cache[1], table, lens, d ** -0.5, counts=counts, k_scales=cache[2], v_scales=cache[3], o=outs[0], lse=outs[1], workspace=space)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    g, gen = np.random.default_rng(2), torch.Generator(device="cuda").manual_seed(2)
    for replay in range(6):
        n = g.integers(0, T + 1, B)
        for x in (q, k, v):
            x.normal_(generator=gen)
        counts.copy_(torch.from_numpy(n.astype(np.int32)))
        positions.copy_(torch.from_numpy(g.integers(0, 5000, (3, B, T)).astype(np.int32)))
        state = [t.clone() for t in (table, *cache)]
        graph.replay()
        torch.cuda.synchronize()
        graphed = [t.clone() for t in (table, *cache, *outs)]
        for t, x in zip((table, *cache), state):
            t.copy_(x)
        step()
        torch.cuda.synchronize()
        for a, b in zip(graphed, (table, *cache, *outs)):
            assert torch.equal(a, b)
        assert outs[2].item() == 0
        c = Case.__new__(Case)
        c.dtype, c.scale, c.rows, c.q, c.lens, c.counts, c.tree = "bf16", d ** -0.5, H // H_kv * T, qr, lens.cpu().numpy(), n, None
        c.host = dict(zip(("k_pages", "v_pages", "k_scales", "v_scales"), (t.cpu().numpy() for t in cache)), block_table=table.cpu().numpy())
        c.check(*outs[:2])
        lens += counts


def test_what_does_not_fit_is_refused():
    c = Case(10, "bf16", 2, 4, 2, 1, 64, 16, [20, 5])
    k = torch.zeros((2, 2, 1, 64), dtype=torch.bfloat16, device="cuda")
    A, p = c.args, ("k_pages", "v_pages", "k_scales", "v_scales")
    write = lambda **kw: binding.fa_cache_write(k, k, **{**{n: A[n] for n in p}, "block_table": A["block_table"], "lens": A["lens"], **kw})  # noqa: E731
    read = lambda **kw: binding.fa_cache_read(**{**{n: A[n] for n in p}, "block_table": A["block_table"], "lens": A["lens"], "N": 9, **kw})  # noqa: E731
    for call in (c.run, write, read):
        for kw in (dict(k_scales=A["k_scales"][..., :1].contiguous()), dict(k_scales=None), dict(v_scales=A["k_scales"].float()), dict(k_scales=A["k_scales"].float()),
                   dict(v_pages=A["v_pages"][:3]), dict(k_pages=A["k_pages"].to(torch.bfloat16)), dict(v_scales=None), dict(k_pages=A["k_pages"][..., :16].contiguous())):
            with pytest.raises(ValueError):
                call(**kw)
    with pytest.raises(ValueError):
        c.run(q=torch.zeros((2, 4, 1, 32), dtype=torch.bfloat16, device="cuda"))
    for t in (torch.float64, torch.int32):
        with pytest.raises(ValueError):
            read(dtype=t)
