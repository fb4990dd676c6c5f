"""fa_fwd_cache against the fp64 oracle, element by element.  Whatever a row must not see holds NaN, in codes and scales too.

The bound of a row, with s_j its scores, w_j = p_j / sum p its weights and eps half a step of a type (bf16 2^-8, fp16 2^-11):
  scores    products are exact in fp32, d of them are summed: e_s = (d + 4) 2^-24 scale max_j sum |q k_j|, and 2 more roundings of
            2^-24 |s| with the scales of codes
  weights   the argument of the exponential, in units of log 2, is rounded at |s| and |m|: 2^-22 max |s|; the exponential itself 2^-21;
            numerator and sum both: e_w = 2 (e_s + 2^-22 max |s| + 2^-21)
  O         e_w sum w |v| + eps_p sum w |v| (probabilities rounded to the type of their product) + n 2^-24 max |v| in fp16 (its
            subnormals, where a probability or the quotient of two scales is small) + n 2^-24 sum w |v| (fp32 sums) + eps_o |O|
  L         e_s + 2^-22 max |s| + 2^-20 + 2^-23 |L|"""
import numpy as np
import pytest
import torch

from helpers import f64
from oracle import cache_oracle
from paper_2407_08608_amd import binding, inputs

pytestmark = pytest.mark.gpu

_T = {"bf16": torch.bfloat16, "f16": torch.float16}
_HALF = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11}


class Case:
    """A filled cache, queries, and what each row may see."""

    def __init__(self, seed, dtype, cache, B, H, H_kv, T, d, page, lens, counts=None, tree=None, width=None, table=None, k_std=1.0):
        self.dtype, self.codes, self.scale = dtype, cache == "e4m3", d ** -0.5
        g = np.random.default_rng(seed)
        self.lens = np.asarray(lens, dtype=np.int32)
        self.counts = np.full(B, T) if counts is None else np.asarray(counts)
        self.tree = tree
        top = int(max(self.lens)) + T
        width = -(-top // page) if width is None else width
        n_pages = B * width + 3
        self.table = g.permutation(n_pages)[:B * width].reshape(B, width).astype(np.int32) if table is None else table
        # everything NaN, then the tokens of every sequence, written by hand
        shape = (n_pages, H_kv, page, d)
        self.host = {"block_table": self.table}
        pages = {}
        for n in ("k", "v"):
            x = inputs.normal_tensor(seed, n, shape, "f32" if self.codes else dtype)
            if n == "k":
                x = (x.float() * k_std).to(x.dtype)
            live = np.zeros((n_pages, page), dtype=bool)
            for b in range(B):
                for p in range(max(int(self.lens[b]), 0) + min(int(self.counts[b]), T)):
                    at = cache_oracle.place({"k_pages": x, "block_table": self.table}, b, p)
                    if at is not None:
                        live[at] = True
            dead = torch.from_numpy(~live)[:, None, :].expand(n_pages, H_kv, page)
            if self.codes:
                codes, s = cache_oracle.quantise_rows(x.numpy() * g.uniform(0.05, 4.0, (n_pages, H_kv, page, 1)).astype(np.float32))
                codes, s = torch.from_numpy(codes), torch.from_numpy(s)
                codes[dead], s[dead] = 0x7F, float("nan")
                pages[n + "_pages"], pages[n + "_scales"] = codes, s
                self.host[n + "_pages"], self.host[n + "_scales"] = codes.numpy(), s.numpy()
            else:
                x[dead] = float("nan")
                pages[n + "_pages"], pages[n + "_scales"] = x, None
                self.host[n + "_pages"] = f64(x)
        self.q = inputs.normal_tensor(seed, "q", (B, H, T, d), dtype)
        self.args = dict(k_pages=pages["k_pages"].cuda(), v_pages=pages["v_pages"].cuda(), block_table=torch.from_numpy(self.table).cuda(),
                         lens=torch.from_numpy(self.lens).cuda(), scale=self.scale,
                         counts=None if counts is None else torch.from_numpy(self.counts.astype(np.int32)).cuda(),
                         k_scales=pages["k_scales"].cuda() if self.codes else None, v_scales=pages["v_scales"].cuda() if self.codes else None,
                         tree=None if tree is None else binding.fa_tree_words(torch.from_numpy(tree)).cuda())

    def run(self, **kw):
        return binding.fa_fwd_cache(**dict(dict(self.args, q=self.q.cuda()), **kw))

    def check(self, o, lse, poison=False):
        """poison: a row that sees a NaN or infinity in V has it in O, column by column"""
        q = f64(self.q)
        want = cache_oracle.attend(q, self.host, self.lens, self.counts, self.tree, self.scale)
        o, lse, d = f64(o), f64(lse), q.shape[-1]
        eps_p = 2.0 ** -11 if self.codes else _HALF[self.dtype]
        fp16_p = self.codes or self.dtype == "f16"
        for (b, h, t), (x, L, K, V) in want.items():
            got, got_l = o[b, h, t], lse[b, h, t]
            if len(K) == 0:
                assert (got == 0).all() and got_l == -np.inf, (b, h, t)
                continue
            s = self.scale * (K @ q[b, h, t])
            w = np.exp(s - L)
            top = np.abs(s).max()
            e_s = (d + 4) * 2.0 ** -24 * self.scale * (np.abs(K) @ np.abs(q[b, h, t])).max() + 2.0 ** -23 * top
            e_w = 2 * (e_s + 2.0 ** -22 * top + 2.0 ** -21)
            size, biggest = w @ np.abs(V), np.abs(V).max()
            bound = (e_w + eps_p + len(K) * 2.0 ** -24) * size + (len(K) * 2.0 ** -24 * biggest if fp16_p else 0) + _HALF[self.dtype] * np.abs(x)
            bound += 2.0 ** -25 if self.dtype == "f16" else 0
            if poison:
                fine = np.isfinite(x)
                np.testing.assert_array_equal(np.isnan(got[~fine]) | np.isinf(got[~fine]), True, err_msg=str((b, h, t)))
                np.testing.assert_array_equal(np.isnan(got[~fine]), np.isnan(x[~fine]), err_msg=str((b, h, t)))
                got, x, bound = got[fine], x[fine], bound[fine]
                ok = np.isfinite(V[:, fine]).all(axis=0)
                bound = np.where(ok, (e_w + eps_p + len(K) * 2.0 ** -23) * (w @ np.abs(V[:, fine])) + (len(K) * 2.0 ** -24 * 8 if fp16_p else 0)
                                 + _HALF[self.dtype] * np.abs(x) + 2.0 ** -25, 0)
            err = np.abs(got - x)
            assert (err <= bound).all(), ((b, h, t), err.max(), bound[np.argmax(err - bound)])
            assert abs(got_l - L) <= e_s + 2.0 ** -22 * top + 2.0 ** -20 + 2.0 ** -23 * abs(L), ((b, h, t), got_l, L)


def _random_tree(seed, B, T, empty=False):
    """Ancestors of random parents; `empty`: some tokens see nothing, not even themselves"""
    g = np.random.default_rng(seed)
    sees = np.zeros((B, T, T), dtype=bool)
    for b in range(B):
        for t in range(T):
            parent = int(g.integers(-1, t)) if t else -1
            if parent >= 0:
                sees[b, t] = sees[b, parent]
            sees[b, t, t] = True
        if empty:
            sees[b, g.random(T) < 0.4] = False
    return sees


_KINDS = [("bf16", "bf16"), ("f16", "f16"), ("bf16", "e4m3"), ("f16", "e4m3")]


@pytest.mark.parametrize("dtype,cache", _KINDS)
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("B,H,H_kv,page,lens", [
    (1, 1, 1, 16, [0]),                      # the token itself
    (4, 4, 4, 16, [1, 15, 16, 17]),          # around a page
    (5, 8, 2, 16, [30, 31, 32, 33, 63]),     # around a tile of 32 keys, with their own key
    (3, 6, 1, 48, [127, 500, 0]),            # pages that no tile divides
    (2, 32, 2, 128, [777, 1290]),            # 16 heads to a key/value head
    (1, 40, 1, 64, [333]),                   # more rows than a tile
])
def test_one_token(dtype, cache, d, B, H, H_kv, page, lens):
    c = Case(100 + d, dtype, cache, B, H, H_kv, 1, d, page, lens)
    c.check(*c.run())


@pytest.mark.parametrize("dtype,cache", _KINDS)
@pytest.mark.parametrize("d,B,H,H_kv,T,page,lens,counts", [
    (64, 2, 4, 4, 2, 16, [0, 31], None),
    (128, 3, 4, 2, 5, 16, [0, 100, 30], [5, 0, 3]),
    (64, 2, 6, 2, 33, 32, [250, 15], [33, 32]),
    (256, 2, 4, 1, 13, 16, [99, 640], [13, 1]),
    (128, 1, 8, 2, 64, 64, [1000], None),
    (128, 2, 2, 1, 100, 16, [5, 300], [77, 100]),
    (64, 1, 2, 2, 256, 48, [123], None),
])
def test_chains_and_trees(dtype, cache, d, B, H, H_kv, T, page, lens, counts):
    for tree in (None, _random_tree(T, B, T), _random_tree(T, B, T, empty=True)):
        c = Case(200 + T, dtype, cache, B, H, H_kv, T, d, page, lens, counts, tree)
        o, lse = torch.full(c.q.shape, 7.0, dtype=c.q.dtype, device="cuda"), torch.full(c.q.shape[:3], 7.0, device="cuda")
        got = c.run(o=o, lse=lse)
        assert got[0] is o and got[1] is lse
        c.check(o, lse)
        for b in range(B):
            assert (o[b, :, c.counts[b]:] == 7).all() and (lse[b, :, c.counts[b]:] == 7).all()


def test_one_tree_for_all_sequences():
    tree = _random_tree(1, 1, 21)
    c = Case(1, "bf16", "bf16", 3, 4, 2, 21, 64, 16, [50, 0, 77], tree=np.repeat(tree, 3, axis=0))
    a = c.run()
    b = c.run(tree=binding.fa_tree_words(torch.from_numpy(tree)).cuda())
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    c.check(*a)


@pytest.mark.parametrize("dtype,cache", _KINDS)
def test_pages_that_are_none_and_places_past_the_table(dtype, cache):
    B, T, page, width = 4, 6, 16, 4
    table = np.array([[0, -1, 2, 3], [-1, -1, -1, -1], [4, 5, 6, 19], [7, 8, 9, 10]], dtype=np.int32)  # of 19 pages
    # a hole; nothing at all; the last page is none; new tokens past the last place, and lengths that are far past it or negative
    for lens in ([60, 20, 50, 61], [10, 0, 3, 64], [2 ** 31 - 1, 5, 64, -5]):
        c = Case(7, dtype, cache, B, 4, 2, T, 64, page, np.minimum(lens, 64), tree=_random_tree(3, B, T), width=width, table=table)
        c.lens = np.asarray(lens, dtype=np.int64)
        at_most = np.where(c.lens > 64, 64, c.lens)
        o, lse = c.run(lens=torch.tensor(lens, dtype=torch.int32).cuda())
        c.lens = at_most
        c.check(o, lse)


@pytest.mark.parametrize("dtype,cache", _KINDS)
@pytest.mark.parametrize("d,H,H_kv,T,lens", [(128, 2, 2, 1, [70001, 40]), (64, 16, 2, 1, [33000, 9000]), (256, 8, 1, 3, [20011, 1]),
                                             (128, 4, 1, 40, [9000, 300])])
def test_long_caches_are_divided_and_joined(dtype, cache, d, H, H_kv, T, lens):
    c = Case(300 + d, dtype, cache, 2, H, H_kv, T, d, 64, lens, tree=_random_tree(T, 2, T) if T > 1 else None)
    o, lse = c.run()
    c.check(o, lse)
    # the expected length only divides the work; too low a one is still right
    for max_len in (1, 5000, 1 << 20):
        c.check(*c.run(max_len=max_len))
    assert torch.equal(c.run()[0], o) and torch.equal(c.run()[1], lse)  # repeatable


@pytest.mark.parametrize("dtype,cache,d,B,H,H_kv,T,lens", [
    ("bf16", "bf16", 64, 48, 8, 8, 1, (1, 400)),      # shares that end inside sequences: some teams have two
    ("f16", "e4m3", 128, 48, 16, 8, 1, (1, 400)),
    ("bf16", "e4m3", 64, 70, 4, 2, 3, (0, 700)),      # more sequences than a wave has lanes
    ("f16", "f16", 64, 130, 2, 1, 1, (0, 900)),
    ("bf16", "bf16", 128, 40, 12, 4, 7, (1, 600)),    # 21 rows
    ("f16", "e4m3", 64, 24, 12, 4, 16, (1, 500)),     # 48 rows
    ("bf16", "bf16", 64, 20, 16, 4, 20, (1, 700)),    # 80 rows, one group of them
    ("bf16", "e4m3", 128, 9, 8, 2, 60, (1, 900)),     # 240 rows, two
    ("f16", "f16", 256, 7, 4, 2, 70, (1, 600)),       # 140 rows, two
    ("bf16", "bf16", 256, 30, 32, 4, 2, (1, 500)),
])
def test_shares_of_many_sequences(dtype, cache, d, B, H, H_kv, T, lens):
    g = np.random.default_rng(B + d)
    lens = g.integers(lens[0], lens[1], B)
    lens[B // 2] = 0
    counts = None if T == 1 else g.integers(0, T + 1, B)
    c = Case(500 + B, dtype, cache, B, H, H_kv, T, d, 16, lens, counts, _random_tree(B, B, T) if T > 1 else None)
    o, lse = torch.full(c.q.shape, 7.0, dtype=c.q.dtype, device="cuda"), torch.full(c.q.shape[:3], 7.0, device="cuda")
    for max_len in (1 << 20, 0):  # teams, and whatever the rule says
        o.fill_(7.0)
        lse.fill_(7.0)
        c.run(o=o, lse=lse, max_len=max_len)
        c.check(o, lse)
        for b in range(B):
            assert (o[b, :, c.counts[b]:] == 7).all() and (lse[b, :, c.counts[b]:] == 7).all()


@pytest.mark.parametrize("dtype,cache", _KINDS)
@pytest.mark.parametrize("d,H,H_kv,T", [(64, 8, 2, 40), (128, 2, 2, 9), (128, 16, 4, 12), (256, 8, 2, 20)])
@pytest.mark.parametrize("max_len", [0, 1 << 20])
def test_unseen_values_in_every_form(dtype, cache, d, H, H_kv, T, max_len):
    # values that are not finite in V of new tokens, in 16 to 160 rows, in one launch and joined
    tree = _random_tree(T, 2, T)
    c = Case(600 + T, dtype, cache, 2, H, H_kv, T, d, 16, [300, 21], tree=tree)
    for b in range(2):
        for u, col, x in ((2, 5, np.nan), (4, d - 1, np.inf), (5, 33, -np.inf), (T - 2, 33, np.inf)):
            page, slot = cache_oracle.place(c.host, b, int(c.lens[b]) + u)
            if cache == "e4m3":
                c.args["v_pages"][page, :, slot, col] = 0x7F
                c.host["v_pages"][page, :, slot, col] = 0x7F
            else:
                c.args["v_pages"][page, :, slot, col] = float(x)
                c.host["v_pages"][page, :, slot, col] = x
    c.check(*c.run(max_len=max_len), poison=True)


def test_rising_scores_and_large_ones():
    # every key block raises the maximum; scores up to several hundred
    for dtype, cache in _KINDS:
        c = Case(9, dtype, cache, 1, 4, 2, 3, 64, 16, [700], k_std=30.0 if cache != "e4m3" else 8.0)
        c.check(*c.run())


def test_values_that_a_row_does_not_see_do_not_reach_it():
    # NaN and infinities in K and V of new tokens that some rows see and others do not
    T, d = 12, 64
    tree = _random_tree(5, 1, T)
    for dtype in ("bf16", "f16"):
        c = Case(11, dtype, dtype, 1, 4, 2, T, d, 16, [37], tree=tree)
        for u, col, x in ((3, 5, np.nan), (4, 6, np.inf), (5, 7, -np.inf), (8, 40, np.inf), (9, 63, np.nan)):
            page, slot = cache_oracle.place(c.host, 0, 37 + u)
            c.args["v_pages"][page, :, slot, col] = x
            c.host["v_pages"][page, :, slot, col] = x
        c.check(*c.run(), poison=True)
        # a NaN key: the rows that see it are NaN, the others as if it were not there
        page, slot = cache_oracle.place(c.host, 0, 37 + 10)
        before = c.run()
        c.args["k_pages"][page, :, slot, 3] = float("nan")
        after = c.run()
        for t in range(T):
            if tree[0, t, 10]:
                assert torch.isnan(after[1][0, :, t]).all() and torch.isnan(after[0][0, :, t]).all()
            else:
                assert torch.equal(before[1][0, :, t], after[1][0, :, t])
                assert torch.equal(before[0][0, :, t].view(torch.int16), after[0][0, :, t].view(torch.int16))
    # codes: NaN codes, and scales that are NaN or infinite, of a new token
    c = Case(12, "bf16", "e4m3", 1, 4, 2, T, d, 16, [37], tree=tree)
    clean = c.run()
    for change in ("code", "nan", "inf"):
        page, slot = cache_oracle.place(c.host, 0, 37 + 4)
        kv = {n: c.args[n].clone() for n in ("v_pages", "v_scales", "k_scales")}
        if change == "code":
            kv["v_pages"][page, :, slot] = 0x7F
        else:
            kv["v_scales"][page, :, slot] = kv["k_scales"][page, :, slot] = float(change)
        got = c.run(**kv)
        for t in range(T):
            if not tree[0, t, 4]:
                assert torch.equal(got[0][0, :, t], clean[0][0, :, t]) and torch.equal(got[1][0, :, t], clean[1][0, :, t])
            else:
                assert not torch.isfinite(got[0][0, :, t]).all()


def test_scales_of_very_different_size():
    # e4m3: values of one token 2^60 times another's
    c = Case(13, "bf16", "e4m3", 1, 2, 1, 4, 64, 16, [90])
    for name in ("k_scales", "v_scales"):
        s = c.args[name].cpu().numpy()
        power = np.random.default_rng(1).integers(-50, 10, s.shape) if name == "v_scales" else np.random.default_rng(2).integers(-10, 1, s.shape)
        s = (s * 2.0 ** power).astype(np.float32)
        c.args[name], c.host[name] = torch.from_numpy(s).cuda(), s
    c.check(*c.run())


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
def test_strided_queries_and_outputs(cache):
    B, H, H_kv, T, d = 2, 8, 2, 7, 128
    c = Case(14, "bf16", cache, B, H, H_kv, T, d, 16, [130, 20], counts=[7, 4])
    want = c.run(o=torch.zeros((B, H, T, d), device="cuda", dtype=torch.bfloat16), lse=torch.zeros((B, H, T), device="cuda"))
    # a projection's [B, T, H, d] in, and out into one with room around it
    q = c.q.cuda().transpose(1, 2).contiguous().transpose(1, 2)
    room = torch.zeros((B, T + 2, H + 1, d + 16), device="cuda", dtype=torch.bfloat16)
    o = room[:, 1:-1, 1:, 8:-8].transpose(1, 2)
    got = c.run(q=q, o=o, lse=torch.zeros((B, H, T), device="cuda"))
    assert got[0] is o and torch.equal(o, want[0]) and torch.equal(got[1], want[1])
    o.zero_()
    assert not room.any()
    one = c.q[:1].cuda().expand(B, H, T, d)
    assert torch.equal(c.run(q=one, o=torch.zeros_like(want[0]))[0][0], want[0][0])


def test_workspaces():
    c = Case(15, "f16", "f16", 2, 2, 1, 2, 128, 32, [6000, 5500])
    want = c.run()
    need = binding.fa_fwd_cache_workspace_bytes(2, 2, 1, 2, 128, 32 * c.table.shape[1], binding.FA_F16)
    ws = torch.full((need + 64,), 255, dtype=torch.uint8, device="cuda")
    got = c.run(workspace=ws[:need])
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and (ws[need:] == 255).all()
    if need:
        with pytest.raises(binding.FaError) as e:
            c.run(workspace=ws[:need - 1])
        assert e.value.status == 6


def test_a_decoding_step_and_a_drafted_tree_as_a_program_makes_them():
    """Prompt and drafts through rotation, cache and attention, and the dense path for comparison: the accepted path of a drafted
    tree is what a causal forward gives for those tokens.  bf16: both sides round P (2^-8 of the weights, at most so much of
    sum w |v|) and O (2^-8 |O|), and nothing else to fewer than 24 bits."""
    B, H, H_kv, N, d, page, T = 2, 8, 2, 150, 128, 16, 5
    parents = [-1, 0, 0, 1, 2]  # two paths: 0 1 3 and 0 2 4
    depth = [0, 1, 1, 2, 2]
    tree = np.zeros((1, T, T), dtype=bool)
    for t, p in enumerate(parents):
        tree[0, t] = tree[0, p] if p >= 0 else False
        tree[0, t, t] = True
    words = binding.fa_tree_words(torch.from_numpy(tree)).cuda()
    f, amplitude = binding.fa_rope_frequencies(d, 10000.0, binding.FA_ROPE_BY_PARTS, 4.0, 4096)
    q, k, v = (inputs.normal_tensor(21, n, (B, h, N + T, d), "bf16").cuda() for n, h in (("q", H), ("k", H_kv), ("v", H_kv)))
    width = -(-(N + T) // page)
    table = torch.from_numpy(np.random.default_rng(1).permutation(B * width).reshape(B, width).astype(np.int32)).cuda()
    kp, vp = (torch.full((B * width, H_kv, page, d), float("nan"), device="cuda", dtype=torch.bfloat16) for _ in range(2))
    lens = torch.zeros(B, dtype=torch.int32, device="cuda")
    # the prompt
    pq, pk = binding.fa_rope(q[:, :, :N], f, k=k[:, :, :N], amplitude=amplitude)
    binding.fa_cache_write(pk, v[:, :, :N], kp, vp, table, lens)
    lens += N
    # the draft
    at = (lens[:, None] + torch.tensor(depth, dtype=torch.int32, device="cuda")).contiguous()
    tq, tk = binding.fa_rope(q[:, :, N:], f, k=k[:, :, N:], positions=at, amplitude=amplitude)
    binding.fa_cache_write(tk, v[:, :, N:], kp, vp, table, lens)
    o, lse = binding.fa_fwd_cache(tq, kp, vp, table, lens, d ** -0.5, tree=words, max_len=N + T)
    for path in ([0, 1, 3], [0, 2, 4]):
        rows = torch.tensor(path, device="cuda")
        Q, K, V = (torch.cat((a, b.index_select(2, rows)), 2) for a, b in ((pq, tq), (pk, tk), (v[:, :, :N], v[:, :, N:])))
        od, ld = binding.fa_fwd_gqa(Q, K, V, d ** -0.5, True)
        x, y = f64(o.index_select(2, rows)), f64(od[:, :, N:])
        K, V, Q = f64(K), f64(V), f64(Q[:, :, N:])
        for b in range(B):
            for h in range(H):
                for i in range(3):
                    s = d ** -0.5 * (K[b, h // 4, :N + i + 1] @ Q[b, h, i])
                    w = np.exp(s - s.max())
                    bound = 2 * 2.0 ** -8 * ((w / w.sum()) @ np.abs(V[b, h // 4, :N + i + 1]) * 1.01 + np.abs(y[b, h, i])) + 1e-6
                    assert (np.abs(x[b, h, i] - y[b, h, i]) <= bound).all()
        np.testing.assert_allclose(f64(lse.index_select(2, rows)), f64(ld[:, :, N:]), atol=1e-4)
    # the accepted path goes to its places; the next single token sees it
    rows = torch.tensor([0, 2, 4], device="cuda")
    binding.fa_cache_write(tk.index_select(2, rows), v[:, :, N:].index_select(2, rows), kp, vp, table, lens)
    lens += 3
    back = binding.fa_cache_read(kp, vp, table, lens, N + 3)
    assert torch.equal(back[0], torch.cat((pk, tk.index_select(2, rows)), 2)) and torch.equal(back[1][:, :, :N], v[:, :, :N])


def test_replayed_steps_match_eager_ones():
    """One decoding step captured into a graph and replayed over growing lengths, eager work and synchronisations in between."""
    B, H, H_kv, d, page, width = 3, 4, 2, 128, 16, 300
    f, _ = binding.fa_rope_frequencies(d)
    q, k, v = (torch.zeros((B, h, 1, d), device="cuda", dtype=torch.bfloat16) for h in (H, H_kv, H_kv))
    table = torch.arange(B * width, dtype=torch.int32, device="cuda").view(B, width)
    start = [torch.randint(0, 100, (B * width, H_kv, page, d), dtype=torch.uint8, device="cuda") for _ in range(2)]
    start += [torch.rand((B * width, H_kv, page), device="cuda") * 0.02 + 0.001 for _ in range(2)]
    pages = [t.clone() for t in start]
    lens = torch.zeros((B,), dtype=torch.int32, device="cuda")
    o, lse = torch.zeros_like(q), torch.zeros((B, H, 1), device="cuda")
    need = binding.fa_fwd_cache_workspace_bytes(B, H, H_kv, 1, d, width * page, binding.FA_FP8_E4M3)
    ws = torch.zeros((max(need, 16),), dtype=torch.uint8, device="cuda")
    tq, tk = torch.zeros_like(q), torch.zeros_like(k)

    def step():
        binding.fa_rope(q, f, k=k, positions=lens[:, None].contiguous(), q_out=tq, k_out=tk)
        binding.fa_cache_write(tk, v, pages[0], pages[1], table, lens, k_scales=pages[2], v_scales=pages[3])
        binding.fa_fwd_cache(tq, pages[0], pages[1], table, lens, 0.1, k_scales=pages[2], v_scales=pages[3], o=o, lse=lse, workspace=ws)

    def fill(i):
        for n, t in (("q", q), ("k", k), ("v", v)):
            t.copy_(inputs.normal_tensor(400 + i, n, tuple(t.shape), "bf16"))
        lens.copy_(torch.tensor([7 + i, 4000 + 16 * i, 1500 * i], dtype=torch.int32))

    eager = []
    for i in range(3):
        fill(i)
        step()
        eager.append((o.clone(), lse.clone()))
    done = [t.clone() for t in pages]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(2):
        for t, s in zip(pages, start):
            t.copy_(s)
        for i in range(3):
            fill(i)
            o.fill_(float("nan"))
            ws.fill_(255)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(o, eager[i][0]) and torch.equal(lse, eager[i][1]), i
        assert all(torch.equal(a, b) for a, b in zip(pages, done))


def test_calls_on_another_stream():
    c = Case(16, "bf16", "bf16", 2, 8, 2, 1, 128, 16, [5000, 300])
    want = c.run()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = [c.run() for _ in range(3)]
    other = c.run()
    side.synchronize()
    torch.cuda.synchronize()
    for o, lse in got + [other]:
        assert torch.equal(o, want[0]) and torch.equal(lse, want[1])


def test_the_binding_refuses_what_does_not_fit():
    c = Case(17, "bf16", "bf16", 2, 4, 2, 3, 64, 16, [20, 9])
    q = c.q.cuda()
    o, lse = c.run()
    words = torch.zeros((2, 3, 1), dtype=torch.int32, device="cuda")
    for kw in (dict(q=q.half()), dict(q=q.float()), dict(q=q[0]), dict(q=q[..., ::2]), dict(q=q.cpu()), dict(tree=words[:, :2]), dict(tree=words.long()),
               dict(tree=torch.zeros((3, 3, 1), dtype=torch.int32, device="cuda")), dict(o=o.half()), dict(o=o[:, :2]), dict(lse=lse.double()),
               dict(lse=lse[:1]), dict(k_scales=lse, v_scales=lse), dict(lens=c.args["lens"][:1]), dict(counts=c.args["lens"].long()),
               dict(workspace=lse), dict(v_pages=c.args["v_pages"].half()), dict(k_pages=c.args["k_pages"].half(), v_pages=c.args["v_pages"].half())):
        with pytest.raises((ValueError, binding.FaError)):
            c.run(**kw)
    for kw in (dict(scale=-1.0), dict(max_len=-1), dict(q=q[:, :3])):
        with pytest.raises(binding.FaError):
            c.run(**kw)
