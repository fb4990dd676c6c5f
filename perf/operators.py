"""Rotary positions, a paged key/value cache and attention over it: the calls that a serving or training program makes next to
dense attention, as cases to be timed and checked.  A case is a dict of plain values; `op` says which call:

  rope    Q and K rotated by their tokens' positions, or (`backward`) their gradients rotated back
  write   K and V of new tokens put into the pages of a cache, as they are or as e4m3 codes with a scale per token and head
  read    the cached K and V of a batch gathered from their pages, as dense tensors
  attend  attention of T new tokens per sequence over a cache that holds them and the tokens before them; T > 1 with a tree mask

q [B, H, T, d], k and v [B, H_kv, T, d]; pages [n_pages, H_kv, page_size, d]; d in {64, 128, 256}, scale d^-1/2.
"""
import math
import random

import torch

own = False

_DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_ELEM = {"f32": 4, "bf16": 2, "f16": 2, "e4m3": 1}


def _rope(name, dtype, B, H, H_kv, N, d, rot, interleaved, scaled, far, backward, token_major):
    c = {"op": "rope", "dtype": dtype, "B": B, "H": H, "H_kv": H_kv, "N": N, "d": d, "rot": rot, "interleaved": interleaved,
         "scaled": scaled, "far": far, "backward": backward, "token_major": token_major}
    return {"name": name, **c} if name else c


def _cached(name, op, dtype, cache, B, H, H_kv, T, d, page, most, least):
    """T: new tokens per sequence (read: unused, 0); most, least: bounds of the lengths that the cache holds before them"""
    c = {"op": op, "dtype": dtype, "cache": cache, "B": B, "H": H, "H_kv": H_kv, "T": T, "d": d, "page": page, "most": most, "least": least}
    return {"name": name, **c} if name else c


def listed():
    return [
        # one decoding step of a small batch: a token each, far into its sequence; launch and latency decide
        _rope("rope_token", "bf16", 8, 16, 4, 1, 128, 128, False, False, 100000, False, False),
        # 16k tokens of prefill, hidden size 2048, with frequencies scaled for a longer context
        _rope("rope_prompt", "bf16", 4, 16, 16, 4096, 128, 128, False, True, 0, False, False),
        # gradients of a training batch of odd length: half of each narrow head rotated, interleaved pairs, projections' layout
        _rope("rope_grad", "f16", 4, 32, 32, 1300, 64, 32, True, False, 0, True, True),
        # one token of each sequence of a batch appended to an e4m3 cache
        _cached("write_token", "write", "bf16", "e4m3", 16, 16, 4, 1, 128, 16, 4000, 100),
        # prompts of ragged lengths written to a fresh e4m3 cache: 16k tokens at most
        _cached("write_prompt", "write", "bf16", "e4m3", 4, 16, 16, 4096, 128, 64, 0, 0),
        # two short prefixes read back from a 16-bit cache
        _cached("read_prefix", "read", "f16", "f16", 2, 16, 8, 0, 64, 16, 333, 100),
        # long contexts read back from an e4m3 cache for a dense pass
        _cached("read_long", "read", "bf16", "e4m3", 4, 16, 8, 0, 128, 64, 8192, 3001),
        # one request, one token, a short cache
        _cached("attend_token", "attend", "bf16", "bf16", 1, 16, 16, 1, 64, 16, 333, 333),
        # a decoding step of a full batch with shared key/value heads, ragged lengths, small pages
        _cached("attend_batch", "attend", "bf16", "bf16", 32, 32, 8, 1, 128, 16, 4096, 500),
        # a few very long contexts in an e4m3 cache, widest heads: few rows, the keys have to be split
        _cached("attend_long", "attend", "bf16", "e4m3", 2, 16, 2, 1, 256, 64, 65536, 50000),
        # verifying small drafted trees of odd size
        _cached("tree_small", "attend", "f16", "f16", 8, 16, 4, 13, 128, 32, 4096, 1000),
        # verifying the largest drafted trees of a batch over long contexts: the matrix products decide
        _cached("tree_large", "attend", "bf16", "bf16", 4, 32, 4, 64, 128, 64, 16384, 12000),
    ]


# no drawn case costs more than the largest listed ones
_MOST_BYTES, _MOST_FLOPS = 2.6e8, 5.5e10


def _size(rng, lo, hi):
    """Spread over the logarithm; odd values as common as regular ones"""
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return max(lo, n // 16 * 16) if n > 64 and rng.random() < 0.4 else n


def draw(rng):
    while True:
        op = rng.choice(["rope", "write", "read", "attend", "attend", "attend"])
        dtype, d = rng.choice(["bf16", "bf16", "f16"]), rng.choice([64, 128, 128, 256])
        B, H = _size(rng, 1, 32), rng.choice([2, 4, 8, 12, 16, 32])
        H_kv = rng.choice([h for h in (1, 2, 4, 8, 16, 32) if H % h == 0])
        cache, page = rng.choice(["e4m3", dtype]), rng.choice([16, 16, 32, 48, 64, 128])
        if op == "rope":
            dtype = rng.choice([dtype, dtype, "f32"])
            c = _rope(None, dtype, B, H, H_kv, _size(rng, 1, 8192), d, rng.choice([d, d, d // 2, d // 4]), rng.random() < 0.5,
                      rng.random() < 0.5, rng.choice([0, 1000, 120000]), rng.random() < 0.4, rng.random() < 0.4)
        elif op == "write":
            most = _size(rng, 1, 8192)
            c = _cached(None, op, dtype, cache, B, H, H_kv, _size(rng, 1, 8192), d, page, most, rng.randint(0, most))
        elif op == "read":
            most = _size(rng, 1, 16384)
            c = _cached(None, op, dtype, cache, B, H, H_kv, 0, d, page, most, rng.randint(1, most))
        else:
            most = _size(rng, 1, 65536)
            c = _cached(None, op, dtype, cache, B, H, H_kv, rng.choice([1, 1, _size(rng, 2, 64), _size(rng, 2, 64)]), d, page, most,
                        rng.randint(most // 2, most))
        w = work(c)
        # (the plain form of attention holds the gathered cache and the scores in 32 bits)
        scores = c["B"] * c["H"] * c.get("T", 1) * (c.get("most", 0) + 64)
        dense = c["B"] * c["H_kv"] * (c.get("most", 0) + c.get("T", 0)) * c["d"]
        if w["bytes"] <= _MOST_BYTES and w["flops"] <= _MOST_FLOPS and scores <= 1 << 28 and dense <= 1 << 27:
            return c


def _lens(c):
    """The lengths before the new tokens, and how many of the T new ones each sequence has (some fewer, as in a padded batch).
    They go by the case alone, so that work() knows them."""
    r = random.Random("%(op)s %(B)d %(T)d %(most)d %(least)d" % c)
    lens = [c["most"]] + [r.randint(c["least"], c["most"]) for _ in range(c["B"] - 1)]
    counts = [c["T"]] + [r.randint((c["T"] + 1) // 2, c["T"]) for _ in range(c["B"] - 1)]
    return lens, counts


def work(case):
    c = case
    e = _ELEM[c["dtype"]]
    if c["op"] == "rope":  # each element in and out; two products and a sum for each that is rotated
        n = c["B"] * (c["H"] + c["H_kv"]) * c["N"]
        return {"bytes": 2.0 * n * c["d"] * e + (4.0 * c["B"] * c["N"] if c["far"] else 0), "flops": 3.0 * n * c["rot"]}
    lens, counts = _lens(c)
    row = c["d"] * _ELEM[c["cache"]] + (4 if c["cache"] == "e4m3" else 0)  # a cached token of one head, K or V
    if c["op"] == "write":
        n = 2.0 * sum(counts) * c["H_kv"]
        return {"bytes": n * (c["d"] * e + row), "flops": 2.0 * n * c["d"]}
    if c["op"] == "read":
        n = 2.0 * sum(lens) * c["H_kv"]
        return {"bytes": n * (c["d"] * e + row), "flops": n * c["d"]}
    keys = 2.0 * c["H_kv"] * sum(a + b for a, b in zip(lens, counts)) * row
    rows = c["H"] * sum(counts) * (2 * c["d"] * e + 4)
    return {"bytes": keys + rows, "flops": sum(4.0 * c["H"] * b * (a + b) * c["d"] for a, b in zip(lens, counts))}


def _frequencies(c):
    """Radians per token of each rotated pair, in 64 bits: base 10000, scaled by parts for 4 times the trained 4096 tokens where asked
    (pairs that turn often over those stay, slow ones are stretched), and the amplitude that goes with it."""
    f = 10000.0 ** (-torch.arange(0, c["rot"], 2, dtype=torch.float64) / c["rot"])
    if not c["scaled"]:
        return f, 1.0
    keep = ((4096 * f / (2 * math.pi) - 1) / 31).clamp(0, 1)
    return f * ((1 - keep) / 4 + keep), 0.1 * math.log(4.0) + 1


def prepare(case, seed):
    c = dict(case)
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 1000003 + 29)
    dt = _DTYPES[c["dtype"]]

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)

    def heads(n, tokens, token_major=False):
        """[B, n, tokens, d], some channels larger than others as in keys; token_major: a view of [B, tokens, n, d]"""
        x = normal(c["B"], tokens, n, c["d"]) if token_major else normal(c["B"], n, tokens, c["d"])
        x = (x * (0.5 + torch.rand(c["d"], generator=g, device="cuda"))).to(dt)
        return x.transpose(1, 2) if token_major else x

    s = {"case": c}
    if c["op"] == "rope":
        f, s["amplitude"] = _frequencies(c)
        s["inv_freq"] = f.cuda()
        s["q"], s["k"] = heads(c["H"], c["N"], c["token_major"]), heads(c["H_kv"], c["N"], c["token_major"])
        s["positions"] = None
        if c["far"]:  # sequences that stand at places of their own
            first = torch.randint(0, c["far"], (c["B"], 1), generator=g, device="cuda", dtype=torch.int32)
            s["positions"] = (first + torch.arange(c["N"], device="cuda", dtype=torch.int32)).contiguous()
        return s

    lens, counts = _lens(c)
    B, T, H_kv, d, page = c["B"], c["T"], c["H_kv"], c["d"], c["page"]
    per = -(-(c["most"] + T) // page)  # pages of the longest sequence: the width of the table
    n_pages = B * per + 3
    order = torch.randperm(n_pages, generator=g, device="cuda")[:B * per]
    s["table"] = order.view(B, per).to(torch.int32)
    s["lens"] = torch.tensor(lens, dtype=torch.int32).cuda()
    s["counts"] = torch.tensor(counts, dtype=torch.int32).cuda() if min(counts) < T else None
    for n in ("k", "v"):
        x = normal(n_pages, H_kv, page, d) * (0.5 + torch.rand(d, generator=g, device="cuda"))
        if c["cache"] == "e4m3":
            amax = x.abs().amax(-1)
            s[n + "_scales"] = amax / 448
            s[n + "_pages"] = (x * (448 / amax)[..., None]).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
        else:
            s[n + "_scales"], s[n + "_pages"] = None, x.to(dt)
    if c["op"] == "write":
        s["k"], s["v"] = heads(H_kv, T), heads(H_kv, T)
    elif c["op"] == "read":  # rows behind a sequence's end stay as they are: zeros here
        s["k"], s["v"] = (torch.zeros((B, H_kv, c["most"], d), device="cuda", dtype=dt) for _ in range(2))
    else:
        s["q"] = heads(c["H"], T)
        s["o"] = s["lse"] = s["tree"] = None
        if s["counts"] is not None:  # rows of a padded batch stay as they are
            s["o"], s["lse"] = torch.zeros_like(s["q"]), torch.zeros(s["q"].shape[:3], device="cuda")
        if T > 1:
            r = random.Random(int(seed) * 7 + T)
            words = torch.zeros((B, T, (T + 31) // 32), dtype=torch.int64)
            for b in range(B):
                sees = []
                for t in range(T):  # each drafted token sees itself and what its parent sees; some have no drafted parent
                    parent = r.randint(max(-1, t - 8), t - 1)
                    sees.append((1 << t) | (sees[parent] if parent >= 0 else 0))
                    for w in range(words.shape[2]):
                        word = (sees[t] >> (32 * w)) & 0xFFFFFFFF
                        words[b, t, w] = word - (1 << 32) if word >> 31 else word
            s["tree"] = words.to(torch.int32).cuda()
    return s


# ------------------------------------------------------------------------------------------
# The plain form: elementary operations in 32 bits


def _plain_rope(s):
    c = s["case"]
    at = s["positions"] if s["positions"] is not None else torch.arange(c["N"], device="cuda")[None, :]
    angle = at.double()[:, None, :, None] * s["inv_freq"]  # (64 bits: far positions)
    cos, sin = (torch.cos(angle) * s["amplitude"]).float(), (torch.sin(angle) * s["amplitude"]).float()
    if c["backward"]:
        sin = -sin

    def turned(x):
        r = x[..., :c["rot"]].float()
        a, b = (r[..., 0::2], r[..., 1::2]) if c["interleaved"] else (r[..., :c["rot"] // 2], r[..., c["rot"] // 2:])
        y, z = a * cos - b * sin, a * sin + b * cos
        y = torch.stack((y, z), -1).flatten(-2) if c["interleaved"] else torch.cat((y, z), -1)
        return torch.cat((y.to(x.dtype), x[..., c["rot"]:]), -1)

    return turned(s["q"]), turned(s["k"])


def _places(s, first, tokens):
    """Page and slot [B, tokens] of the tokens from `first` [B, 1] on"""
    at = first + torch.arange(tokens, device="cuda")
    return torch.gather(s["table"].long(), 1, at // s["case"]["page"]), at % s["case"]["page"]


def _plain_write(s):
    c = s["case"]
    page, slot = _places(s, s["lens"][:, None].long(), c["T"])
    there = None if s["counts"] is None else torch.arange(c["T"], device="cuda")[None, :] < s["counts"][:, None]

    def put(into, x):  # x [B, H_kv, T, ...]
        x = x.transpose(1, 2)
        if there is not None:
            x = torch.where(there.reshape(there.shape + (1,) * (x.dim() - 2)), x, into[page, :, slot])
        into[page, :, slot] = x

    def one(x, pages, scales):
        if scales is None:
            put(pages, x)
            return
        x = x.float()
        amax = x.abs().amax(-1)
        full = amax > 0
        scale, factor = torch.where(full, amax / 448, 1.0), torch.where(full, 448 / amax, 1.0)
        put(pages, (x * factor[..., None]).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8))
        put(scales, scale)

    one(s["k"], s["k_pages"], s["k_scales"])
    one(s["v"], s["v_pages"], s["v_scales"])


def _gathered(s, pages, scales, tokens):
    """[B, H_kv, tokens, d] in 32 bits: the first `tokens` of each sequence (behind its end whatever its last page holds)"""
    B, H_kv, d = s["case"]["B"], s["case"]["H_kv"], s["case"]["d"]
    per = -(-tokens // s["case"]["page"])
    table = s["table"][:, :per].long()
    x = pages[table]  # [B, per, H_kv, page, d]
    x = x.float() if scales is None else x.view(torch.float8_e4m3fn).float() * scales[table][..., None]
    return x.transpose(1, 2).reshape(B, H_kv, per * s["case"]["page"], d)[:, :, :tokens]


def _plain_read(s):
    n = s["k"].shape[2]
    there = (torch.arange(n, device="cuda")[None, :] < s["lens"][:, None])[:, None, :, None]
    return tuple(torch.where(there, _gathered(s, s[x + "_pages"], s[x + "_scales"], n).to(s[x].dtype), s[x]) for x in ("k", "v"))


def _plain_attend(s):
    c = s["case"]
    B, H, H_kv, T, d = c["B"], c["H"], c["H_kv"], c["T"], c["d"]
    keys = c["most"] + T
    K, V = (_gathered(s, s[x + "_pages"], s[x + "_scales"], keys) for x in ("k", "v"))
    q = s["q"].float().view(B, H_kv, H // H_kv * T, d)
    score = torch.matmul(q, K.transpose(-1, -2)).view(B, H, T, keys) * d ** -0.5
    new = (torch.arange(keys, device="cuda")[None, :] - s["lens"][:, None])[:, None, :]  # number among the new tokens
    seen = new < 0
    if s["tree"] is None:
        seen = seen | (new <= torch.arange(T, device="cuda")[None, :, None])
    else:
        u = new.clamp(0, T - 1).long().expand(B, T, keys)
        bit = torch.gather(s["tree"], 2, u // 32) >> (u % 32).int() & 1
        seen = seen | ((bit != 0) & (new < T))
    score = score.masked_fill(~seen[:, None], -math.inf)
    m = score.amax(-1, keepdim=True)
    p = torch.exp(score - m)
    total = p.sum(-1, keepdim=True)
    # (a cached value that a row does not see is none of its business: those of the pages' free slots are finite)
    o = torch.matmul(p.view(B, H_kv, H // H_kv * T, keys), V).view(B, H, T, d) / total
    o, lse = o.to(s["q"].dtype), (m + torch.log(total))[..., 0]
    if s["counts"] is not None:
        there = (torch.arange(T, device="cuda")[None, :] < s["counts"][:, None])[:, None]
        o, lse = torch.where(there[..., None], o, s["o"]), torch.where(there, lse, s["lse"])
    return o, lse


def _cache_as_values(s):
    if s["k_scales"] is None:
        return s["k_pages"], s["v_pages"]
    return s["k_pages"].view(torch.float8_e4m3fn), s["v_pages"].view(torch.float8_e4m3fn), s["k_scales"], s["v_scales"]


def run(state):
    s, c = state, state["case"]
    if not own:
        if c["op"] == "rope":
            return _plain_rope(s)
        if c["op"] == "write":
            _plain_write(s)
            return _cache_as_values(s)
        return _plain_read(s) if c["op"] == "read" else _plain_attend(s)
    from paper_2407_08608_amd import binding
    if c["op"] == "rope":
        call = binding.fa_rope_bwd if c["backward"] else binding.fa_rope
        return call(s["q"], s["inv_freq"], k=s["k"], positions=s["positions"], rot_dim=c["rot"], interleaved=c["interleaved"],
                    amplitude=s["amplitude"])
    if c["op"] == "write":
        binding.fa_cache_write(s["k"], s["v"], s["k_pages"], s["v_pages"], s["table"], s["lens"], counts=s["counts"],
                               k_scales=s["k_scales"], v_scales=s["v_scales"])
        return _cache_as_values(s)
    if c["op"] == "read":
        return binding.fa_cache_read(s["k_pages"], s["v_pages"], s["table"], s["lens"], k_scales=s["k_scales"], v_scales=s["v_scales"],
                                     k=s["k"], v=s["v"])
    return binding.fa_fwd_cache(s["q"], s["k_pages"], s["v_pages"], s["table"], s["lens"], c["d"] ** -0.5, tree=s["tree"],
                                counts=s["counts"], k_scales=s["k_scales"], v_scales=s["v_scales"], max_len=c["most"] + c["T"],
                                o=s["o"], lse=s["lse"])


# ------------------------------------------------------------------------------------------
# The definitions in 64 bits, sequence by sequence


def _sequence(s, name, b, tokens):
    """K or V of one sequence's first `tokens`, [H_kv, tokens, d]"""
    page = s["case"]["page"]
    parts = []
    for i in range(-(-tokens // page)):
        p = int(s["host_table"][b][i])
        x = s[name + "_pages"][p]
        if s[name + "_scales"] is None:
            x = x.double()
        else:
            x = x.view(torch.float8_e4m3fn).double() * s[name + "_scales"][p].double()[..., None]
        parts.append(x)
    return torch.cat(parts, 1)[:, :tokens]


def _exact_rope(s):
    c = s["case"]
    f, amplitude = _frequencies(c)
    at = s["positions"].double() if s["positions"] is not None else torch.arange(c["N"], device="cuda", dtype=torch.float64).expand(c["B"], c["N"])
    turn = torch.polar(torch.full((), amplitude, device="cuda", dtype=torch.float64).expand(c["B"], c["N"], c["rot"] // 2).contiguous(),
                       at[:, :, None] * f.cuda() * (-1 if c["backward"] else 1))
    out = []
    for x in (s["q"], s["k"]):
        y = x.double().contiguous()
        for h in range(x.shape[1]):
            r = y[:, h, :, :c["rot"]]
            pair = r.unflatten(-1, (c["rot"] // 2, 2)) if c["interleaved"] else r.unflatten(-1, (2, c["rot"] // 2)).transpose(-1, -2)
            z = torch.view_as_real(torch.view_as_complex(pair.contiguous()) * turn)
            y[:, h, :, :c["rot"]] = (z if c["interleaved"] else z.transpose(-1, -2)).flatten(-2)
        out.append(y)
    return tuple(out)


def exact(case, seed):
    s = prepare(case, seed)
    c = s["case"]
    if c["op"] == "rope":
        return _exact_rope(s)
    B, H_kv, T, d, page = c["B"], c["H_kv"], c["T"], c["d"], c["page"]
    lens, counts = _lens(c)
    if B * -(-(c["most"] + T) // page) > 40000:  # page by page: too long
        return None
    s["host_table"] = s["table"].tolist()
    if c["op"] == "write":
        out = []
        for n in ("k", "v"):
            quantised = s[n + "_scales"] is not None
            pages = (s[n + "_pages"].view(torch.float8_e4m3fn) if quantised else s[n + "_pages"]).double()
            scales = s[n + "_scales"].double() if quantised else None
            for b in range(B):
                x = s[n][b].double()
                if quantised:  # the codes as they are before they are rounded
                    amax = x.abs().amax(-1)
                    scale = torch.where(amax > 0, amax / 448, torch.ones_like(amax))
                    x = x / scale[..., None]
                t = 0
                while t < counts[b]:
                    at = lens[b] + t
                    n_here = min(page - at % page, counts[b] - t)
                    p, lo = s["host_table"][b][at // page], at % page
                    pages[p, :, lo:lo + n_here] = x[:, t:t + n_here]
                    if quantised:
                        scales[p, :, lo:lo + n_here] = scale[:, t:t + n_here]
                    t += n_here
            out.append((pages, scales))
        (kp, ks), (vp, vs) = out
        return (kp, vp) if ks is None else (kp, vp, ks, vs)
    if c["op"] == "read":
        out = []
        for n in ("k", "v"):
            x = s[n].double()
            for b in range(B):
                x[b, :, :lens[b]] = _sequence(s, n, b, lens[b])
            out.append(x)
        return tuple(out)
    group = c["H"] // H_kv
    o = torch.zeros((B, c["H"], T, d), device="cuda", dtype=torch.float64)
    lse = torch.zeros((B, c["H"], T), device="cuda", dtype=torch.float64)
    tree = None if s["tree"] is None else s["tree"].tolist()
    for b in range(B):
        n = lens[b] + counts[b]
        K, V = _sequence(s, "k", b, n), _sequence(s, "v", b, n)
        hidden = torch.zeros((counts[b], n), dtype=torch.bool)
        for t in range(counts[b]):
            for u in range(counts[b]):
                hidden[t, lens[b] + u] = u > t if tree is None else not (tree[b][t][u // 32] >> (u % 32)) & 1
        hidden = hidden.cuda()
        for h in range(c["H"]):
            score = torch.mm(s["q"][b, h, :counts[b]].double(), K[h // group].t().contiguous()) / math.sqrt(d)
            score[hidden] = -math.inf
            lse[b, h, :counts[b]] = torch.logsumexp(score, 1)
            o[b, h, :counts[b]] = torch.mm(torch.softmax(score, 1), V[h // group])
    return o, lse
