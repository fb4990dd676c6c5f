"""A key/value cache held in 4 bits, its pages' bookkeeping, and rotary positions with several axes: calls that serving and training
programs make next to those on a 16-bit or e4m3 cache, as cases to be timed and checked.  A case is a dict of plain values; `op` says
which call:

  axes     Q and K rotated by positions of several axes (time, height, width), or (`backward`) their gradients rotated back
  store    K and V of new tokens put into the pages of a 4-bit cache, and the whole prefix read back as dense tensors
  attend   attention of T new tokens per sequence over a 4-bit cache that holds them and the tokens before them; T > 1 with a tree
  fork     the batch of the next step: every new sequence continues an old one and shares its whole pages, the pages that several
           would write to are copied, and each gets a page for its next token
  compact  pages in use moved to the lowest numbers of the pool

q [B, H, T, d], k and v [B, H_kv, T, d]; pages [n_pages, H_kv, page_size, ...]; d in {64, 128, 256}, scale d^-1/2.  The 4-bit format: e2m1
codes, two to a byte, the even element in the low half, and a power of two (its biased exponent in a byte) for each 32 elements of a row.
"""
import math
import random

import torch

own = False

_DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_ELEM = {"f32": 4, "bf16": 2, "f16": 2}
_GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)  # the magnitudes of e2m1


def _axes(name, dtype, B, H, H_kv, N, d, rot, axes, dealt, interleaved, backward, token_major):
    """dealt: the pairs go to the axes in turn; otherwise in one run for each axis"""
    c = {"op": "axes", "dtype": dtype, "B": B, "H": H, "H_kv": H_kv, "N": N, "d": d, "rot": rot, "axes": axes, "dealt": dealt,
         "interleaved": interleaved, "backward": backward, "token_major": token_major}
    return {"name": name, **c} if name else c


def _cached(name, op, dtype, B, H, H_kv, T, d, page, most, least):
    """T: new tokens per sequence; most, least: bounds of the lengths that the cache holds before them"""
    c = {"op": op, "dtype": dtype, "B": B, "H": H, "H_kv": H_kv, "T": T, "d": d, "page": page, "most": most, "least": least}
    return {"name": name, **c} if name else c


def _fork(name, cache, groups, before, beams, H_kv, d, page, layers, most, least, spare):
    """groups of `before` old sequences each, of which `beams` new ones continue; spare: pages of the pool that nobody holds"""
    c = {"op": "fork", "cache": cache, "groups": groups, "before": before, "beams": beams, "H_kv": H_kv, "d": d, "page": page, "layers": layers,
         "most": most, "least": least, "spare": spare}
    return {"name": name, **c} if name else c


def _compact(name, cache, B, H_kv, d, page, layers, most, least, pool, held):
    """pool: the pages there are for each 100 in use; held: for each 100 of the pool, those that stay where they are"""
    c = {"op": "compact", "cache": cache, "B": B, "H_kv": H_kv, "d": d, "page": page, "layers": layers, "most": most, "least": least, "pool": pool,
         "held": held}
    return {"name": name, **c} if name else c


def listed():
    return [
        # a decoding step behind images: a token each, its three positions far apart; launch and latency decide
        _axes("axes_token", "bf16", 8, 16, 4, 1, 128, 128, 3, False, False, False, False),
        # gradients of 16k tokens of images and text in a projection's layout, pairs dealt to the axes in turn
        _axes("axes_grad", "bf16", 4, 16, 16, 4096, 128, 128, 3, True, False, True, True),
        # a few new tokens on short prefixes, narrow heads: written, and the prefix read back
        _cached("store_chunk", "store", "f16", 4, 4, 4, 13, 64, 16, 333, 100),
        # prompts of ragged lengths into a fresh cache, read back for a dense pass over them: 16k tokens at most
        _cached("store_prompt", "store", "bf16", 4, 16, 16, 4096, 128, 64, 0, 0),
        # one request, one token, a short cache
        _cached("attend_token", "attend", "bf16", 1, 16, 16, 1, 64, 16, 333, 333),
        # a decoding step of a full batch with shared key/value heads, ragged lengths, small pages
        _cached("attend_batch", "attend", "bf16", 32, 32, 8, 1, 128, 16, 4096, 500),
        # a few very long contexts, widest heads: few rows, the keys have to be split
        _cached("attend_long", "attend", "bf16", 2, 16, 2, 1, 256, 64, 65536, 50000),
        # verifying drafted trees of a batch over long contexts: the matrix products decide
        _cached("attend_tree", "attend", "f16", 8, 16, 4, 32, 128, 32, 8192, 5000),
        # a step of a small beam search: four beams of four requests, one layer's cache
        _fork("fork_beams", "bf16", 4, 4, 4, 8, 128, 16, 1, 500, 100, 40),
        # eight answers to each of 16 long prompts: whole pages shared, the last ones copied, four layers
        _fork("fork_answers", "e4m3", 16, 1, 8, 8, 128, 64, 4, 16384, 3000, 300),
        # a small pool after a few requests have ended
        _compact("compact_small", "f16", 4, 8, 64, 16, 1, 333, 100, 170, 0),
        # a large 4-bit pool, two thirds in use, with pages of a shared prefix that must not move, two layers
        _compact("compact_large", "4bit", 64, 8, 128, 64, 2, 8192, 2000, 150, 2),
    ]


# no drawn case costs more than the largest listed ones
_MOST_BYTES, _MOST_FLOPS = 3.4e8, 1.6e10


def _size(rng, lo, hi):
    """Spread over the logarithm; odd values as common as regular ones"""
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return max(lo, n // 16 * 16) if n > 64 and rng.random() < 0.4 else n


def draw(rng):
    while True:
        op = rng.choice(["axes", "store", "attend", "attend", "attend", "fork", "compact"])
        dtype, d = rng.choice(["bf16", "bf16", "f16"]), rng.choice([64, 128, 128, 256])
        B, H, page = _size(rng, 1, 32), rng.choice([2, 4, 8, 12, 16, 32]), rng.choice([16, 16, 32, 48, 64, 128])
        H_kv = rng.choice([h for h in (1, 2, 4, 8, 16, 32) if H % h == 0])
        if op == "axes":
            c = _axes(None, rng.choice([dtype, dtype, "f32"]), B, H, H_kv, _size(rng, 1, 8192), d, rng.choice([d, d, d // 2, d // 4]), rng.choice([2, 3, 3, 4]),
                      rng.random() < 0.5, rng.random() < 0.5, rng.random() < 0.4, rng.random() < 0.4)
        elif op == "store":
            most = _size(rng, 1, 8192)
            c = _cached(None, op, dtype, B, H, H_kv, _size(rng, 1, 4096), d, page, most, rng.randint(0, most))
        elif op == "attend":
            most = _size(rng, 1, 65536)
            c = _cached(None, op, dtype, B, H, H_kv, rng.choice([1, 1, _size(rng, 2, 64), _size(rng, 2, 64)]), d, page, most, rng.randint(most // 2, most))
        elif op == "fork":
            most = _size(rng, 2, 16384)
            c = _fork(None, rng.choice(["bf16", "f16", "e4m3", "4bit"]), _size(rng, 1, 24), rng.choice([1, 1, 2, 4, 5]), rng.choice([1, 2, 4, 5, 8]), H_kv, d, page,
                      rng.choice([1, 1, 2, 4]), most, rng.randint(1, most), _size(rng, 1, 400))
        else:
            most = _size(rng, 2, 8192)
            c = _compact(None, rng.choice(["bf16", "f16", "e4m3", "4bit"]), _size(rng, 1, 64), H_kv, d, page, rng.choice([1, 1, 2, 4]), most, rng.randint(1, most),
                         rng.choice([105, 150, 200, 400]), rng.choice([0, 0, 3]))
        w = work(c)
        if w["bytes"] > _MOST_BYTES or w["flops"] > _MOST_FLOPS:
            continue
        if op in ("store", "attend"):  # (the plain form holds the dense cache and the scores in 32 bits)
            if c["B"] * c["H"] * c["T"] * (c["most"] + 64) > 1 << 28 or c["B"] * c["H_kv"] * (c["most"] + c["T"]) * c["d"] > 1 << 27:
                continue
        elif op != "axes" and _pool(c) * _page_bytes(c) * 2.0 * c["layers"] > 1e9:
            continue
        return c


def _lens(c):
    """The lengths before the new tokens, and how many of the T new ones each sequence has (some fewer, as in a padded batch).
    They go by the case alone, so that work() knows them."""
    r = random.Random("%(op)s %(B)d %(T)d %(most)d %(least)d" % c)
    lens = [c["most"]] + [r.randint(c["least"], c["most"]) for _ in range(c["B"] - 1)]
    counts = [c["T"]] + [r.randint((c["T"] + 1) // 2, c["T"]) for _ in range(c["B"] - 1)]
    return lens, counts


def _page_bytes(c):
    """Of K, or V, of a page of one layer, scales included"""
    row = {"bf16": 2 * c["d"], "f16": 2 * c["d"], "e4m3": c["d"] + 4, "4bit": c["d"] // 2 + c["d"] // 32}[c["cache"]]
    return c["H_kv"] * c["page"] * row


def _sequences(c):
    """Of a fork: the old sequences' lengths, how many whole pages a group shares, and the new ones' parents (-1: a request has ended and an
    empty one takes its place); by the case alone"""
    r = random.Random("%(groups)d %(before)d %(beams)d %(page)d %(most)d %(least)d" % c)
    lens, shared, parents = [], [], []
    for g in range(c["groups"]):
        n = c["most"] if g == 0 else r.randint(c["least"], c["most"])
        lens += [n] * c["before"]
        shared.append(r.randint(0, n // c["page"]) if c["before"] > 1 else 0)
        ends = g > 0 and r.random() < 0.1
        parents += [-1 if ends else g * c["before"] + r.randrange(c["before"]) for _ in range(c["beams"])]
    return lens, shared, parents


def _pages_of(c):
    """Of a compaction: how many pages each sequence holds"""
    r = random.Random("%(B)d %(page)d %(most)d %(least)d" % c)
    return [-(-(c["most"] if b == 0 else r.randint(c["least"], c["most"])) // c["page"]) for b in range(c["B"])]


def _pool(c):
    if c["op"] == "fork":
        lens, shared, _ = _sequences(c)
        own_pages = sum(-(-n // c["page"]) - shared[i // c["before"]] for i, n in enumerate(lens))
        return own_pages + sum(shared) + c["groups"] * c["beams"] + c["spare"]
    used = sum(_pages_of(c))
    return used * c["pool"] // 100 + 3


def work(case):
    c = case
    if c["op"] == "axes":  # each element in and out; two products and a sum for each that is rotated
        n = c["B"] * (c["H"] + c["H_kv"]) * c["N"]
        return {"bytes": 2.0 * n * c["d"] * _ELEM[c["dtype"]] + 4.0 * c["axes"] * c["B"] * c["N"], "flops": 3.0 * n * c["rot"]}
    if c["op"] == "fork":
        lens, _, parents = _sequences(c)
        kept, copies = set(), 0
        for p in parents:
            if p >= 0 and lens[p] % c["page"]:
                copies += p in kept
                kept.add(p)
        entries = sum(-(-lens[p] // c["page"]) for p in parents if p >= 0)
        return {"bytes": 4.0 * copies * c["layers"] * _page_bytes(c) + 8.0 * entries + 12.0 * len(parents), "flops": 1.0 * entries}
    if c["op"] == "compact":  # (about: which pages a sequence holds goes by the seed)
        used, pool = sum(_pages_of(c)), _pool(c)
        moves = used * (1 - used / pool) * (1 - c["held"] / 100)
        return {"bytes": 4.0 * moves * c["layers"] * _page_bytes(c) + 8.0 * used, "flops": 1.0 * used}
    lens, counts = _lens(c)
    e, row = _ELEM[c["dtype"]], c["d"] / 2 + c["d"] / 32  # a cached token of one head, K or V
    if c["op"] == "store":
        new, n = 2.0 * c["H_kv"] * sum(counts), 2.0 * c["H_kv"] * (sum(lens) + sum(counts))
        return {"bytes": new * (c["d"] * e + row) + n * (row + c["d"] * e), "flops": (2.0 * new + n) * c["d"]}
    keys = 2.0 * c["H_kv"] * sum(a + b for a, b in zip(lens, counts)) * row
    rows = c["H"] * sum(counts) * (2 * c["d"] * e + 4)
    return {"bytes": keys + rows, "flops": sum(4.0 * c["H"] * b * (a + b) * c["d"] for a, b in zip(lens, counts))}


def _axis_of_pairs(c):
    """Which axis each rotated pair goes by"""
    n, a = c["rot"] // 2, c["axes"]
    if c["dealt"]:
        return [i % a for i in range(n)]
    first = n - (a - 1) * (3 * n // (4 * a))  # (time has the most pairs, the others as many as each other)
    return [0 if i < first else 1 + (i - first) // (3 * n // (4 * a)) for i in range(n)]


def _frequencies(c):
    return 10000.0 ** (-torch.arange(0, c["rot"], 2, dtype=torch.float64) / c["rot"])


# ------------------------------------------------------------------------------------------
# What a program has in hand


def _codes_of(x):
    """The 4-bit form of x [..., d] in 32 bits: bytes [..., d / 2] and scales' exponents [..., d / 32].  The scale is the least power of
    two s (no less than 2^-100) with max |x| <= 7 s; a quotient goes to the nearest magnitude, from the middle to the one of even code."""
    g = x.unflatten(-1, (-1, 32))
    bits = g.abs().amax(-1).view(torch.int32)
    exponent = ((bits >> 23) - 129 + ((bits & 0x7FFFFF) > 0x600000).int()).clamp(min=-100)
    y = torch.ldexp(g.abs(), -exponent[..., None])
    code = (y > 0.25).int() + (y >= 0.75).int() + (y > 1.25).int() + (y >= 1.75).int() + (y > 2.5).int() + (y >= 3.5).int() + (y > 5).int()
    code = (code + 8 * torch.signbit(g).int()).flatten(-2)
    return (code[..., 0::2] | code[..., 1::2] << 4).to(torch.uint8), (exponent + 127).to(torch.uint8)


def _values_of(codes, scales):
    """What codes [..., d / 2] and exponents [..., d / 32] stand for, in 32 bits"""
    grid = torch.tensor(_GRID + tuple(-x for x in _GRID), device=codes.device)
    x = grid[torch.stack((codes & 15, codes >> 4), -1).flatten(-2).int()]
    s = (scales.int() << 23).view(torch.float32)
    return (x.unflatten(-1, (-1, 32)) * s[..., None]).flatten(-2)


def _random_pages(c, g, n_pages, cache):
    """[pages, scales] of one layer's K or V"""
    if cache == "4bit" and c["op"] not in ("store", "attend"):  # (moved as they are)
        shape = (n_pages, c["H_kv"], c["page"])
        return [torch.randint(0, 256, shape + (c["d"] // 2,), generator=g, device="cuda", dtype=torch.uint8),
                torch.randint(118, 130, shape + (c["d"] // 32,), generator=g, device="cuda", dtype=torch.uint8)]
    x = torch.randn((n_pages, c["H_kv"], c["page"], c["d"]), generator=g, device="cuda") * (0.5 + torch.rand(c["d"], generator=g, device="cuda"))
    if cache == "4bit":
        return list(_codes_of(x))
    if cache == "e4m3":
        amax = x.abs().amax(-1)
        return [(x * (448 / amax)[..., None]).clamp(-448, 448).to(torch.float8_e4m3fn), amax / 448]
    return [x.to(_DTYPES[cache]), None]


def _prepare_axes(c, g, s):
    B, N, A = c["B"], c["N"], c["axes"]
    dt = _DTYPES[c["dtype"]]

    def heads(n):
        """[B, n, N, d], some channels larger than others; token_major: a view of [B, N, n, d]"""
        x = torch.randn((B, N, n, c["d"]) if c["token_major"] else (B, n, N, c["d"]), generator=g, device="cuda")
        x = (x * (0.5 + torch.rand(c["d"], generator=g, device="cuda"))).to(dt)
        return x.transpose(1, 2) if c["token_major"] else x

    s["q"], s["k"] = heads(c["H"]), heads(c["H_kv"])
    s["inv_freq"], s["axis"] = _frequencies(c).cuda(), torch.tensor(_axis_of_pairs(c), dtype=torch.int32).cuda()
    # sequences that stand at places of their own, images of 24 x 32 patches in them: one place in time, rows and columns of their own
    n = torch.arange(N, device="cuda", dtype=torch.int32)
    first = torch.randint(0, 20000, (B, 1), generator=g, device="cuda", dtype=torch.int32)
    image, patch = n // 1000, n % 1000
    inside = (patch < 768)[None]
    ways = [torch.zeros_like(patch), patch // 32, patch % 32]
    s["positions"] = torch.stack([first + torch.where(inside, (image * 264 + ways[a % 3])[None], (n - 768 * image)[None] + a) for a in range(A)]).to(torch.int32).contiguous()


def _prepare_cached(c, g, s, seed):
    dt = _DTYPES[c["dtype"]]
    lens, counts = _lens(c)
    B, T, H_kv, d, page = c["B"], c["T"], c["H_kv"], c["d"], c["page"]
    per = -(-(c["most"] + T) // page)  # pages of the longest sequence: the width of the table
    n_pages = B * per + 3
    s["table"] = torch.randperm(n_pages, generator=g, device="cuda")[:B * per].view(B, per).to(torch.int32)
    s["lens"] = torch.tensor(lens, dtype=torch.int32).cuda()
    s["counts"] = torch.tensor(counts, dtype=torch.int32).cuda() if min(counts) < T else None
    for n in ("k", "v"):
        s[n + "_pages"], s[n + "_scales"] = _random_pages(c, g, n_pages, "4bit")
    if c["op"] == "store":
        s["all"] = s["lens"] + torch.tensor(counts, dtype=torch.int32).cuda()
        for n in ("k", "v"):
            x = torch.randn((B, H_kv, T, d), generator=g, device="cuda") * (0.5 + torch.rand(d, generator=g, device="cuda"))
            s["new_" + n] = x.to(dt)
            s[n] = torch.zeros((B, H_kv, c["most"] + T, d), device="cuda", dtype=dt)  # rows behind a sequence's end stay as they are
        return
    s["q"] = torch.randn((B, c["H"], T, d), generator=g, device="cuda").to(dt)
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


def _prepare_fork(c, g, s):
    lens, shared, parents = _sequences(c)
    page, n_pages = c["page"], _pool(c)
    numbers = torch.randperm(n_pages, generator=g, device="cuda").tolist()
    at, rows = 0, []
    for group in range(c["groups"]):
        prefix = numbers[at:at + shared[group]]
        at += len(prefix)
        for i in range(c["before"]):
            tail = -(-lens[group * c["before"]] // page) - len(prefix)
            rows.append(prefix + numbers[at:at + tail])
            at += tail
    wide = -(-(c["most"] + 1) // page)
    s["table"] = torch.tensor([r + [-1] * (wide - len(r)) for r in rows], dtype=torch.int32).cuda()
    s["lens"] = torch.tensor(lens, dtype=torch.int32).cuda()
    s["parents"] = torch.tensor(parents, dtype=torch.int32).cuda()
    s["held"] = None
    s["n_pages"] = n_pages


def _prepare_compact(c, g, s):
    holds, n_pages = _pages_of(c), _pool(c)
    numbers = torch.randperm(n_pages, generator=g, device="cuda").tolist()
    wide, at, rows = max(holds) + 2, 0, []
    for n in holds:
        rows.append(numbers[at:at + n] + [-1] * (wide - n))
        at += n
    s["table"] = torch.tensor(rows, dtype=torch.int32).cuda()
    s["held"] = (torch.rand(n_pages, generator=g, device="cuda") < c["held"] / 100).to(torch.int32) if c["held"] else None
    s["n_pages"] = n_pages


def prepare(case, seed):
    c = dict(case)
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 1000003 + 31)
    s = {"case": c}
    if c["op"] == "axes":
        _prepare_axes(c, g, s)
    elif c["op"] in ("store", "attend"):
        _prepare_cached(c, g, s, seed)
    else:
        (_prepare_fork if c["op"] == "fork" else _prepare_compact)(c, g, s)
        s["layers"] = [_random_pages(c, g, s["n_pages"], c["cache"]) + _random_pages(c, g, s["n_pages"], c["cache"]) for _ in range(c["layers"])]
    return s


# ------------------------------------------------------------------------------------------
# The plain form: elementary operations in 32 bits


def _plain_axes(s):
    c = s["case"]
    at = s["positions"][s["axis"].long()].permute(1, 2, 0)  # [B, N, pairs]
    angle = (at.double() * s["inv_freq"])[:, None]  # (64 bits: far positions)
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    if c["backward"]:
        sin = -sin

    def turned(x):
        r = x[..., :c["rot"]].float()
        a, b = (r[..., 0::2], r[..., 1::2]) if c["interleaved"] else (r[..., :c["rot"] // 2], r[..., c["rot"] // 2:])
        y, z = a * cos - b * sin, a * sin + b * cos
        y = torch.stack((y, z), -1).flatten(-2) if c["interleaved"] else torch.cat((y, z), -1)
        return torch.cat((y.to(x.dtype), x[..., c["rot"]:]), -1)

    return turned(s["q"]), turned(s["k"])


def _gathered(s, name, tokens):
    """[B, H_kv, tokens, d] in 32 bits: the first `tokens` of each sequence (behind its end whatever its last page holds)"""
    B, H_kv, d, page = (s["case"][n] for n in ("B", "H_kv", "d", "page"))
    per = -(-tokens // page)
    table = s["table"][:, :per].long()
    x = _values_of(s[name + "_pages"][table], s[name + "_scales"][table])  # [B, per, H_kv, page, d]
    return x.transpose(1, 2).reshape(B, H_kv, per * page, d)[:, :, :tokens]


def _plain_store(s):
    c = s["case"]
    at = s["lens"][:, None].long() + torch.arange(c["T"], device="cuda")
    page, slot = torch.gather(s["table"].long(), 1, at // c["page"]), at % c["page"]
    there = None if s["counts"] is None else (torch.arange(c["T"], device="cuda")[None, :] < s["counts"][:, None])[:, :, None, None]
    for n in ("k", "v"):
        for into, x in zip((s[n + "_pages"], s[n + "_scales"]), _codes_of(s["new_" + n].float())):
            x = x.transpose(1, 2)
            into[page, :, slot] = x if there is None else torch.where(there, x, into[page, :, slot])
    N = s["k"].shape[2]
    there = (torch.arange(N, device="cuda")[None, :] < s["all"][:, None])[:, None, :, None]
    return tuple(torch.where(there, _gathered(s, n, N).to(s[n].dtype), s[n]) for n in ("k", "v"))


def _plain_attend(s):
    c = s["case"]
    B, H, H_kv, T, d = c["B"], c["H"], c["H_kv"], c["T"], c["d"]
    keys = c["most"] + T
    K, V = _gathered(s, "k", keys), _gathered(s, "v", keys)
    q = s["q"].float().view(B, H_kv, H // H_kv * T, d)
    score = torch.matmul(q, K.transpose(-1, -2).contiguous()).view(B, H, T, keys) * d ** -0.5
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
    o = torch.matmul(p.view(B, H_kv, H // H_kv * T, keys), V).view(B, H, T, d) / total
    o, lse = o.to(s["q"].dtype), (m + torch.log(total))[..., 0]
    if s["counts"] is not None:
        there = (torch.arange(T, device="cuda")[None, :] < s["counts"][:, None])[:, None]
        o, lse = torch.where(there[..., None], o, s["o"]), torch.where(there, lse, s["lse"])
    return o, lse


def _in(numbers, chosen, n_pages):
    """Whether each page of the pool is among numbers[chosen]"""
    mark = torch.zeros(n_pages + 1, dtype=torch.bool, device=numbers.device)
    mark[torch.where(chosen, numbers, n_pages).long().flatten()] = True
    return mark[:n_pages]


def _free_first(used):
    """The pages that are not used in ascending order, then the others; and how many those are"""
    n = torch.arange(used.numel(), device=used.device)
    return torch.sort(torch.where(used, n + used.numel(), n))[1], (~used).sum()


def _given(need, free, n_free):
    """A free page for each that needs one, in order; -1 without, or where there are none left"""
    rank = torch.cumsum(need.int(), 0) - 1
    there = need & (rank < n_free)
    return torch.where(there, free[rank.clamp(0, free.numel() - 1)], -1), (need & ~there).sum()


def _plain_copy(layer, src, dst):
    """Page src[i] to dst[i], pairs of -1 left out (they rewrite a page with itself that no pair writes to)"""
    n = layer[0].shape[0]
    there = src >= 0
    spare = (~_in(dst, there, n)).int().argmax()
    a, b = torch.where(there, src.long(), spare), torch.where(there, dst.long(), spare)
    for x in layer:
        if x is not None:
            x = x.view(torch.uint8) if x.element_size() == 1 else x
            x[b] = x[a]


def _plain_fork(s):
    c, table, n_pages = s["case"], s["table"], s["n_pages"]
    page, wide = c["page"], s["table"].shape[1]
    from_old = s["parents"] >= 0
    p = s["parents"].long().clamp(min=0)
    lens = torch.where(from_old, s["lens"][p], 0)
    rows, col = table[p], torch.arange(wide, device="cuda")[None, :]
    whole, last = lens // page, lens % page > 0
    held = col < (whole + last.int())[:, None]
    new = torch.where(held, rows, -1)
    part = torch.gather(rows, 1, whole.clamp(max=wide - 1)[:, None].long())[:, 0]
    order = torch.arange(p.numel(), device="cuda", dtype=torch.int32)
    first = torch.full((n_pages + 1,), 1 << 30, dtype=torch.int32, device="cuda")
    first.scatter_reduce_(0, torch.where(last, part, n_pages).long(), order, "amin")
    inside = _in(rows, col < whole[:, None], n_pages)
    need = last & ((first[part.clamp(min=0).long()] != order) | inside[part.clamp(min=0).long()])
    dst, missing = _given(need, *_free_first(_in(new, new >= 0, n_pages)))
    new.scatter_(1, whole.clamp(max=wide - 1)[:, None].long(), torch.where(need, dst.int(), torch.gather(new, 1, whole.clamp(max=wide - 1)[:, None].long())[:, 0])[:, None])
    dst = dst.int()
    src = torch.where(dst >= 0, part, -1)
    for layer in s["layers"]:
        _plain_copy(layer, src, dst)
    at = (lens // page).long()[:, None]  # the page of the next token
    have = torch.gather(new, 1, at)[:, 0]
    more, none = _given(have < 0, *_free_first(_in(new, new >= 0, n_pages)))
    new.scatter_(1, at, torch.where(have < 0, more.int(), have)[:, None])
    return new, lens, src, dst, missing.int().view(1), none.int().view(1)


def _plain_compact(s):
    table, n_pages = s["table"], s["n_pages"]
    inside = _in(table, table >= 0, n_pages)
    stays = s["held"] != 0 if s["held"] is not None else torch.zeros_like(inside)
    used, movable = inside | stays, inside & ~stays
    half = n_pages // 2
    n = torch.arange(n_pages, device="cuda")
    free = torch.sort(torch.where(used, n_pages, n))[0][:half]
    high = torch.sort(torch.where(movable, n, -1), descending=True)[0][:half]
    there = free < high
    src, dst = torch.where(there, high, -1).int(), torch.where(there, free, -1).int()
    to = torch.cat((n, n[:1]))
    to[torch.where(there, high, n_pages)] = free
    new = torch.where(table >= 0, to[table.clamp(min=0).long()].int(), table)
    now = torch.cat((used, used[:1]))
    now[torch.where(there, high, n_pages)] = False
    now[torch.where(there, free, n_pages)] = True
    top = torch.where(now[:n_pages], n + 1, 0).amax()
    for layer in s["layers"]:
        _plain_copy(layer, src, dst)
    return new, src, dst, top.int().view(1)


def _flat(layers):
    return [x for layer in layers for x in layer if x is not None]


def run(state):
    s, c = state, state["case"]
    if not own:
        if c["op"] in ("fork", "compact"):
            return list((_plain_fork if c["op"] == "fork" else _plain_compact)(s)) + _flat(s["layers"])
        return {"axes": _plain_axes, "store": _plain_store, "attend": _plain_attend}[c["op"]](s)
    from paper_2407_08608_amd import binding
    if c["op"] == "axes":
        call = binding.fa_rope_axes_bwd if c["backward"] else binding.fa_rope_axes
        return call(s["q"], s["inv_freq"], s["axis"], s["positions"], k=s["k"], rot_dim=c["rot"], interleaved=c["interleaved"])
    if c["op"] == "store":
        binding.fa_cache_write(s["new_k"], s["new_v"], s["k_pages"], s["v_pages"], s["table"], s["lens"], counts=s["counts"], k_scales=s["k_scales"],
                               v_scales=s["v_scales"])
        return binding.fa_cache_read(s["k_pages"], s["v_pages"], s["table"], s["all"], k_scales=s["k_scales"], v_scales=s["v_scales"], k=s["k"], v=s["v"])
    if c["op"] == "attend":
        return binding.fa_fwd_cache(s["q"], s["k_pages"], s["v_pages"], s["table"], s["lens"], c["d"] ** -0.5, tree=s["tree"], counts=s["counts"],
                                    k_scales=s["k_scales"], v_scales=s["v_scales"], max_len=c["most"] + c["T"], o=s["o"], lse=s["lse"])
    if c["op"] == "fork":
        table, lens, src, dst, missing = binding.fa_cache_fork(s["table"], s["lens"], s["parents"], c["page"], s["n_pages"])
        for k, ks, v, vs in s["layers"]:
            binding.fa_cache_copy(k, v, src, dst, k_scales=ks, v_scales=vs)
        table, none = binding.fa_cache_extend(table, lens, 1, c["page"], s["n_pages"])
        return [table, lens, src, dst, missing, none] + _flat(s["layers"])
    table, src, dst, top = binding.fa_cache_compact(s["table"], s["n_pages"], held=s["held"])
    for k, ks, v, vs in s["layers"]:
        binding.fa_cache_copy(k, v, src, dst, k_scales=ks, v_scales=vs)
    return [table, src, dst, top] + _flat(s["layers"])


# ------------------------------------------------------------------------------------------
# The definitions in 64 bits, token by token and page by page


def _row_values(codes, scales):
    """[..., d] in 64 bits, by the format's own fields: s e e m"""
    n = torch.empty(codes.shape[:-1] + (codes.shape[-1], 2), dtype=torch.int64, device=codes.device)
    n[..., 0], n[..., 1] = codes.long() % 16, codes.long() // 16
    n = n.flatten(-2)
    e, m = n // 2 % 4, (n % 2).double()
    x = torch.where(e == 0, 0.5 * m, (1 + 0.5 * m) * 2.0 ** (e.double() - 1)) * (1 - 2 * (n // 8)).double()
    return x * torch.repeat_interleave(2.0 ** (scales.double() - 127), 32, -1)


def _row_rounded(x):
    """x [..., d] in 64 bits as the cache holds it"""
    g = x.reshape(x.shape[:-1] + (x.shape[-1] // 32, 32))
    a = g.abs().amax(-1, keepdim=True)
    s = 2.0 ** torch.ceil(torch.log2(a / 7).clamp(min=-100))
    s = torch.where(a <= 3.5 * s, s / 2, torch.where(a > 7 * s, 2 * s, s)).clamp(min=2.0 ** -100)  # (where the logarithm's rounding decides)
    grid = torch.tensor(_GRID, dtype=torch.float64, device=x.device)
    y = (g.abs() / s)[..., None] - grid
    away = y.abs() - 1e-9 * (torch.arange(8, device=x.device) % 2 == 0)  # (from the middle to an even code)
    return (torch.copysign(grid[away.argmin(-1)], g) * s).reshape(x.shape)


def _exact_axes(s):
    c = s["case"]
    f, axis = _frequencies(c).cuda(), _axis_of_pairs(c)
    angle = torch.stack([s["positions"][a].double() * f[i] for i, a in enumerate(axis)], -1)
    turn = torch.polar(torch.ones_like(angle), -angle if c["backward"] else angle)
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


def _sequence(s, table, name, b, tokens):
    """K or V of one sequence's first `tokens`, [H_kv, tokens, d]"""
    numbers = table[b][:-(-tokens // s["case"]["page"])]
    x = [_row_values(s[name + "_pages"][p], s[name + "_scales"][p]) for p in numbers]
    return torch.cat(x, 1)[:, :tokens] if x else torch.zeros((s["case"]["H_kv"], 0, s["case"]["d"]), device="cuda", dtype=torch.float64)


def _exact_cached(s):
    c = s["case"]
    B, H_kv, T, d, page = c["B"], c["H_kv"], c["T"], c["d"], c["page"]
    if B * -(-(c["most"] + T) // page) > 15000:  # page by page: too long
        return None
    lens, counts = _lens(c)
    table = s["table"].tolist()
    if c["op"] == "store":
        out = []
        for n in ("k", "v"):
            x = s[n].double()
            for b in range(B):
                x[b, :, :lens[b]] = _sequence(s, table, n, b, lens[b])
                x[b, :, lens[b]:lens[b] + counts[b]] = _row_rounded(s["new_" + n][b, :, :counts[b]].double())
            out.append(x)
        return tuple(out)
    group = c["H"] // H_kv
    o = torch.zeros((B, c["H"], T, d), device="cuda", dtype=torch.float64)
    lse = torch.zeros((B, c["H"], T), device="cuda", dtype=torch.float64)
    tree = None if s["tree"] is None else s["tree"].tolist()
    for b in range(B):
        n = lens[b] + counts[b]
        K, V = _sequence(s, table, "k", b, n), _sequence(s, table, "v", b, n)
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


def _moved(s, pairs):
    out = []
    for layer in s["layers"]:
        for x in layer:
            if x is not None:
                b = x.view(torch.uint8) if x.element_size() == 1 else x
                for p, q in pairs:
                    b[q] = b[p]
                out.append(x.double() if x.is_floating_point() else x)
    return out


def _listed_pairs(pairs, n):
    src, dst = ([p[i] for p in pairs] for i in range(2))
    return [torch.tensor(x + [-1] * (n - len(x)), dtype=torch.int32) for x in (src, dst)]


def _exact_fork(s):
    c, page, table, lens = s["case"], s["case"]["page"], s["table"].tolist(), s["lens"].tolist()
    rows, wide = [], s["table"].shape[1]
    new_lens = [lens[p] if p >= 0 else 0 for p in s["parents"].tolist()]
    whole_pages, last_pages = set(), set()
    for p, n in zip(s["parents"].tolist(), new_lens):
        rows.append(table[p][:-(-n // page)] if n else [])
        whole_pages.update(rows[-1][:n // page])
        last_pages.update(rows[-1][n // page:])
    free = sorted(set(range(s["n_pages"])) - whole_pages - last_pages, reverse=True)
    kept, src, dst, missing = set(whole_pages), [], [], 0
    for row, n in zip(rows, new_lens):
        src.append(-1)
        dst.append(-1)
        if n % page:
            if row[-1] in kept:
                if free:
                    src[-1], dst[-1] = row[-1], free.pop()
                missing += dst[-1] < 0
                row[-1] = dst[-1]
            else:
                kept.add(row[-1])
    pages = _moved(s, [(a, b) for a, b in zip(src, dst) if a >= 0])
    used = {p for row in rows for p in row if p >= 0}
    free, none = sorted(set(range(s["n_pages"])) - used, reverse=True), 0
    for row, n in zip(rows, new_lens):
        row += [-1] * (wide - len(row))
        if row[n // page] < 0:
            row[n // page] = free.pop() if free else -1
            none += row[n // page] < 0
    return [torch.tensor(x, dtype=torch.int32) for x in (rows, new_lens, src, dst, [missing], [none])] + pages


def _exact_compact(s):
    table, n_pages = s["table"].tolist(), s["n_pages"]
    held = {p for p, h in enumerate(s["held"].tolist()) if h} if s["held"] is not None else set()
    used = {p for row in table for p in row if p >= 0}
    free, high = sorted(set(range(n_pages)) - used - held), sorted(used - held, reverse=True)
    pairs = [(p, q) for p, q in zip(high, free) if q < p]
    to = dict(pairs)
    rows = [[to.get(p, p) for p in row] for row in table]
    top = 1 + max({p for row in rows for p in row if p >= 0} | held)
    return [torch.tensor(rows, dtype=torch.int32)] + _listed_pairs(pairs, n_pages // 2) + [torch.tensor([top], dtype=torch.int32)] + _moved(s, pairs)


def exact(case, seed):
    s = prepare(case, seed)
    if s["case"]["op"] in ("store", "attend"):
        return _exact_cached(s)
    return {"axes": _exact_axes, "fork": _exact_fork, "compact": _exact_compact}[s["case"]["op"]](s)
