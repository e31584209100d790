"""The key-value cache operators of this library as cases that can be timed and compared: rotary positions with several axes (and their
gradient), keys and values written into a paged cache (rotated, and in 8 bits with a scale for each token and head), rows of the cache read
back, and the attention of new tokens over the cache.

``run`` computes a case's operator in elementary torch operations (fp32; angles in 64 bits), or, where ``own`` is true, through the public
Python entry points of ``paper_2608_03537_b200``.  A user's program keeps the caches, page tables, output buffers and the attention's workspace,
so ``prepare`` makes them.  Caches are [pages, heads, page, D], and a sequence's pages lie anywhere in them.

    rotary   angle = pos[axis(p), t] * freq[p];  a pair (a, b) -> (a cos - b sin, a sin + b cos), or back (the gradient)
    write    q and k rotated, k and v into the cache's slots; in 8 bits: s = max|y| / 127, code = rint(y / s), and the rows read back
    read     rows of the cache by slot, as 16-bit values
    attend   softmax over the visible keys of cap * tanh(alpha q.k / cap) + slope * (pos_k - pos_q), times the values
"""
import math

import numpy as np
import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
_BYTES = {"bf16": 2, "f16": 2, "f32": 4}
BASE = 10000.0


def listed():
    return [
        # queries of a video model's latent patches: positions in time, height and width
        {"name": "rotary_video", "path": "rotary", "tokens": 16384, "heads": 24, "D": 128, "rotated": 128, "axes": 3, "adjacent": False, "inverse": False, "dtype": "bf16"},
        # the gradient of an image model's rotated keys, fp32, pairs side by side
        {"name": "rotary_gradient", "path": "rotary", "tokens": 777, "heads": 12, "D": 64, "rotated": 64, "axes": 2, "adjacent": True, "inverse": True, "dtype": "f32"},
        # one new token of one sequence: the latency of a call
        {"name": "write_token", "path": "write", "tokens": 1, "Hq": 32, "Hkv": 8, "D": 128, "rotated": 128, "axes": 1, "adjacent": False, "page": 16, "dtype": "bf16", "int8": False},
        # one decoding step of 64 sequences, some of them padding, into 8 bits and read back
        {"name": "write_step_q8", "path": "write", "tokens": 64, "Hq": 64, "Hkv": 8, "D": 128, "rotated": 128, "axes": 1, "adjacent": False, "page": 64, "dtype": "bf16", "int8": True},
        # 8192 tokens of prefill
        {"name": "write_prefill", "path": "write", "tokens": 8192, "Hq": 32, "Hkv": 8, "D": 128, "rotated": 128, "axes": 1, "adjacent": False, "page": 64, "dtype": "bf16", "int8": False},
        # a short prefix, pages of a size that fits nothing
        {"name": "read_short", "path": "read", "tokens": 500, "Hkv": 6, "D": 64, "page": 24, "dtype": "f16", "int8": False},
        # a long cached prefix in 8 bits, read back for the attention of the prompt behind it
        {"name": "read_prefix_q8", "path": "read", "tokens": 32768, "Hkv": 8, "D": 128, "page": 64, "dtype": "bf16", "int8": True},
        # one sequence of a thousand tokens: latency
        {"name": "attend_token", "path": "attend", "B": 1, "T": 1, "L": 1000, "Hq": 32, "Hkv": 8, "D": 128, "page": 16, "window": 0, "slopes": False, "cap": 0.0, "dtype": "bf16", "int8": False},
        # one sequence with a long context
        {"name": "attend_long", "path": "attend", "B": 1, "T": 1, "L": 131072, "Hq": 32, "Hkv": 8, "D": 128, "page": 64, "window": 0, "slopes": False, "cap": 0.0, "dtype": "bf16", "int8": False},
        # a decoding step of 24 sequences, a head of keys for each of queries, nearer keys weighing more, the last 512 visible
        {"name": "attend_window", "path": "attend", "B": 24, "T": 1, "L": 2000, "Hq": 16, "Hkv": 16, "D": 64, "page": 24, "window": 512, "slopes": True, "cap": 0.0, "dtype": "f16", "int8": False},
        # five drafted tokens of 8 sequences, checked at once; wide heads, capped scores
        {"name": "attend_draft", "path": "attend", "B": 8, "T": 5, "L": 5000, "Hq": 16, "Hkv": 2, "D": 256, "page": 64, "window": 0, "slopes": False, "cap": 50.0, "dtype": "bf16", "int8": False},
        # a decoding step of 64 sequences of all lengths over a cache in 8 bits
        {"name": "attend_batch_q8", "path": "attend", "B": 64, "T": 1, "L": 16384, "Hq": 64, "Hkv": 8, "D": 128, "page": 64, "window": 0, "slopes": False, "cap": 0.0, "dtype": "bf16", "int8": True},
    ]


def _log(rng, lo, hi, step=1):
    """An integer multiple of `step` in [lo, hi], spread evenly over the logarithm."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return min(hi, max(lo, int(round(v / step)) * step))


def draw(rng):
    path = rng.choice(["rotary", "write", "write", "read", "attend", "attend", "attend", "attend"])
    flag = lambda: rng.random() < 0.5  # noqa: E731
    D = rng.choice([64, 64, 80, 96, 128, 128, 128, 256])
    page = rng.choice([8, 16, 16, 24, 64, 64, 100, 128])
    type16 = rng.choice(["bf16", "bf16", "f16"])
    if path == "rotary":
        tokens = _log(rng, 1, 16384)
        heads = _log(rng, 1, max(1, min(64, (1 << 25) // (tokens * D))))
        return {"path": path, "tokens": tokens, "heads": heads, "D": D, "rotated": rng.choice([D, D, D // 2]), "axes": rng.choice([1, 1, 2, 3]), "adjacent": flag(), "inverse": flag(),
                "dtype": rng.choice([type16, type16, "f32"])}
    if path == "write":
        Hkv = _log(rng, 1, 16)
        return {"path": path, "tokens": _log(rng, 1, 8192 * 8 * 128 // (max(8, Hkv) * max(128, D))), "Hq": Hkv * rng.choice([1, 2, 4]), "Hkv": Hkv, "D": D, "rotated": rng.choice([D, D, D // 2]),
                "axes": rng.choice([1, 1, 2, 3]), "adjacent": flag(), "page": page, "dtype": type16, "int8": flag()}
    if path == "read":
        Hkv = _log(rng, 1, 16)
        return {"path": path, "tokens": _log(rng, 1, 32768 * 8 * 128 // (max(8, Hkv) * max(128, D))), "Hkv": Hkv, "D": D, "page": page, "dtype": type16, "int8": flag()}
    B, Hkv = _log(rng, 1, 64), _log(rng, 1, 16)
    L = _log(rng, 1, min(131072, (1 << 28) // (B * Hkv * D)))
    return {"path": path, "B": B, "T": min(L, rng.choice([1, 1, 1, 2, 5, 8])), "L": L, "Hq": Hkv * rng.choice([1, 1, 2, 4, 4, 5, 8, 8, 16]), "Hkv": Hkv, "D": D, "page": page,
            "window": rng.choice([0, 0, 0, _log(rng, 16, 4096)]), "slopes": rng.random() < 0.25, "cap": rng.choice([0.0, 0.0, 30.0]), "dtype": type16, "int8": flag()}


def _lengths(case):
    """The sequences' lengths: from the longest down to a few tokens, none at all among more than four."""
    B, L, T = case["B"], case["L"], case["T"]
    r = np.random.RandomState(B * 131 + L)
    n = np.maximum(T, np.minimum(L, np.ceil(L * r.uniform(0.02, 1.0, B)).astype(np.int64)))
    n[0] = L
    if B > 4:
        n[B // 2] = 0
    return n


def _sections(pairs, axes):
    """Pairs of each axis: the first takes fewer, as time does."""
    if axes == 1:
        return None
    rest = (pairs * 3 // 8 if axes == 3 else pairs // 2)
    return (pairs - rest * (axes - 1),) + (rest,) * (axes - 1)


class _Make:
    """Device tensors from one seeded generator."""

    def __init__(self, seed):
        self.g = torch.Generator(device="cuda").manual_seed(int(seed))
        self.seed = int(seed)

    def normal(self, *shape, std=1.0):
        return torch.empty(shape, dtype=torch.float32, device="cuda").normal_(0.0, std, generator=self.g)

    def values(self, t, *shape):
        """N(0, 1) of type t; a large tensor in parts."""
        x = torch.empty(shape, dtype=t, device="cuda")
        for part in x.view(-1).split(1 << 27):
            part.copy_(self.normal(part.numel()))
        return x

    def codes(self, *shape):
        """8-bit rows and scales as a cache holds them: a row's largest value has the code 127 or -127."""
        q = torch.empty(shape, dtype=torch.int8, device="cuda")
        for part in q.view(-1, shape[-1]).split(1 << 20):
            x = self.normal(*part.shape)
            part.copy_((x * (127 / x.abs().amax(-1, keepdim=True))).round_())
        return q, 0.02 * torch.exp(0.5 * self.normal(*shape[:-1]))

    def order(self, n):
        return torch.randperm(n, device="cuda", generator=self.g)


def _positions(g, case, tokens):
    """Running text, or the grid of an image or a video, from some place on; [tokens] for one axis, else [axes, tokens]."""
    n = torch.arange(tokens, dtype=torch.int32, device="cuda")
    at = int(np.random.RandomState(g.seed % (1 << 31)).randint(0, 100000))
    if case["axes"] == 1:
        return n + at
    side = max(1, int(round(tokens ** (1 / case["axes"]))))
    rows = [n // (side * side) + at % 1000, n // side % side, n % side] if case["axes"] == 3 else [n // side + at % 1000, n % side]
    return torch.stack(rows).to(torch.int32)


def _rotary_plan(g, case, tokens):
    pairs = case["rotated"] // 2
    freqs = BASE ** (-torch.arange(pairs, dtype=torch.float64, device="cuda") / pairs)
    sections = _sections(pairs, case["axes"])
    axis = torch.from_numpy(np.repeat(np.arange(case["axes"]), sections or (pairs,))).cuda()   # of each pair
    return {"freqs": freqs, "positions": _positions(g, case, tokens), "sections": sections, "axis": axis}


def _cache(g, t, int8, pages, heads, page, D):
    """(keys, values, scales of keys, scales of values), filled with what stands in a cache that is in use."""
    if int8:
        k, ks = g.codes(pages, heads, page, D)
        v, vs = g.codes(pages, heads, page, D)
        return {"k_cache": k, "v_cache": v, "k_scale": ks, "v_scale": vs}
    return {"k_cache": g.values(t, pages, heads, page, D), "v_cache": g.values(t, pages, heads, page, D), "k_scale": None, "v_scale": None}


def _slots(g, tokens, pages, page):
    """Running slots through pages that lie anywhere; in 16 tokens or more, three of padding."""
    table = g.order(pages)
    n = torch.arange(tokens, device="cuda")
    slots = table[n // page] * page + n % page
    if tokens >= 16:
        slots[[3, tokens // 2, tokens - 1]] = -1
    return slots


def prepare(case, seed):
    g, t = _Make(seed), _TYPES[case["dtype"]]
    s, D = {"case": case}, case["D"]
    if case["path"] == "rotary":
        s |= _rotary_plan(g, case, case["tokens"])
        s["x"] = g.normal(case["tokens"], case["heads"], D).to(t)
        s["out"] = torch.empty_like(s["x"])
        return s
    if case["path"] in ("write", "read"):
        tokens, H, page = case["tokens"], case["Hkv"], case["page"]
        pages = (tokens + page - 1) // page + 2
        s |= _cache(g, t, case["int8"], pages, H, page, D)
        s["slots"] = _slots(g, tokens, pages, page)
        s["k"], s["v"] = torch.zeros(tokens, H, D, dtype=t, device="cuda"), torch.zeros(tokens, H, D, dtype=t, device="cuda")
        if case["path"] == "write":   # one projection's output: queries, keys and values of a token side by side
            s |= _rotary_plan(g, case, tokens)
            qkv = g.normal(tokens, case["Hq"] + 2 * H, D).to(t)
            s["new_q"], s["new_k"], s["new_v"] = qkv.split((case["Hq"], H, H), dim=1)
            s["q_out"] = torch.empty(tokens, case["Hq"], D, dtype=t, device="cuda")
        return s
    B, L, page = case["B"], case["L"], case["page"]
    n = _lengths(case)[np.random.RandomState(int(seed) % (1 << 31)).permutation(B)]
    need = (n + page - 1) // page
    width, pages = (L + page - 1) // page, int(need.sum())
    s |= _cache(g, t, case["int8"], pages, case["Hkv"], page, D)
    table = np.full((B, width), -1, np.int32)
    order = g.order(pages).cpu().numpy()
    at = 0
    for b in range(B):
        table[b, : need[b]] = order[at: at + need[b]]
        at += need[b]
    s["table"], s["lengths"] = torch.from_numpy(table).cuda(), torch.from_numpy(n.astype(np.int32)).cuda()
    s["q"] = (1.5 * g.normal(B, case["T"], case["Hq"], D)).to(t)
    s["out"], s["lse"] = torch.empty_like(s["q"]), torch.empty(B, case["T"], case["Hq"], dtype=torch.float32, device="cuda")
    s["slopes"] = 2.0 ** (-8 * torch.arange(1, case["Hq"] + 1, dtype=torch.float32, device="cuda") / case["Hq"]) if case["slopes"] else None
    s["workspace"] = torch.empty(32 << 20, dtype=torch.uint8, device="cuda")
    return s


# ---------------------------------------------------------------------------------------------- plain forms
def _rotate(s, x, inverse=False):
    """fp32 [tokens, heads, D] rotated; angles in 64 bits."""
    pairs, adjacent = s["case"]["rotated"] // 2, s["case"]["adjacent"]
    pos = s["positions"].reshape(-1, x.shape[0]).double()
    angle = pos[s["axis"]].T * s["freqs"]
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    if inverse:
        sin = -sin
    r = x[..., : 2 * pairs]
    a, b = (r[..., 0::2], r[..., 1::2]) if adjacent else (r[..., :pairs], r[..., pairs:])
    y, z = a * cos - b * sin, a * sin + b * cos
    r = torch.stack((y, z), -1).flatten(-2) if adjacent else torch.cat((y, z), -1)
    return torch.cat((r, x[..., 2 * pairs:]), -1)


def _quantize(y):
    """(whole numbers as fp32, scale) of fp32 rows."""
    scale = y.abs().amax(-1, keepdim=True) / 127
    return torch.where(scale > 0, torch.round(y / scale), 0.0), scale


def _plain_write(s):
    case, t = s["case"], _TYPES[s["case"]["dtype"]]
    put = s["slots"] >= 0
    at = s["slots"][put]
    page, row = at // case["page"], at % case["page"]
    q, k, v = _rotate(s, s["new_q"].float()).to(t), _rotate(s, s["new_k"].float())[put], s["new_v"].float()[put]
    if not case["int8"]:
        s["k_cache"][page, :, row], s["v_cache"][page, :, row] = k.to(t), v.to(t)
        return {"q": q, "k_cache": s["k_cache"], "v_cache": s["v_cache"]}
    (k, ks), (v, vs) = _quantize(k), _quantize(v)
    s["k_cache"][page, :, row], s["v_cache"][page, :, row] = k.to(torch.int8), v.to(torch.int8)
    s["k_scale"][page, :, row], s["v_scale"][page, :, row] = ks[..., 0], vs[..., 0]
    return {"q": q, "k_scale": s["k_scale"], "v_scale": s["v_scale"], **_plain_read(s)}


def _plain_read(s):
    case, t = s["case"], _TYPES[s["case"]["dtype"]]
    at = s["slots"].clamp_min(0)
    page, row, put = at // case["page"], at % case["page"], (s["slots"] >= 0)[:, None, None]
    k, v = s["k_cache"][page, :, row].float(), s["v_cache"][page, :, row].float()
    if case["int8"]:
        k, v = k * s["k_scale"][page, :, row][..., None], v * s["v_scale"][page, :, row][..., None]
    return {"k": torch.where(put, k.to(t), s["k"]), "v": torch.where(put, v.to(t), s["v"])}


def _plain_attend(s):
    case = s["case"]
    B, T, H, D = case["B"], case["T"], case["Hkv"], case["D"]
    G = case["Hq"] // H
    at = s["table"].clamp_min(0).long()
    n = at.shape[1] * case["page"]

    def rows(cache, scale):   # [B, heads, positions, D]
        x = cache[at].float()
        if scale is not None:
            x = x * scale[at][..., None]
        return x.transpose(1, 2).reshape(B, H, n, D)

    q = s["q"].float().view(B, T, H, G, D).permute(0, 2, 1, 3, 4).reshape(B, H, T * G, D)
    z = ((q @ rows(s["k_cache"], s["k_scale"]).mT) * D ** -0.5).view(B, H, T, G, n)
    if case["cap"]:
        z = case["cap"] * torch.tanh(z / case["cap"])
    pos = s["lengths"].long()[:, None] - T + torch.arange(T, device="cuda")
    gap = torch.arange(n, device="cuda") - pos[..., None]   # [B, T, n]
    if case["slopes"]:
        z = z + s["slopes"].view(H, 1, G, 1) * gap[:, None, :, None]
    hidden = (gap > 0) | (gap <= -case["window"]) if case["window"] else gap > 0
    z = z.masked_fill(hidden[:, None, :, None], -math.inf)
    top = z.amax(-1, keepdim=True)
    p = torch.exp(z - torch.where(top == -math.inf, 0.0, top))
    total = p.sum(-1, keepdim=True)
    o = (p.view(B, H, T * G, n) @ rows(s["v_cache"], s["v_scale"])).view(B, H, T, G, D) / torch.where(total > 0, total, 1.0)
    lse = (top + torch.log(total))[..., 0]
    return {"out": o.permute(0, 2, 1, 3, 4).reshape(B, T, case["Hq"], D).to(s["q"].dtype), "lse": lse.permute(0, 2, 1, 3).reshape(B, T, case["Hq"])}


def _plain(s):
    path = s["case"]["path"]
    if path == "rotary":
        return _rotate(s, s["x"].float(), s["case"]["inverse"]).to(s["x"].dtype)
    return _plain_write(s) if path == "write" else _plain_read(s) if path == "read" else _plain_attend(s)


# ---------------------------------------------------------------------------------------------- the library's entry points
def _library(s):
    import paper_2608_03537_b200 as cf
    case = s["case"]
    if case["path"] == "rotary":
        return cf.rotary(s["x"], s["positions"], s["freqs"], s["out"], sections=s["sections"], adjacent=case["adjacent"], inverse=case["inverse"])
    scales = {"k_scale": s["k_scale"], "v_scale": s["v_scale"]}
    if case["path"] == "attend":
        cf.paged_attention(s["q"], s["k_cache"], s["v_cache"], s["table"], s["lengths"], s["out"], lse=s["lse"], slopes=s["slopes"], window=case["window"], softcap=case["cap"],
                           alpha=case["D"] ** -0.5, max_length=case["L"], workspace=s["workspace"], **scales)
        return {"out": s["out"], "lse": s["lse"]}
    if case["path"] == "write":
        cf.cache_write(s["new_k"], s["new_v"], s["k_cache"], s["v_cache"], s["slots"], q=s["new_q"], q_out=s["q_out"], positions=s["positions"], freqs=s["freqs"], sections=s["sections"],
                       adjacent=case["adjacent"], **scales)
        if not case["int8"]:
            return {"q": s["q_out"], "k_cache": s["k_cache"], "v_cache": s["v_cache"]}
    cf.cache_read(s["k_cache"], s["v_cache"], s["slots"], s["k"], s["v"], **scales)
    if case["path"] == "read":
        return {"k": s["k"], "v": s["v"]}
    return {"q": s["q_out"], "k_scale": s["k_scale"], "v_scale": s["v_scale"], "k": s["k"], "v": s["v"]}


def run(state):
    if own:
        return _library(state)
    return _plain(state)


def work(case):
    e, D = _BYTES[case["dtype"]], case["D"]
    plan = 4 * case.get("tokens", 0) * case.get("axes", 0) + 4 * case.get("rotated", 0)
    if case["path"] == "rotary":
        n = case["tokens"] * case["heads"] * D
        return {"bytes": 2 * n * e + plan, "flops": 3 * n}
    if case["path"] == "write":
        q, kv = case["tokens"] * case["Hq"] * D, 2 * case["tokens"] * case["Hkv"]
        held = D + 4 if case["int8"] else D * e   # a row of the cache
        back = held + D * e if case["int8"] else 0
        return {"bytes": 2 * q * e + kv * (D * e + held + back) + plan + 8 * case["tokens"], "flops": 3 * q + 4 * kv * D}
    if case["path"] == "read":
        held = D + 4 if case["int8"] else D * e
        return {"bytes": 2 * case["tokens"] * case["Hkv"] * (held + D * e) + 8 * case["tokens"], "flops": 2 * case["tokens"] * case["Hkv"] * D}
    n = _lengths(case)
    seen = int(np.minimum(n, case["window"] + case["T"] - 1).sum() if case["window"] else n.sum())
    held = D + 4 if case["int8"] else D * e
    rows = case["B"] * case["T"] * case["Hq"]
    return {"bytes": 2 * seen * case["Hkv"] * held + 2 * rows * D * e + 4 * rows + 4 * case["B"], "flops": 4 * seen * case["T"] * case["Hq"] * D}


# ---------------------------------------------------------------------------------------------- the definitions in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    f = lambda name: None if s.get(name) is None else s[name].to(torch.float64)  # noqa: E731
    D, page = case["D"], case.get("page")

    def turned(x, back=False):
        pairs = case["rotated"] // 2
        i = torch.arange(pairs, device="cuda")
        first, second = (2 * i, 2 * i + 1) if case["adjacent"] else (i, i + pairs)
        y = x.clone()
        start = 0
        for axis, n in enumerate(s["sections"] or (pairs,)):
            pos = s["positions"] if s["positions"].dim() == 1 else s["positions"][axis]
            some = slice(start, start + n)
            angle = torch.outer(pos.to(torch.float64), s["freqs"][some])
            turn = torch.polar(torch.ones_like(angle), -angle if back else angle)[:, None, :]
            z = torch.complex(x[..., first[some]], x[..., second[some]]) * turn
            y[..., first[some]], y[..., second[some]] = z.real, z.imag
            start += n
        return y

    if case["path"] == "rotary":
        return turned(f("x"), case["inverse"])
    if case["path"] in ("write", "read"):
        slots = s["slots"].tolist()
        real = [i for i, n in enumerate(slots) if n >= 0]
        at = torch.tensor([slots[i] for i in real], device="cuda")
        where = (torch.div(at, page, rounding_mode="floor"), slice(None), at % page)

        def back(codes, scale, into):
            y = f(into)
            y[real] = codes.to(torch.float64) * (1 if scale is None else scale.to(torch.float64)[..., None])
            return y

        if case["path"] == "read":
            return {w: back(s[w + "_cache"][where], None if s[w + "_scale"] is None else s[w + "_scale"][where], w) for w in ("k", "v")}
        k, v = turned(f("new_k"))[real], f("new_v")[real]
        got = {"q": turned(f("new_q"))}
        for w, y in (("k", k), ("v", v)):
            if not case["int8"]:
                c = f(w + "_cache")
                c[where] = y
                got[w + "_cache"] = c
                continue
            top = torch.linalg.vector_norm(y, ord=math.inf, dim=-1)
            scale = f(w + "_scale")
            scale[where] = top / 127
            got[w + "_scale"] = scale
            got[w] = back(torch.round(127 * y / top[..., None]), top / 127, w)
        return got
    B, T, H, G = case["B"], case["T"], case["Hkv"], case["Hq"] // case["Hkv"]
    out = torch.zeros(B, T, case["Hq"], D, dtype=torch.float64, device="cuda")
    lse = torch.full((B, T, case["Hq"]), -math.inf, dtype=torch.float64, device="cuda")
    for b, n in enumerate(s["lengths"].tolist()):
        if n == 0:
            continue
        pages = s["table"][b, : (n + page - 1) // page].long()
        for h in range(H):
            k, v = (s[w + "_cache"][pages, h].to(torch.float64).reshape(-1, D)[:n] for w in ("k", "v"))
            if case["int8"]:
                k, v = (x * s[w + "_scale"][pages, h].to(torch.float64).reshape(-1, 1)[:n] for x, w in ((k, "k"), (v, "v")))
            for i in range(T):
                last = n - T + i
                if last < 0:
                    continue
                lo = max(0, last - case["window"] + 1) if case["window"] else 0
                mine = slice(h * G, (h + 1) * G)
                z = torch.einsum("gd,nd->gn", s["q"][b, i, mine].to(torch.float64), k[lo: last + 1]) / math.sqrt(D)
                if case["cap"]:
                    z = case["cap"] * torch.tanh(z / case["cap"])
                if case["slopes"]:
                    z = z - torch.outer(s["slopes"][mine].to(torch.float64), (last - torch.arange(lo, last + 1, device="cuda")).to(torch.float64))
                lse[b, i, mine] = torch.logsumexp(z, -1)
                out[b, i, mine] = torch.einsum("gn,nd->gd", torch.softmax(z, -1), v[lo: last + 1])
    return {"out": out, "lse": lse}
