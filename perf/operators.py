"""The operators around a kept scene, as cases that can be timed and compared: norms and rotation of queries and keys (and their
gradients), appending keys and values to a paged cache, attention of a batch to a shared prefix and its own keys.

A case is one pass through one of them.  With `own` false `run` computes it from elementary torch operations in 32 bits, rounded once
at the end; with `own` true it makes the calls a program makes of `paper_2511_21317_b200.kv_cache`.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

_DEVICE = "cuda:0"
_SPECIAL = 5            # special tokens in front of a frame's patches: one camera token and four registers
_EPS = 1e-5
_TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


# ------------------------------------------------------------------------------------------------------------------ cases

def _rows_case(op, frames, grid, heads, kv_heads, dim, **kw):
    """Norms and rotation of a batch of tokens; grid (0, 0): `frames` single tokens of a sequence instead of images."""
    c = {"op": op, "frames": frames, "grid_h": grid[0], "grid_w": grid[1], "heads": heads, "kv_heads": kv_heads, "dim": dim,
         "type": "bf16", "norm": "layer" if grid[0] else "rms", "axes": 2 if grid[0] else 1, "rotated": dim, "interleaved": False,
         "layout": "fused"}
    c.update(kw)
    return c


def _cache_case(op, sequences, shortest, longest, prefix, heads, kv_heads, dim, page, **kw):
    """Sequences with `shortest` .. `longest` new tokens each on top of `past_shortest` .. `past_longest` kept ones, behind a shared prefix;
    `grid_h`, `grid_w`: the new tokens of a sequence are an image instead."""
    c = {"op": op, "sequences": sequences, "shortest": shortest, "longest": longest, "prefix": prefix, "heads": heads,
         "kv_heads": kv_heads, "dim": dim, "page": page, "past_shortest": 0, "past_longest": 0, "type": "bf16", "causal": True,
         "grid_h": 0, "grid_w": 0, "norm": "rms", "interleaved": False, "layout": "fused"}
    c.update(kw)
    return c


def _named(name, case):
    return dict(case, name=name)


def listed():
    image = 37 * 37 + _SPECIAL
    return [
        # One token of one sequence between the projection and the attention of a layer: launches and latency count.
        _named("rows_token", _rows_case("rows", 1, (0, 0), 32, 8, 128)),
        # The benchmark's scene (24 images of 37 x 37 patches): q and k as views of the fused projection output.
        _named("rows_scene", _rows_case("rows", 24, (37, 37), 16, 16, 64)),
        # A packed batch of text-like sequences: half precision, a part of the channels rotated, neighbouring channels paired.
        _named("rows_partial_fp16", _rows_case("rows", 2743, (0, 0), 12, 3, 128, type="fp16", rotated=64, interleaved=True, layout="heads")),
        # A fine-tuning step on a pair of small images (the "tiny" workload).
        _named("back_tiny", _rows_case("back", 4, (16, 16), 16, 16, 64)),
        # A fine-tuning step on the benchmark's scene.
        _named("back_scene", _rows_case("back", 24, (37, 37), 16, 16, 64)),
        # A decoding step: one new token for each of 64 sequences of different lengths, small pages.
        _named("append_tokens", _cache_case("append", 64, 1, 1, 2000, 32, 8, 128, 16, past_longest=1000)),
        # Six new images go to the cache at once.
        _named("append_images", _cache_case("append", 6, image, image, 1000, 16, 16, 64, 128, grid_h=37, grid_w=37, norm="layer")),
        # One token each of a few sequences against a short prefix: latency.
        _named("attend_short", _cache_case("attend", 4, 1, 1, image, 16, 16, 64, 64, past_longest=40)),
        # A decoding step of 32 sequences behind a long common document: the cache's bytes count.
        _named("attend_tokens", _cache_case("attend", 32, 1, 1, 32801, 32, 8, 128, 64, past_longest=2000)),
        # Five drafted tokens for each of 24 sequences, half precision, three query heads to a key head, small pages.
        _named("attend_drafts_fp16", _cache_case("attend", 24, 5, 5, 4001, 24, 8, 128, 16, past_shortest=17, past_longest=900, type="fp16")),
        # Prompts of very different lengths behind a common one.
        _named("attend_prompts", _cache_case("attend", 5, 61, 1500, 6001, 32, 8, 128, 64, past_longest=500)),
        # Four new images looked up in the benchmark's scene, all of their tokens at once.
        _named("attend_images", _cache_case("attend", 4, image, image, 24 * image, 16, 16, 64, 128, grid_h=37, grid_w=37, causal=False,
                                            norm="layer")),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: 1 .. 33 000 tokens, 1 .. 32 heads in groups of 1 .. 8, prefixes of 0 .. 33 000 keys, images and single tokens, both
    types, layouts, norms and pairings, pages of 16 .. 256."""
    top = {"flops": 0.0, "bytes": 0.0}
    for c in listed():
        top = {k: max(top[k], work(c)[k]) for k in top}
    while True:
        op = rng.choice(["rows", "rows", "back", "back", "append", "append", "attend", "attend", "attend", "attend"])
        dim = rng.choice([64, 64, 128])
        kv_heads = rng.choice([1, 2, 3, 4, 8, 8, 16])
        heads = kv_heads * rng.choice([g for g in (1, 1, 2, 3, 4, 5, 8) if g * kv_heads <= 32])
        kind = rng.choice(["bf16", "bf16", "fp16"])
        layout = rng.choice(["fused", "heads"])
        grid = (rng.randint(5, 37), rng.randint(5, 37)) if rng.random() < 0.5 else (0, 0)
        if op in ("rows", "back"):
            frames = _log_int(rng, 1, 24) if grid[0] else _log_int(rng, 1, 33000)
            dim = rng.choice([32, 64, 64, 128, 128, 256])
            axes = 2 if grid[0] else 1
            rotated = dim if rng.random() < 0.7 else rng.randrange(8 * axes, dim + 1, 8 * axes)
            c = _rows_case(op, frames, grid, heads, kv_heads, dim, type=kind, layout=layout, rotated=rotated,
                           norm=rng.choice(["layer", "rms"]), interleaved=rng.random() < 0.3)
        else:
            sequences = _log_int(rng, 1, 64)
            image = grid[0] * grid[1] + _SPECIAL
            longest = image if grid[0] else rng.choice([1, 1, 1, rng.randint(2, 8), _log_int(rng, 2, 1500)])
            shortest = image if grid[0] else max(1, longest // rng.randint(1, 9))
            c = _cache_case(op, sequences, shortest, longest, rng.choice([0, _log_int(rng, 16, 33000), _log_int(rng, 16, 33000)]), heads,
                            kv_heads, dim, rng.choice([16, 32, 64, 128, 256]), past_longest=_log_int(rng, 1, 2000), type=kind,
                            layout=layout, causal=not grid[0], grid_h=grid[0], grid_w=grid[1], norm=rng.choice(["layer", "rms"]),
                            interleaved=rng.random() < 0.3)
            c["past_shortest"] = c["past_longest"] // rng.randint(1, 40)
        w = work(c)
        if all(w[k] <= top[k] for k in top):
            return c


def _spread(lo, hi, n):
    """n whole numbers between lo and hi, unevenly spread and the same every time."""
    return [lo + int((hi - lo) * ((i * 0.6180339887 + 0.37) % 1.0) ** 2 + 0.5) for i in range(n)]


def _lengths(c):
    """(new tokens, tokens kept before) of every sequence."""
    return _spread(c["shortest"], c["longest"], c["sequences"]), _spread(c["past_shortest"], c["past_longest"], c["sequences"])


def _n_rows(c):
    return c["frames"] * (c["grid_h"] * c["grid_w"] + _SPECIAL) if c["grid_h"] else c["frames"]


def work(case):
    c, size = case, 2
    if c["op"] in ("rows", "back"):
        rows = _n_rows(c) * (c["heads"] + c["kv_heads"])
        passes = 2 if c["op"] == "rows" else 3   # x -> y; x, dy -> dx
        return {"bytes": float(passes * rows * c["dim"] * size + 4 * _n_rows(c) * c["axes"] + 32 * c["dim"]),
                "flops": float(rows * c["dim"] * (8 if c["op"] == "rows" else 20))}
    new, past = _lengths(c)
    tokens, own_keys = sum(new), sum(new) + sum(past)
    if c["op"] == "append":
        return {"bytes": float(4 * tokens * c["kv_heads"] * c["dim"] * size), "flops": float(8 * tokens * c["kv_heads"] * c["dim"])}
    pairs = 0
    for n, p in zip(new, past):
        pairs += n * (c["prefix"] + p) + (n * (n + 1) // 2 if c["causal"] else n * n)
    return {"bytes": float(2 * (c["prefix"] + own_keys) * c["kv_heads"] * c["dim"] * size + 2 * tokens * c["heads"] * c["dim"] * size),
            "flops": 4.0 * c["dim"] * c["heads"] * pairs}


# ----------------------------------------------------------------------------------------------------------------- inputs

def _grid_positions(c, images, device):
    """(row, column) of every token of `images` images: 0 for the special tokens, counted from 1 for the patches."""
    h, w = c["grid_h"], c["grid_w"]
    p = torch.zeros(h * w + _SPECIAL, 2, dtype=torch.int32, device=device)
    p[_SPECIAL:, 0] = torch.arange(h, device=device).repeat_interleave(w) + 1
    p[_SPECIAL:, 1] = torch.arange(w, device=device).repeat(h) + 1
    return p.repeat(images, 1)


def _frequencies(c, axes, rotated):
    """Angles per position of the channel pairs of one axis (64 bits)."""
    d = rotated // axes
    return (100.0 if axes == 2 else 10000.0) ** (-2.0 * torch.arange(d // 2, dtype=torch.float64) / d)


def _views(c, tokens, parts, gen):
    """Tensors [heads][tokens][dim] for every (heads, scale) of `parts`: views of one [tokens][all heads][dim] matrix, as a fused
    projection leaves them, or tensors of their own."""
    kind = _TYPES[c["type"]]
    if c["layout"] == "fused":
        whole = torch.randn(tokens, sum(h for h, _ in parts), c["dim"], generator=gen, device=gen.device)
        at = 0
        for h, scale in parts:
            whole[:, at:at + h] *= scale
            at += h
        whole = whole.to(kind)
        return list(t.permute(1, 0, 2) for t in whole.split([h for h, _ in parts], dim=1))
    return [(torch.randn(h, tokens, c["dim"], generator=gen, device=gen.device) * scale).to(kind) for h, scale in parts]


def _norm_weights(c, gen):
    dim, dev = c["dim"], gen.device
    out = {}
    for t in ("q", "k"):
        out[t + "_weight"] = 1.0 + 0.2 * torch.randn(dim, generator=gen, device=dev)
        out[t + "_bias"] = 0.1 * torch.randn(dim, generator=gen, device=dev) if c["norm"] == "layer" else None
    return out


def _inputs(c, seed):
    """What both sides get, from the seed alone."""
    gen = torch.Generator(device=_DEVICE).manual_seed(seed)
    st = {"case": c}
    if c["op"] in ("rows", "back"):
        n = _n_rows(c)
        st["q"], st["k"], _ = _views(c, n, [(c["heads"], 1.7), (c["kv_heads"], 1.3), (c["kv_heads"], 1.0)], gen)
        st.update(_norm_weights(c, gen))
        if c["grid_h"]:
            st["positions"] = _grid_positions(c, c["frames"], _DEVICE)
            st["n_positions"] = max(c["grid_h"], c["grid_w"]) + 1
        else:   # tokens of sequences packed one behind the other
            st["positions"] = (torch.arange(n, device=_DEVICE, dtype=torch.int32) % 4099).view(n, 1)
            st["n_positions"] = 4100
        if c["op"] == "back":
            st["dq"], st["dk"], _ = _views(c, n, [(c["heads"], 0.02), (c["kv_heads"], 0.02), (c["kv_heads"], 1.0)], gen)
        st["frequencies"] = _frequencies(c, c["axes"], c["rotated"])
        return st
    new, past = _lengths(c)
    page, prefix = c["page"], c["prefix"]
    length = [a + b for a, b in zip(new, past)]
    need = [-(-n // page) for n in [prefix] + length]
    n_pages = sum(need) + 3
    order = torch.randperm(n_pages, generator=torch.Generator().manual_seed(seed)).tolist()   # pages in the order a busy pool gives them out
    tables, at = [], 0
    for n in need:
        tables.append(order[at:at + n])
        at += n
    st.update(new=new, length=length, prefix_pages=tables[0], tables=tables[1:], n_pages=n_pages)
    kind = _TYPES[c["type"]]
    shape = (n_pages, c["kv_heads"], page, c["dim"])
    for name in ("k_pages", "v_pages"):
        pool = torch.empty(shape, dtype=kind, device=_DEVICE)
        step = max(1, (1 << 26) // (shape[1] * shape[2] * shape[3]))
        for i in range(0, n_pages, step):
            m = min(step, n_pages - i)
            pool[i:i + m] = torch.randn((m,) + shape[1:], generator=gen, device=_DEVICE).to(kind)
        st[name] = pool
    tokens = sum(new)
    st["q"], st["k"], st["v"] = _views(c, tokens, [(c["heads"], 2.0), (c["kv_heads"], 1.3), (c["kv_heads"], 1.0)], gen)
    if c["op"] == "append":
        st.update(_norm_weights(c, gen))
        axes = 2 if c["grid_h"] else 1
        if c["grid_h"]:
            st["positions"] = _grid_positions(c, c["sequences"], _DEVICE)
            st["n_positions"] = max(c["grid_h"], c["grid_w"]) + 1
        else:   # a token's place behind the prefix
            where = np.concatenate([prefix + np.arange(p, p + n) for n, p in zip(new, past)]).astype(np.int32)
            st["positions"] = torch.from_numpy(where).to(_DEVICE).view(tokens, 1)
            st["n_positions"] = prefix + max(length)
        st["frequencies"] = _frequencies(c, axes, c["dim"])
    return st


def prepare(case, seed):
    c, st = case, _inputs(case, seed)
    kind = _TYPES[c["type"]]
    if c["op"] in ("rows", "back", "append"):   # cos and sin of every position: a program keeps them
        angles = torch.arange(st["n_positions"], dtype=torch.float64)[:, None] * st["frequencies"][None]
        st["cos"], st["sin"] = angles.cos().float().to(_DEVICE), angles.sin().float().to(_DEVICE)
    if c["op"] in ("append", "attend"):   # where every new token goes, and the pages of every sequence
        page = c["page"]
        rows = [[(t[p // page], p % page) for p in range(n - m, n)] for t, n, m in zip(st["tables"], st["length"], st["new"])]
        flat = torch.tensor([x for r in rows for x in r], dtype=torch.long).view(-1, 2).to(_DEVICE)
        st["page_of"], st["slot_of"] = flat[:, 0].contiguous(), flat[:, 1].contiguous()
        st["prefix_index"] = torch.tensor(st["prefix_pages"], dtype=torch.long, device=_DEVICE)
        st["table_index"] = [torch.tensor(t, dtype=torch.long, device=_DEVICE) for t in st["tables"]]
    if c["op"] in ("rows", "back"):
        st["out"] = [torch.empty(t.shape, dtype=kind, device=_DEVICE) for t in (st["q"], st["k"])]
    if c["op"] == "attend":
        st["out"] = torch.empty(st["q"].shape[1], c["heads"] * c["dim"], dtype=kind, device=_DEVICE)
    if own:
        from paper_2511_21317_b200 import kv_cache as kc
        if c["op"] != "attend":
            axes = c["axes"] if c["op"] != "append" else (2 if c["grid_h"] else 1)
            rotated = c["rotated"] if c["op"] != "append" else c["dim"]
            st["rotary"] = kc.Rotary(head_dim=c["dim"], n_positions=st["n_positions"], axes=axes, rotated_dim=rotated,
                                     frequencies=st["frequencies"].tolist(), interleaved=c["interleaved"], norm=c["norm"], eps=_EPS)
        if c["op"] in ("append", "attend"):
            st["cache"] = kc.KvCache(st["k_pages"], st["v_pages"])
            st["batch"] = kc.CacheBatch(heads=c["heads"], kv_heads=c["kv_heads"], head_dim=c["dim"], page_size=c["page"],
                                        n_pages=st["n_pages"], causal=c["causal"])
            st["batch"].set(st["tables"], st["length"], st["new"], st["prefix_pages"], c["prefix"])
    return st


# -------------------------------------------------------------------------------------------------------------------- run

def _pair_index(dim, axes, rotated, interleaved):
    """Channels a and b of every rotated pair, pairs of axis 0 first."""
    d = rotated // axes
    i = torch.arange(d // 2, device=_DEVICE)
    a = torch.cat([x * d + (2 * i if interleaved else i) for x in range(axes)])
    return a, a + (1 if interleaved else d // 2)


def _angles(st, axes):
    """cos and sin [tokens][pairs] of the tokens' positions."""
    pos = st["positions"].long()
    return (torch.cat([t[pos[:, x]] for x in range(axes)], dim=1) for t in (st["cos"], st["sin"]))


def _normalised(x, norm):
    """(x - mean) / deviation in 32 bits, and 1 / deviation."""
    x = x.float()
    if norm == "layer":
        x = x - x.mean(dim=-1, keepdim=True)
    r = torch.rsqrt((x * x).mean(dim=-1, keepdim=True) + _EPS)
    return x * r, r


def _plain_rows(x, weight, bias, cos, sin, a, b, norm):
    z, _ = _normalised(x, norm)
    z = z * weight
    if bias is not None:
        z = z + bias
    y = z.clone()
    y[..., a] = z[..., a] * cos - z[..., b] * sin
    y[..., b] = z[..., a] * sin + z[..., b] * cos
    return y


def _plain_back(x, dy, weight, cos, sin, a, b, norm):
    xh, r = _normalised(x, norm)
    dy = dy.float()
    g = dy.clone()
    g[..., a] = dy[..., a] * cos + dy[..., b] * sin
    g[..., b] = dy[..., b] * cos - dy[..., a] * sin
    u = g * weight
    dx = u - xh * (u * xh).mean(dim=-1, keepdim=True)
    if norm == "layer":
        dx = dx - u.mean(dim=-1, keepdim=True)
    return dx * r, (g * xh).sum(dim=(0, 1)), g.sum(dim=(0, 1))


def _keys_of(pool, index, n):
    """The first n rows [kv heads][n][dim] of the pages `index`, in 32 bits."""
    t = pool[index]                                                      # [pages][kv heads][page][dim]
    return t.permute(1, 0, 2, 3).reshape(t.shape[1], t.shape[0] * t.shape[2], t.shape[3])[:, :n].float()


def _plain_attention(st):
    c = st["case"]
    group, scale = c["heads"] // c["kv_heads"], c["dim"] ** -0.5
    pk, pv = (_keys_of(st[p], st["prefix_index"], c["prefix"]) for p in ("k_pages", "v_pages"))
    q = st["q"].float() * scale
    tokens = q.shape[1]
    out = st["out"].view(tokens, c["heads"], c["dim"])
    own_keys = []
    for index, n in zip(st["table_index"], st["length"]):
        own_keys.append((_keys_of(st["k_pages"], index, n), _keys_of(st["v_pages"], index, n)))
    for h in range(c["kv_heads"]):
        qh = q[h * group:(h + 1) * group]                                 # [group][tokens][dim]
        shared = torch.matmul(qh, pk[h].t())                              # scores of all tokens against the prefix, once
        at = 0
        for (k, v), n, m in zip(own_keys, st["length"], st["new"]):
            s = torch.matmul(qh[:, at:at + m], k[h].t())                  # [group][m][n]
            if c["causal"]:
                i = torch.arange(m, device=_DEVICE)[:, None] + (n - m)
                s = s.masked_fill(torch.arange(n, device=_DEVICE)[None] > i, float("-inf"))
            both = torch.cat([shared[:, at:at + m], s], dim=-1)
            e = torch.exp(both - both.amax(dim=-1, keepdim=True))
            o = torch.matmul(e[..., :c["prefix"]], pv[h]) + torch.matmul(e[..., c["prefix"]:], v[h])
            o = o / e.sum(dim=-1, keepdim=True)
            out[at:at + m, h * group:(h + 1) * group] = o.permute(1, 0, 2).to(out.dtype)
            at += m
    return st["out"]


def run(state):
    st, c = state, state["case"]
    op = c["op"]
    if own:
        if op == "rows":
            return st["rotary"].norm_rotate(st["q"], st["k"], st["positions"], st["q_weight"], st["k_weight"], st["q_bias"], st["k_bias"],
                                            out_q=st["out"][0], out_k=st["out"][1])
        if op == "back":
            grads = st["rotary"].norm_rotate_backward(st["dq"], st["dk"], st["q"], st["k"], st["positions"], st["q_weight"], st["k_weight"],
                                                      st["q_bias"], st["k_bias"], out_q=st["out"][0], out_k=st["out"][1])
            return tuple(g for g in grads if g is not None)   # no gradient of a bias that is not there
        if op == "append":
            st["cache"].append(st["batch"], st["k"], st["v"], rotary=st["rotary"], positions=st["positions"], k_weight=st["k_weight"],
                               k_bias=st["k_bias"])
            return st["k_pages"], st["v_pages"]
        return st["cache"].attention(st["batch"], st["q"], out=st["out"])
    if op == "attend":
        return _plain_attention(st)
    axes, rotated = (c["axes"], c["rotated"]) if op != "append" else ((2 if c["grid_h"] else 1), c["dim"])
    a, b = _pair_index(c["dim"], axes, rotated, c["interleaved"])
    cos, sin = _angles(st, axes)
    if op == "rows":
        for t, out in zip(("q", "k"), st["out"]):
            out.copy_(_plain_rows(st[t], st[t + "_weight"], st[t + "_bias"], cos, sin, a, b, c["norm"]))
        return tuple(st["out"])
    if op == "back":
        sums = []
        for t, out in zip(("q", "k"), st["out"]):
            dx, dw, db = _plain_back(st[t], st["d" + t], st[t + "_weight"], cos, sin, a, b, c["norm"])
            out.copy_(dx)
            sums += [dw, db if st[t + "_bias"] is not None else None]
        return tuple(st["out"]) + tuple(s for s in sums if s is not None)
    y = _plain_rows(st["k"], st["k_weight"], st["k_bias"], cos, sin, a, b, c["norm"])
    st["k_pages"][st["page_of"], :, st["slot_of"]] = y.permute(1, 0, 2).to(st["k_pages"].dtype)
    st["v_pages"][st["page_of"], :, st["slot_of"]] = st["v"].permute(1, 0, 2)
    return st["k_pages"], st["v_pages"]


# ------------------------------------------------------------------------------------------------------------------ exact

def _exact_rows(x, weight, bias, turn, norm, pairing):
    """One tensor's rows in 64 bits, with the rotation as a product of complex numbers.  turn: [tokens][axes][pairs of an axis]."""
    x = x.double()
    centred = x - x.mean(-1, keepdim=True) if norm == "layer" else x
    z = centred / torch.sqrt(centred.square().mean(-1, keepdim=True) + _EPS) * weight.double()
    if bias is not None:
        z = z + bias.double()
    axes, half = turn.shape[1:]
    head = z[..., :axes * 2 * half].reshape(*z.shape[:2], axes, 2 * half)
    if pairing:
        t = torch.view_as_complex(head.reshape(*head.shape[:3], half, 2).contiguous()) * turn
        head = torch.view_as_real(t).reshape(head.shape)
    else:
        t = torch.complex(head[..., :half].contiguous(), head[..., half:].contiguous()) * turn
        head = torch.cat([t.real, t.imag], -1)
    return torch.cat([head.reshape(*z.shape[:2], -1), z[..., axes * 2 * half:]], -1)


def _exact_attention(c, st):
    tokens, heads, dim = st["q"].shape[1], c["heads"], c["dim"]
    out = torch.empty(tokens, heads, dim, dtype=torch.float64, device=_DEVICE)
    first = 0
    for table, n, m in zip(st["tables"], st["length"], st["new"]):
        at = [(p, s) for pages, total in ((st["prefix_pages"], c["prefix"]), (table, n)) for i, p in enumerate(pages)
              for s in range(min(c["page"], total - i * c["page"]))]
        pages, slots = torch.tensor(at, dtype=torch.long, device=_DEVICE).T
        for g in range(c["kv_heads"]):
            k, v = st["k_pages"][pages, g, slots].double(), st["v_pages"][pages, g, slots].double()
            seen = torch.arange(len(k), device=_DEVICE)
            for h in range(g * heads // c["kv_heads"], (g + 1) * heads // c["kv_heads"]):
                for i in range(0, m, 512):
                    rows = torch.arange(i, min(m, i + 512), device=_DEVICE)
                    s = st["q"][h, first + rows].double() @ k.T / math.sqrt(dim)
                    if c["causal"]:
                        s = s.where(seen[None, :] <= (c["prefix"] + n - m + rows)[:, None], -math.inf)
                    out[first + rows, h] = s.softmax(-1) @ v
        first += m
    return out.view(tokens, heads * dim)


def exact(case, seed):
    c = case
    if c["op"] == "attend" and work(c)["flops"] > 1e12:
        return None
    st = _inputs(c, seed)
    if c["op"] == "attend":
        return _exact_attention(c, st)
    angle = st["positions"].double()[:, :, None] * st["frequencies"].to(_DEVICE)[None, None, :]
    turn = torch.polar(torch.ones_like(angle), angle)
    names = ("q", "k") if c["op"] != "append" else ("k",)
    grads, outs = [], []
    for t in names:
        x, w = st[t].double(), st[t + "_weight"].double()
        b = st[t + "_bias"].double() if st[t + "_bias"] is not None else None
        if c["op"] != "back":
            outs.append(_exact_rows(x, w, b, turn, c["norm"], c["interleaved"]))
            continue
        wants = [v.detach().clone().requires_grad_(True) for v in (x, w, b) if v is not None]
        y = _exact_rows(wants[0], wants[1], wants[2] if b is not None else None, turn, c["norm"], c["interleaved"])
        got = torch.autograd.grad(y, wants, st["d" + t].double())
        outs.append(got[0])
        grads += got[1:]
    if c["op"] != "append":
        return tuple(outs) + tuple(grads)
    pools = [st["k_pages"].double(), st["v_pages"].double()]
    at = 0
    for table, n, m in zip(st["tables"], st["length"], st["new"]):
        for p in range(n - m, n):
            pools[0][table[p // c["page"]], :, p % c["page"]] = outs[0][:, at]
            pools[1][table[p // c["page"]], :, p % c["page"]] = st["v"][:, at].double()
            at += 1
    return tuple(pools)
