"""The paged cache and the attention over it, against a plain implementation in 64 bits.  Needs a B200.

Tolerances of the attention.  With p the weights and o = sum p v / sum p: each p is rounded once to the values' type before it meets v (half a
step: 2^-8 in bf16, whose significand has 8 bits, 2^-11 in fp16, and 2^-25 absolutely below fp16's normal range, where the largest weight of a row is at least 1 / 2^8), the
exponential is good to 2^-20, and the scores, sums of head_dim products in 32 bits, to (head_dim / 4) 2^-24 of the sum of the products' sizes,
which shifts a weight by as much relatively.  Hence |error| <= (step + 2 d + 2^-18) sum p |v| / sum p + step |o|, d that bound on the scores."""
import pytest
import torch

from paper_2511_21317_b200 import binding as hb
from paper_2511_21317_b200 import kv_cache as kc

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
STEP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


class Scene:
    """Sequences over pages in a shuffled order; everything that no sequence owns, and every place past a length, holds NaN or infinity."""

    def __init__(self, lengths, queries, prefix, heads, kv_heads, dim, page, dtype=torch.bfloat16, causal=True, seed=0, order="nhsd", layout="heads",
                 spread=1.0):
        gen = torch.Generator(device=DEV).manual_seed(seed)
        self.lengths, self.queries, self.prefix, self.page, self.dtype, self.causal = lengths, queries, prefix, page, dtype, causal
        self.heads, self.kv_heads, self.dim = heads, kv_heads, dim
        need = [-(-n // page) for n in [prefix] + list(lengths)]
        n_pages = sum(need) + 2
        ids = torch.randperm(n_pages, generator=torch.Generator().manual_seed(seed)).tolist()
        self.tables, at = [], 0
        for n in need:
            self.tables.append(ids[at:at + n])
            at += n
        self.prefix_pages = self.tables.pop(0)
        self.n_pages = n_pages
        shape = {"nhsd": (n_pages, kv_heads, page, dim), "nshd": (n_pages, page, kv_heads, dim), "hnsd": (kv_heads, n_pages, page, dim)}[order]
        back = {"nhsd": (0, 1, 2, 3), "nshd": (0, 2, 1, 3), "hnsd": (1, 0, 2, 3)}[order]
        junk = torch.tensor([float("nan"), float("inf"), -float("inf")], device=DEV)
        self.pools = []
        for scale in (spread, 1.0):
            pool = junk[torch.randint(0, 3, shape, generator=gen, device=DEV)].to(dtype).permute(*back)
            for table, n in [(self.prefix_pages, prefix)] + list(zip(self.tables, lengths)):
                for i, p in enumerate(table):
                    m = min(page, n - i * page)
                    pool[p, :, :m] = (torch.randn(kv_heads, m, dim, generator=gen, device=DEV) * scale).to(dtype)
            self.pools.append(pool)
        self.cache = kc.KvCache(*self.pools)
        self.batch = kc.CacheBatch(heads, kv_heads, dim, page, n_pages, causal)
        self.batch.set(self.tables, lengths, queries, self.prefix_pages, prefix)
        t = sum(queries)
        q = (torch.randn(heads, t, dim, generator=gen, device=DEV) * spread).to(dtype)
        if layout == "fused":
            whole = torch.full((t, heads + 2, dim), 7.0, dtype=dtype, device=DEV)
            whole[:, 1:1 + heads] = q.permute(1, 0, 2)
            q = whole[:, 1:1 + heads].permute(1, 0, 2)
        self.q = q

    def keys(self, i):
        """Keys and values [kv_heads][n][dim] that sequence i sees, in 64 bits: the prefix, then its own."""
        out = []
        for pool in self.pools:
            parts = [pool[p, :, :min(self.page, n - j * self.page)] for table, n in ((self.prefix_pages, self.prefix), (self.tables[i], self.lengths[i]))
                     for j, p in enumerate(table)]
            out.append(torch.cat(parts, 1).double() if parts else torch.zeros(self.kv_heads, 0, self.dim, dtype=torch.float64, device=DEV))
        return out

    def check(self, out, scale=None, what=""):
        scale = self.dim ** -0.5 if scale is None else scale
        out = out.view(-1, self.heads, self.dim).double()
        step, g, at = STEP[self.dtype], self.heads // self.kv_heads, 0
        for i, (n, m) in enumerate(zip(self.lengths, self.queries)):
            if m == 0:
                continue
            k, v = (t.repeat_interleave(g, 0) for t in self.keys(i))
            q = self.q[:, at:at + m].double()
            s = scale * q @ k.transpose(1, 2)
            sees = torch.ones(m, self.prefix + n, dtype=torch.bool, device=DEV)
            if self.causal:
                sees = torch.arange(self.prefix + n, device=DEV)[None] <= (self.prefix + n - m + torch.arange(m, device=DEV))[:, None]
                sees[:, :self.prefix] = True
            s = s.masked_fill(~sees, -float("inf"))
            empty = ~sees.any(1)
            p = torch.softmax(s, -1)
            p[:, empty] = 0.0
            want, size = p @ v, p @ v.abs()
            if k.shape[1] > 0:
                d = self.dim / 4 * 2.0 ** -24 * abs(scale) * (q.abs() @ k.abs().transpose(1, 2)).amax(-1, keepdim=True)
            else:
                d = torch.zeros(self.heads, m, 1, dtype=torch.float64, device=DEV)
            tiny = 0.0
            if self.dtype == torch.float16:   # weights below the normal range
                many = torch.minimum(sees.sum(1)[None, :, None].double() * 2.0 ** -14, torch.tensor(1.0, device=DEV))
                tiny = 2.0 ** -25 + 2.0 ** -17 * many * (v.abs().amax() if v.numel() else 0.0)
            got = out[at:at + m].permute(1, 0, 2)
            bad = (got - want).abs() - ((step + 2 * d + 2.0 ** -18) * size + step * want.abs() + tiny)
            assert not got.isnan().any(), f"{what} sequence {i}: not a number"
            assert (bad <= 0).all(), f"{what} sequence {i}: off by {(got - want).abs().max():.3e}, over the bound by {bad.max():.3e}"
            assert (got[:, empty] == 0).all()
            at += m


ATTEND = {
    # lengths, queries, prefix, heads, kv heads, dim, page, others
    "one key": ([1], [1], 0, 4, 4, 64, 16, {}),
    "one token, prefix alone": ([0], [1], 77, 4, 4, 64, 16, dict(causal=False)),
    "nothing to see": ([0, 5, 0], [2, 1, 1], 0, 2, 2, 64, 16, dict(causal=False)),
    "nothing to see, others do": ([0, 5, 3], [2, 0, 4], 0, 2, 2, 128, 16, dict(causal=True)),
    "tokens": ([9, 1, 130, 64, 65, 300], [1] * 6, 200, 16, 16, 64, 64, {}),
    "tokens, groups of 4": ([9, 1, 130, 64, 65, 300, 7, 8], [1] * 8, 1000, 32, 8, 128, 16, {}),
    "tokens, groups of 3, fp16": ([33, 48, 17], [1] * 3, 129, 9, 3, 128, 32, dict(dtype=torch.float16)),
    "tokens, groups of 5": ([33, 48, 17, 1, 90], [1] * 5, 64, 10, 2, 64, 128, dict(layout="fused")),
    "one key head": ([40, 41], [1, 1], 300, 17, 1, 64, 256, {}),
    "drafts": ([12, 80, 5, 200, 31], [5, 3, 5, 2, 4], 250, 12, 4, 128, 16, dict(order="nshd")),
    "drafts, 32 rows": ([12, 80, 50], [8, 7, 8], 250, 8, 2, 64, 16, dict(order="hnsd")),
    "drafts, 64 rows, fp16": ([64, 80, 150], [16, 15, 13], 190, 8, 2, 128, 64, dict(dtype=torch.float16)),
    "all at once": ([20, 300, 70], [20, 300, 70], 0, 4, 4, 64, 32, {}),
    "prompts behind a prefix": ([150, 129, 257, 128], [100, 129, 250, 127], 333, 8, 2, 128, 64, dict(layout="fused")),
    "prompts, groups of 3": ([150, 129], [100, 129], 130, 6, 2, 64, 16, {}),
    "images": ([261, 261, 200], [261, 261, 200], 600, 4, 4, 64, 128, dict(causal=False, layout="fused")),
    "images, fp16": ([261, 133], [261, 133], 128, 2, 2, 128, 256, dict(causal=False, dtype=torch.float16)),
    "tokens among prompts": ([50, 300, 7, 200, 9, 10], [1, 290, 1, 130, 2, 1], 140, 4, 2, 64, 64, {}),
    "no prefix, tokens among prompts": ([50, 300, 7, 200], [1, 290, 1, 130], 0, 4, 2, 128, 16, {}),
    "more queries than keys": ([10, 3], [30, 200], 0, 4, 2, 64, 16, {}),
    "other states": ([100, 37, 0, 260], [5, 150, 3, 1], 0, 4, 4, 64, 64, dict(causal=False)),
    "groups of 64": ([40, 90], [1, 3], 100, 64, 1, 64, 64, {}),
    "groups of 17": ([40, 90], [2, 9], 100, 34, 2, 128, 32, {}),
    "many sequences": (list(range(1, 140)), [1] * 139, 500, 4, 2, 64, 16, {}),
    "long": ([3000, 5], [1, 1], 20011, 4, 2, 128, 64, {}),
    "sharp scores": ([100, 200, 90], [1, 3, 80], 700, 4, 4, 64, 64, dict(spread=3.0)),
    "sharp scores, prompts, fp16": ([300, 290], [300, 140], 700, 4, 4, 128, 64, dict(spread=2.5, dtype=torch.float16)),
}


@pytest.mark.parametrize("name", ATTEND)
def test_attention(name):
    *a, kw = ATTEND[name]
    sc = Scene(*a, **kw, seed=len(name))
    out = torch.full((sum(sc.queries), sc.heads * sc.dim), float("nan"), dtype=sc.dtype, device=DEV)
    sc.cache.attention(sc.batch, sc.q, out)
    assert sc.batch.status() == 0
    sc.check(out, what=name)
    again = sc.cache.attention(sc.batch, sc.q)
    assert torch.equal(again, out)   # no sum depends on who arrives first


def test_scale_and_output_layouts():
    sc = Scene([30, 200], [2, 150], 90, 4, 2, 64, 16, seed=3)
    sc.check(sc.cache.attention(sc.batch, sc.q, scale=0.37), scale=0.37)
    sc.check(sc.cache.attention(sc.batch, sc.q, scale=-0.2), scale=-0.2)
    sc.check(sc.cache.attention(sc.batch, sc.q, scale=0.0), scale=0.0)
    whole = torch.full((152, 6, 64), 7.0, dtype=torch.bfloat16, device=DEV)
    sc.check(sc.cache.attention(sc.batch, sc.q, out=whole[:, 1:5]).contiguous())
    assert (whole[:, 0] == 7).all() and (whole[:, 5] == 7).all()


def test_scores_that_rise_from_tile_to_tile():
    """Every later key tile has larger scores by far (the running maximum moves at every tile), or only smaller ones."""
    for rise in (0.4, -0.4):
        for queries, heads in ([1, 1], 2), ([140, 150], 4):
            sc = Scene([700, 650], queries, 900, heads, 2, 64, 64, causal=False, seed=4)
            direction = torch.ones(64, device=DEV) / 8
            for table, n, first in [(sc.prefix_pages, 900, 0)] + [(t, n, 900) for t, n in zip(sc.tables, sc.lengths)]:
                for i, p in enumerate(table):
                    m = min(64, n - 64 * i)
                    place = (first + 64 * i + torch.arange(m, device=DEV)).float()
                    sc.pools[0][p, :, :m] += (rise * place[:, None] * direction).to(sc.dtype)
            sc.q += (8 * direction).to(sc.dtype)
            sc.check(sc.cache.attention(sc.batch, sc.q), what=f"rise {rise}")


def test_a_query_or_a_sequence_that_is_not_a_number_stays_alone():
    sc = Scene([40, 170, 9, 300], [1, 160, 2, 150], 150, 4, 2, 64, 16, seed=5)
    ref = sc.cache.attention(sc.batch, sc.q).clone()
    sc.q[1, 30] = float("nan")
    got = sc.cache.attention(sc.batch, sc.q)
    same = torch.ones(sum(sc.queries), 4, dtype=torch.bool, device=DEV)
    same[30, 1] = False
    assert got.view(-1, 4, 64)[30, 1].isnan().all() and torch.equal(got.view(-1, 4, 64)[same], ref.view(-1, 4, 64)[same])
    for pool in sc.pools:   # the keys and values of sequence 2 (tokens 161 and 162)
        for p in sc.tables[2]:
            pool[p] = float("inf")
    sc.q[1, 30] = 0.5
    ref[30] = sc.cache.attention(sc.batch, sc.q)[30]
    got = sc.cache.attention(sc.batch, sc.q)
    assert got[161:163].isnan().all() and torch.equal(got[:161], ref[:161]) and torch.equal(got[163:], ref[163:])


def test_an_infinite_score_below_all_others():
    """A key whose score is minus infinity takes no weight."""
    sc = Scene([70], [1], 130, 2, 2, 64, 16, seed=6)
    sc.q.abs_().add_(0.1)
    ref = sc.cache.attention(sc.batch, sc.q).clone()
    sc.pools[0][sc.prefix_pages[0], :, 5] = -float("inf")
    got = sc.cache.attention(sc.batch, sc.q)
    assert not got.isnan().any() and not torch.equal(got, ref)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_one_key_that_is_not_a_number_reaches_every_row_that_sees_it(dtype):
    """Whatever the place of the key in its tile, and whether it is the row's first tile or not."""
    sc = Scene([300, 10], [290, 1], 200, 4, 2, 64, 16, dtype=dtype, seed=11)
    ref = sc.cache.attention(sc.batch, sc.q).clone()
    for place in list(range(16)) + [130, 137, 199]:
        p, slot = sc.prefix_pages[place // 16], place % 16
        kept = sc.pools[0][p, :, slot].clone()
        sc.pools[0][p, :, slot, 3] = float("nan")
        assert sc.cache.attention(sc.batch, sc.q).isnan().all(), place
        sc.pools[0][p, :, slot] = kept
    p = sc.tables[0][100 // 16]   # an own key that tokens 90 .. of the first sequence see (token i sees keys up to 10 + i)
    for slot in range(100 % 16, 100 % 16 + 1):
        sc.pools[0][p, :, slot, 3] = float("nan")
        got = sc.cache.attention(sc.batch, sc.q)
        assert got[90:290].isnan().all() and torch.equal(got[:90], ref[:90]) and torch.equal(got[290:], ref[290:])


def test_append_then_attend():
    """Tokens go to their places and nothing else is written; the attention then sees them."""
    for dtype, dim, page, order, layout in ((torch.bfloat16, 64, 16, "nhsd", "fused"), (torch.float16, 128, 64, "nshd", "heads"),
                                            (torch.bfloat16, 128, 256, "hnsd", "fused")):
        lengths, queries = [40, 17, 300, 6, 1], [3, 17, 130, 0, 1]
        sc = Scene(lengths, queries, 100, 6, 2, dim, page, dtype=dtype, order=order, seed=page)
        gen = torch.Generator(device=DEV).manual_seed(page)
        t = sum(queries)
        whole = torch.randn(t, 4, dim, generator=gen, device=DEV).to(dtype)
        k, v = (whole[:, 2 * i:2 * i + 2].permute(1, 0, 2) for i in range(2))
        if layout == "heads":
            k, v = k.contiguous(), v.contiguous()
        want = [p.clone() for p in sc.pools]
        at = 0
        for table, n, m in zip(sc.tables, lengths, queries):
            for j in range(n - m, n):
                want[0][table[j // page], :, j % page] = k[:, at]
                want[1][table[j // page], :, j % page] = v[:, at]
                at += 1
        sc.cache.append(sc.batch, k, v)
        assert sc.batch.status() == 0
        for got, w in zip(sc.pools, want):
            assert torch.equal(got.view(torch.int16), w.view(torch.int16))
        sc.check(sc.cache.attention(sc.batch, sc.q), what="after append")


@pytest.mark.parametrize("norm,axes,dim,dtype", [("rms", 1, 128, torch.bfloat16), ("layer", 2, 64, torch.bfloat16), ("rms", 1, 64, torch.float16),
                                                 ("none", 1, 64, torch.bfloat16)])
def test_append_norms_and_rotates_as_norm_rotate_does(norm, axes, dim, dtype):
    lengths, queries = [40, 17, 300, 6, 1], [3, 17, 130, 0, 1]
    sc = Scene(lengths, queries, 100, 4, 2, dim, 16, dtype=dtype, seed=8)
    gen = torch.Generator(device=DEV).manual_seed(1)
    t = sum(queries)
    k, v = ((torch.randn(2, t, dim, generator=gen, device=DEV)).to(dtype) for _ in range(2))
    w = 1.0 + 0.2 * torch.randn(dim, generator=gen, device=DEV) if norm != "none" else None
    b = 0.2 * torch.randn(dim, generator=gen, device=DEV) if norm == "layer" else None
    rot = kc.Rotary(dim, 500, axes=axes, base=100.0, norm=norm, eps=1e-6)
    if axes == 2:
        pos = torch.randint(0, 500, (t, 2), generator=gen, device=DEV, dtype=torch.int32)
    else:
        pos = torch.cat([100 + torch.arange(n - m, n) for n, m in zip(lengths, queries)]).to(torch.int32).to(DEV).view(t, 1)
    rows = rot.norm_rotate(None, k, pos, None, w, None, b)[1]
    for given in ([pos] if axes == 2 else [pos, None]):
        sc.cache.append(sc.batch, k, v, rotary=rot, positions=given, k_weight=w, k_bias=b)
        at = 0
        for table, n, m in zip(sc.tables, lengths, queries):
            for j in range(n - m, n):
                assert torch.equal(sc.pools[0][table[j // 16], :, j % 16], rows[:, at]) and torch.equal(sc.pools[1][table[j // 16], :, j % 16], v[:, at])
                at += 1
        sc.pools[0].fill_(0)
        sc.pools[1].fill_(0)
    assert sc.batch.status() == 0


def test_places_beyond_32_bits():
    """A pool of more than 2^31 elements: places in its far end."""
    page, dim, n_pages = 256, 128, 68000
    if torch.cuda.mem_get_info()[0] < 12 << 30:
        pytest.skip("needs 10 GB")
    pools = [torch.zeros(n_pages, 1, page, dim, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    assert pools[0].numel() > 1 << 31
    gen = torch.Generator(device=DEV).manual_seed(2)
    cache = kc.KvCache(*pools)
    tables, prefix = [[67999, 3], [67000]], [66000, 5]
    for queries in ([1, 2], [200, 1]):
        batch = kc.CacheBatch(2, 1, dim, page, n_pages)
        lengths = [300, 9]
        batch.set([[66000, 5]], [400], [400])
        k, v = (torch.randn(1, 400, dim, generator=gen, device=DEV).to(torch.bfloat16) for _ in range(2))
        cache.append(batch, k, v)
        batch.set(tables, lengths, lengths, prefix, 400)
        k2, v2 = (torch.randn(1, 309, dim, generator=gen, device=DEV).to(torch.bfloat16) for _ in range(2))
        cache.append(batch, k2, v2)
        batch.set(tables, lengths, queries, prefix, 400)
        q = torch.randn(2, sum(queries), dim, generator=gen, device=DEV).to(torch.bfloat16)
        out = cache.attention(batch, q).view(-1, 2, dim)
        at = 0
        for i, (n, m) in enumerate(zip(lengths, queries)):
            ks = torch.cat([k, k2[:, 300 * i:300 * i + n]], 1).double()[0]
            vs = torch.cat([v, v2[:, 300 * i:300 * i + n]], 1).double()[0]
            s = q[:, at:at + m].double() @ ks.T * dim ** -0.5
            s = s.masked_fill(torch.arange(400 + n, device=DEV)[None] > (400 + n - m + torch.arange(m, device=DEV))[:, None], -float("inf"))
            p = s.softmax(-1)
            want, size = p @ vs, p @ vs.abs()
            # (scores of order 1: their own error is far below the rounding of the weights)
            assert ((out[at:at + m].permute(1, 0, 2).double() - want).abs() <= 2.0 ** -8 * want.abs() + (2.0 ** -8 + 2.0 ** -16) * size).all()
            at += m


def test_batches_of_changing_size_and_layers_back_to_back():
    """One batch handle, set again for every step with calls of several layers in flight, on a stream of its own."""
    s = torch.cuda.Stream()
    small, large = Scene([9, 30], [1, 1], 64, 4, 2, 64, 16, seed=1), Scene([400, 30, 77], [350, 1, 70], 200, 4, 2, 64, 16, seed=2)
    batch = kc.CacheBatch(4, 2, 64, 16, 1)
    torch.cuda.synchronize()
    with pytest.raises(hb.HttmError):
        batch.set(small.tables, small.lengths, small.queries, small.prefix_pages, 64)   # pages that it has not got
    batch = kc.CacheBatch(4, 2, 64, 16, min(small.n_pages, large.n_pages))
    outs = []
    with pytest.raises(hb.HttmError):
        small.cache.attention(batch, small.q)   # not set yet
    big = kc.CacheBatch(4, 2, 64, 16, max(small.n_pages, large.n_pages))
    with torch.cuda.stream(s):
        for i in range(6):
            sc = (small, large)[i % 2]
            b = kc.CacheBatch(4, 2, 64, 16, sc.n_pages) if i == 0 else None
            use = sc.batch if b is None else b
            use.set(sc.tables, sc.lengths, sc.queries, sc.prefix_pages, sc.prefix)
            outs.append([sc.cache.attention(use, sc.q) for _ in range(3)])
    s.synchronize()
    for i, layers in enumerate(outs):
        for out in layers:
            (small, large)[i % 2].check(out)
    big.set([], [], [])
    assert small.n_pages <= big.n_pages


def test_a_captured_step_can_be_replayed():
    sc = Scene([90, 300, 8], [1, 200, 1], 150, 4, 2, 64, 16, seed=9)
    want = sc.cache.attention(sc.batch, sc.q).clone()
    out = torch.zeros_like(want)
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        sc.cache.attention(sc.batch, sc.q, out)
    out.zero_()
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)


def test_empty_batches():
    sc = Scene([9, 30], [0, 0], 64, 4, 2, 64, 16, seed=1)
    assert sc.cache.attention(sc.batch, sc.q).shape == (0, 256)
    sc.cache.append(sc.batch, sc.q[:2], sc.q[:2])
    sc.batch.set([], [], [], sc.prefix_pages, 64)
    assert sc.cache.attention(sc.batch, sc.q).shape == (0, 256)


def test_refusals():
    sc = Scene([40, 30], [3, 2], 64, 4, 2, 64, 16, seed=1)
    k, v = (torch.zeros(2, 5, 64, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    T, L, Q, P = sc.tables, sc.lengths, sc.queries, sc.prefix_pages

    def refuses(code, f, *a, **kw):
        with pytest.raises(hb.HttmError) as e:
            f(*a, **kw)
        assert e.value.code == code, str(e.value)

    b = sc.batch
    refuses(-1, sc.cache.attention, b, sc.q.half())
    refuses(-1, sc.cache.attention, b, sc.q[:, :4])
    refuses(-1, sc.cache.attention, b, sc.q[:2])
    refuses(-1, sc.cache.attention, b, sc.q, scale=float("nan"))
    refuses(-1, sc.cache.attention, b, sc.q, out=torch.empty(5, 255, dtype=torch.bfloat16, device=DEV))
    refuses(-1, sc.cache.attention, b, sc.q, out=sc.q.permute(1, 0, 2))                      # out is q
    refuses(-1, sc.cache.attention, kc.CacheBatch(4, 2, 64, 32, 4), sc.q)                    # another page size
    refuses(-1, sc.cache.attention, kc.CacheBatch(4, 2, 64, 16, sc.n_pages + 1), sc.q)       # more pages than the cache has
    refuses(-1, sc.cache.append, b, k, v, k_weight=torch.ones(64, device=DEV))               # a norm without its handle
    refuses(-1, sc.cache.append, b, k[:1], v)
    refuses(-1, sc.cache.append, b, k, v, rotary=kc.Rotary(64, 50))                          # places 64 + 37 .. are outside the table
    refuses(-1, sc.cache.append, b, k, v, rotary=kc.Rotary(64, 50, axes=2))                  # two axes need positions
    refuses(-1, sc.cache.append, b, k, v, rotary=kc.Rotary(128, 500))
    refuses(-1, kc.KvCache, sc.pools[0], sc.pools[1].half())
    refuses(-1, kc.KvCache, sc.pools[0].float(), sc.pools[1].float())
    refuses(-1, kc.KvCache, sc.pools[0][0], sc.pools[1][0])
    flat = torch.zeros(sc.n_pages, 2, 16, 68, dtype=torch.bfloat16, device=DEV)[..., :64]
    refuses(-3, kc.KvCache(flat, flat.clone(memory_format=torch.preserve_format)).attention, b, sc.q)
    one = torch.zeros(1, 2, 16, 64, dtype=torch.bfloat16, device=DEV).expand(sc.n_pages, 2, 16, 64)
    refuses(-1, kc.KvCache(one, one).append, b, k, v)                                        # all pages are the same memory
    refuses(-1, b.set, [T[0], [10 ** 6] * 3], L, Q, P, 64)
    refuses(-1, b.set, [T[0], [-1] * 3], L, Q, P, 64)
    refuses(-1, sc.cache.attention, b, sc.q)                                                 # a batch whose setting failed is empty
    refuses(-1, b.set, T, [40, -1], Q, P, 64)
    refuses(-1, b.set, T, L, [3, -2], P, 64)
    refuses(-1, b.set, T, [40, 500], Q, P, 64)                                               # more keys than pages
    refuses(-1, b.set, T, L, Q, P, 65)
    refuses(-1, b.set, T, L, Q, [10 ** 6] * 4, 64)
    refuses(-1, b.set, T, L, Q, P, -1)
    refuses(-1, b.set, T, L, Q[:1], P, 64)
    b.set(T, [2, 30], Q, P, 64)                                                              # fewer keys than queries: may attend, not append
    assert sc.cache.attention(b, sc.q).shape == (5, 256)
    refuses(-1, sc.cache.append, b, k, v)
    b.set([T[0], T[0]], [40, 40], Q, P, 64)                                                  # the same pages twice: may attend, not append
    assert sc.cache.attention(b, sc.q).shape == (5, 256)
    refuses(-1, sc.cache.append, b, k, v)
    b.set([T[0], P], [40, 64], Q, P, 64)                                                     # a page of the prefix
    refuses(-1, sc.cache.append, b, k, v)
    with pytest.raises(hb.HttmError):
        b.set(T, L, [[1], [2]], P, 64)
    b.close()
    refuses(-1, sc.cache.attention, b, sc.q)


STEPS = {
    "more jobs than a CTA reads at once": ([1 + i % 3 for i in range(700)], [1] * 700, 0, 32, 8, 128, 16, {}),
    "two kernels, few parts to a row": ([1 + i % 70 for i in range(300)], [1] * 300, 130, 32, 8, 128, 16, {}),
    "two kernels, one row to a task, fp16": ([1 + i % 40 for i in range(300)], [1] * 300, 100, 16, 16, 64, 64, dict(dtype=torch.float16)),
    "two kernels, tiles of 16, 32 and 64 rows": ([20 + 7 * i for i in range(64)], [(1, 8, 16, 4)[i % 4] for i in range(64)], 5000, 32, 8, 128, 32, {}),
    "two kernels, one row tile, long prefix": ([1 + i for i in range(32)], [1] * 32, 9000, 16, 4, 64, 64, {}),
    "much for the wide kernel, tokens beside it": ([300 + i for i in range(30)] + [40] * 20, [300] * 30 + [2] * 20, 2000, 32, 8, 128, 64, {}),
}


@pytest.mark.parametrize("name", STEPS)
def test_steps_of_many_sequences(name):
    """Both kernels side by side and one behind the other; jobs of different heights one after the other in a CTA; every way to add parts up."""
    *a, kw = STEPS[name]
    sc = Scene(*a, **kw, seed=len(name))
    for _ in range(3):   # (the same workspace again, nothing waited for)
        out = torch.full((sum(sc.queries), sc.heads * sc.dim), float("nan"), dtype=sc.dtype, device=DEV)
        sc.cache.attention(sc.batch, sc.q, out)
    first = sc.cache.attention(sc.batch, sc.q)
    assert sc.batch.status() == 0
    assert torch.equal(first, out)
    sc.check(out, what=name)


def test_a_batch_is_not_set_while_its_stream_is_captured():
    sc = Scene([40, 30], [3, 2], 64, 4, 2, 64, 16, seed=1)
    fresh = kc.CacheBatch(4, 2, 64, 16, sc.n_pages)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for batch in (sc.batch, fresh):
            with pytest.raises(hb.HttmError) as e:
                batch.set(sc.tables, sc.lengths, sc.queries, sc.prefix_pages, 64)
            assert e.value.code == -2
        doubled = sc.q * 2   # (the capture goes on)
    graph.replay()
    assert torch.equal(doubled, sc.q * 2)
    for batch in (sc.batch, fresh):
        batch.set(sc.tables, sc.lengths, sc.queries, sc.prefix_pages, 64)
        sc.check(sc.cache.attention(batch, sc.q))
