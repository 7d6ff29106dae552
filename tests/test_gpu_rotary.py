"""Norms and rotation of queries and keys, and their gradients, against a plain implementation in 64 bits.  Needs a B200.

Tolerances.  An output is rounded once (half a step: 2^-8 of its size in bf16, whose significand has 8 bits, 2^-11 in fp16, and 2^-25 below fp16's normal range); the
arithmetic in front of that is 32-bit and a few dozen operations deep, 2^-19 of the sizes of its terms.  Sums over rows (dw, db) are
32-bit: at most 2^-24 times the number of additions a term goes through (bounded by the number of rows, and by 1024: longer sums are
spread over threads) of the sum of the terms' sizes, with the terms themselves good to 2^-19."""
import pytest
import torch

from paper_2511_21317_b200 import binding as hb
from paper_2511_21317_b200 import kv_cache as kc

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
STEP = {torch.bfloat16: (2.0 ** -8, 0.0), torch.float16: (2.0 ** -11, 2.0 ** -25)}


def pairs(dim, axes, rotated, interleaved):
    d = rotated // axes
    out = []
    for x in range(axes):
        for i in range(d // 2):
            out.append((x * d + 2 * i, x * d + 2 * i + 1, x, i) if interleaved else (x * d + i, x * d + i + d // 2, x, i))
    return out


def turn64(positions, dim, axes, rotated, interleaved, base):
    """[tokens][dim][dim] rotation matrices in 64 bits: y = R z."""
    n = positions.shape[0]
    r = torch.eye(dim, dtype=torch.float64, device=DEV).repeat(n, 1, 1)
    d = rotated // axes
    for a, b, x, i in pairs(dim, axes, rotated, interleaved):
        t = positions[:, x].double() * base ** (-2.0 * i / d)
        r[:, a, a] = t.cos()
        r[:, b, b] = t.cos()
        r[:, a, b] = -t.sin()
        r[:, b, a] = t.sin()
    return r


def norm64(x, norm, eps):
    x = x.double()
    if norm == "layer":
        x = x - x.mean(-1, keepdim=True)
    if norm == "none":
        return x, torch.ones_like(x[..., :1])
    r = 1.0 / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    return x * r, r


def forward64(x, w, b, turn, norm, eps):
    """y, and the size of the terms it is made of."""
    xh, r = norm64(x, norm, eps)
    z = xh * (w.double() if w is not None else 1.0) + (b.double() if b is not None else 0.0)
    size = (xh.abs() + (x.double().mean(-1, keepdim=True).abs() * r if norm == "layer" else 0.0)) * (w.double().abs() if w is not None else 1.0)
    size = size + (b.double().abs() if b is not None else 0.0)
    return torch.einsum("tij,htj->hti", turn, z), torch.einsum("tij,htj->hti", turn.abs(), size)


def tensors(heads, n, dim, dtype, layout, gen, scale=1.0, offset=0.0):
    """[heads][n][dim]: contiguous, a view of [n][3][heads][dim] with other things around it, or a view with padded rows."""
    t = torch.randn(heads, n, dim, generator=gen, device=DEV) * scale + offset
    t = t.to(dtype)
    if layout == "heads":
        return t.contiguous()
    if layout == "fused":
        whole = torch.full((n, 3, heads, dim), 7.0, dtype=dtype, device=DEV)
        whole[:, 1] = t.permute(1, 0, 2)
        return whole[:, 1].permute(1, 0, 2)
    whole = torch.full((heads, n, dim + 24), 7.0, dtype=dtype, device=DEV)
    whole[..., 8:8 + dim] = t
    return whole[..., 8:8 + dim]


def make(dim, norm, axes, rotated, interleaved, n, hq, hk, dtype, layout, seed, n_positions=40, offset=0.0, weights=True):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    q, k = (tensors(h, n, dim, dtype, layout, gen, s, offset) for h, s in ((hq, 1.5), (hk, 0.7)))
    pos = torch.randint(0, n_positions, (n, axes), generator=gen, device=DEV, dtype=torch.int32)
    if n > 2:
        pos[0] = 0
        pos[1] = n_positions - 1
    w = [(1.0 + 0.3 * torch.randn(dim, generator=gen, device=DEV)) if weights and norm != "none" else None for _ in range(2)]
    b = [(0.2 * torch.randn(dim, generator=gen, device=DEV)) if weights and norm == "layer" else None for _ in range(2)]
    rot = kc.Rotary(dim, n_positions, axes=axes, rotated_dim=rotated, base=100.0, interleaved=interleaved, norm=norm, eps=1e-6)
    return q, k, pos, w, b, rot


CASES = [  # dim, norm, axes, rotated, interleaved, tokens, q heads, k heads, type, layout
    (64, "layer", 2, 64, False, 1, 16, 16, torch.bfloat16, "fused"),
    (64, "layer", 2, 64, False, 133, 16, 16, torch.bfloat16, "fused"),
    (64, "layer", 2, 64, True, 77, 5, 1, torch.bfloat16, "padded"),
    (64, "rms", 1, 64, False, 61, 3, 3, torch.float16, "heads"),
    (128, "rms", 1, 128, False, 1, 32, 8, torch.bfloat16, "heads"),
    (128, "rms", 1, 64, True, 45, 12, 3, torch.float16, "padded"),
    (128, "layer", 2, 48, False, 19, 6, 2, torch.bfloat16, "heads"),
    (128, "none", 1, 128, False, 31, 4, 4, torch.bfloat16, "fused"),
    (32, "rms", 2, 32, False, 259, 2, 9, torch.bfloat16, "heads"),
    (32, "layer", 1, 8, False, 40, 1, 1, torch.float16, "heads"),
    (256, "rms", 1, 256, False, 23, 4, 1, torch.bfloat16, "fused"),
    (256, "layer", 1, 0, False, 9, 2, 2, torch.bfloat16, "heads"),
    (64, "rms", 1, 64, False, 5000, 2, 1, torch.bfloat16, "heads"),
]


def check_forward(got, x, w, b, turn, norm, eps, what):
    step, tiny = STEP[got.dtype]
    y, size = forward64(x, w, b, turn, norm, eps)
    bad = (got.double() - y).abs() - (step * y.abs() + tiny + 2.0 ** -19 * size)
    assert (bad <= 0).all(), f"{what}: off by {(got.double() - y).abs().max():.3e}, over the bound by {bad.max():.3e}"


@pytest.mark.parametrize("case", CASES)
def test_forward(case):
    dim, norm, axes, rotated, inter, n, hq, hk, dtype, layout = case
    q, k, pos, w, b, rot = make(*case[:5], n, hq, hk, dtype, layout, seed=n + dim)
    turn = turn64(pos, dim, axes, rotated, inter, 100.0) if rotated else torch.eye(dim, dtype=torch.float64, device=DEV).repeat(n, 1, 1)
    yq, yk = rot.norm_rotate(q, k, pos, w[0], w[1], b[0], b[1])
    assert rot.status() == 0
    check_forward(yq, q, w[0], b[0], turn, norm, 1e-6, "q")
    check_forward(yk, k, w[1], b[1], turn, norm, 1e-6, "k")
    # one tensor alone, without weights, and in place
    alone, none = rot.norm_rotate(None, k, pos)[1], rot.norm_rotate(q, None, pos, w[0], None, b[0])
    assert none[1] is None and torch.equal(none[0], yq)
    check_forward(alone, k, None, None, turn, norm, 1e-6, "k alone")
    back = k.clone(memory_format=torch.preserve_format)
    around = k._base.clone() if k._base is not None else None
    rot.norm_rotate(None, k, pos, None, w[1], None, b[1], out_k=k)
    assert torch.equal(k, yk)
    if around is not None:   # what lies around the rows stays as it was
        k.copy_(back)
        assert torch.equal(k._base, around)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_rows_far_from_zero_constant_rows_and_large_values(dtype):
    q, k, pos, w, b, rot = make(64, "layer", 2, 64, False, 50, 3, 2, dtype, "heads", seed=5, offset=30.0)
    k[0, :7] = 12.5          # a row of equal values: its norm is 0 / sqrt(eps)
    k[1, :7] = 0.0
    q[0, :7] = 3.0e4 * torch.sign(q[0, :7] - 30.0)
    turn = turn64(pos, 64, 2, 64, False, 100.0)
    yq, yk = rot.norm_rotate(q, k, pos, w[0], w[1], b[0], b[1])
    check_forward(yq, q, w[0], b[0], turn, "layer", 1e-6, "q")
    check_forward(yk, k, w[1], b[1], turn, "layer", 1e-6, "k")


def test_large_positions_keep_their_digits():
    """Positions of a long sequence: the table's angles are computed in 64 bits."""
    gen = torch.Generator(device=DEV).manual_seed(1)
    k = tensors(2, 64, 64, torch.bfloat16, "heads", gen)
    rot = kc.Rotary(64, 200000, base=10000.0, norm="rms", eps=1e-6)
    pos = torch.randint(199000, 200000, (64, 1), generator=gen, device=DEV, dtype=torch.int32)
    y = rot.norm_rotate(None, k, pos.view(64))[1]
    check_forward(y, k, None, None, turn64(pos, 64, 1, 64, False, 10000.0), "rms", 1e-6, "k")


def test_own_frequencies():
    gen = torch.Generator(device=DEV).manual_seed(2)
    k = tensors(2, 33, 32, torch.bfloat16, "heads", gen)
    f = [7.0 ** (-2.0 * i / 32) for i in range(16)]
    rot = kc.Rotary(32, 50, frequencies=f, norm="rms", eps=1e-6)
    pos = torch.arange(33, device=DEV, dtype=torch.int32).view(33, 1)
    check_forward(rot.norm_rotate(None, k, pos)[1], k, None, None, turn64(pos, 32, 1, 32, False, 7.0), "rms", 1e-6, "k")


def test_a_row_that_is_not_a_number_stays_alone():
    q, k, pos, w, b, rot = make(64, "layer", 2, 64, False, 40, 3, 2, torch.bfloat16, "heads", seed=6)
    ref = rot.norm_rotate(q, k, pos, w[0], w[1], b[0], b[1])
    q2 = q.clone()
    q2[1, 7] = float("inf")
    q2[2, 9, 3] = float("nan")
    got = rot.norm_rotate(q2, k, pos, w[0], w[1], b[0], b[1])
    assert got[0][1, 7].isnan().all() and got[0][2, 9].isnan().all()
    same = torch.ones(3, 40, dtype=torch.bool, device=DEV)
    same[1, 7] = same[2, 9] = False
    assert torch.equal(got[0][same], ref[0][same]) and torch.equal(got[1], ref[1])


def test_a_position_outside_the_table_is_reported_and_its_rows_are_not_numbers():
    q, k, pos, w, b, rot = make(64, "rms", 1, 32, False, 30, 3, 2, torch.bfloat16, "heads", seed=7)
    ref = rot.norm_rotate(q, k, pos, w[0], w[1])
    assert rot.status() == 0
    pos2 = pos.clone()
    pos2[4], pos2[5] = 40, -1
    got = rot.norm_rotate(q, k, pos2, w[0], w[1])
    torch.cuda.synchronize()
    for r, g in zip(ref, got):
        assert g[:, 4:6, :32].isnan().all() and torch.equal(g[:, 4:6, 32:], r[:, 4:6, 32:])
        assert torch.equal(g[:, :4], r[:, :4]) and torch.equal(g[:, 6:], r[:, 6:])
    with pytest.raises(hb.HttmError):
        rot.status()


def grad64(x, dy, w, turn, norm, eps):
    xh, r = norm64(x, norm, eps)
    g = torch.einsum("tji,htj->hti", turn, dy.double())
    u = g * (w.double() if w is not None else 1.0)
    if norm == "none":
        return u, torch.zeros_like(u), g, xh
    mean = u.mean(-1, keepdim=True) if norm == "layer" else torch.zeros_like(u[..., :1])
    dx = r * (u - mean - xh * (u * xh).mean(-1, keepdim=True))
    ga = torch.einsum("tji,htj->hti", turn.abs(), dy.double().abs()) * (w.double().abs() if w is not None else 1.0)
    size = r * (ga + ga.mean(-1, keepdim=True) + xh.abs() * (ga * xh.abs()).mean(-1, keepdim=True))
    return dx, size, g, xh


def check_grad(dx, dw, db, x, dy, w, turn, norm, eps, what):
    step, tiny = STEP[dx.dtype]
    want, size, g, xh = grad64(x, dy, w, turn, norm, eps)
    bad = (dx.double() - want).abs() - (step * want.abs() + tiny + 2.0 ** -18 * size)
    assert (bad <= 0).all(), f"{what}: dx off by {(dx.double() - want).abs().max():.3e}, over the bound by {bad.max():.3e}"
    ga = torch.einsum("tji,htj->hti", turn.abs(), dy.double().abs())
    depth = min(x.shape[0] * x.shape[1] + 16, 1024) * 2.0 ** -24 + 2.0 ** -19
    for got, terms, sizes, name in ((dw, g * xh, ga * xh.abs(), "dw"), (db, g, ga, "db")):
        if got is not None:
            bad = (got.double() - terms.sum((0, 1))).abs() - depth * sizes.sum((0, 1)) - 1e-30
            assert (bad <= 0).all(), f"{what}: {name} over the bound by {bad.max():.3e}"


@pytest.mark.parametrize("case", CASES)
def test_backward(case):
    dim, norm, axes, rotated, inter, n, hq, hk, dtype, layout = case
    q, k, pos, w, b, rot = make(*case[:5], n, hq, hk, dtype, layout, seed=n + dim + 1)
    gen = torch.Generator(device=DEV).manual_seed(n)
    dq, dk = tensors(hq, n, dim, dtype, layout, gen, 0.3), tensors(hk, n, dim, dtype, "heads", gen, 0.3)
    turn = turn64(pos, dim, axes, rotated, inter, 100.0) if rotated else torch.eye(dim, dtype=torch.float64, device=DEV).repeat(n, 1, 1)
    got = rot.norm_rotate_backward(dq, dk, q, k, pos, w[0], w[1], b[0], b[1])
    assert rot.status() == 0
    check_grad(got[0], got[2], got[3], q, dq, w[0], turn, norm, 1e-6, "q")
    check_grad(got[1], got[4], got[5], k, dk, w[1], turn, norm, 1e-6, "k")
    assert (got[2] is None) == (w[0] is None) and (got[3] is None) == (b[0] is None)
    again = rot.norm_rotate_backward(dq, dk, q, k, pos, w[0], w[1], b[0], b[1])
    assert all(x is None and y is None or torch.equal(x, y) for x, y in zip(got, again))   # sums in a fixed order
    alone = rot.norm_rotate_backward(None, dk, None, k, pos, None, w[1], None, b[1], out_k=dk)   # in place, and one tensor alone
    assert alone[0] is None and torch.equal(dk, got[1]) and (w[1] is None or torch.equal(alone[4], got[4]))


def test_gradients_over_many_tokens():
    case = (64, "layer", 2, 64, False)
    q, k, pos, w, b, rot = make(*case, 6001, 8, 3, torch.bfloat16, "fused", seed=3)
    gen = torch.Generator(device=DEV).manual_seed(4)
    dq, dk = tensors(8, 6001, 64, torch.bfloat16, "heads", gen, 0.3, 0.1), tensors(3, 6001, 64, torch.bfloat16, "heads", gen, 0.3, 0.1)
    turn = turn64(pos, 64, 2, 64, False, 100.0)
    got = rot.norm_rotate_backward(dq, dk, q, k, pos, w[0], w[1], b[0], b[1])
    check_grad(got[0], got[2], got[3], q, dq, w[0], turn, "layer", 1e-6, "q")
    check_grad(got[1], got[4], got[5], k, dk, w[1], turn, "layer", 1e-6, "k")


def test_no_tokens():
    rot = kc.Rotary(64, 8, norm="layer")
    w, b = torch.ones(64, device=DEV), torch.zeros(64, device=DEV)
    q, k = (torch.empty(h, 0, 64, dtype=torch.bfloat16, device=DEV) for h in (4, 2))
    pos = torch.empty(0, 1, dtype=torch.int32, device=DEV)
    assert [t.shape for t in rot.norm_rotate(q, k, pos, w, w, b, b)] == [(4, 0, 64), (2, 0, 64)]
    got = rot.norm_rotate_backward(q, k, q, k, pos, w, w, b, b)
    assert all((t == 0).all() for t in got[2:])   # sums over nothing


@pytest.mark.parametrize("norm,axes", [("layer", 2), ("rms", 1)])
def test_gradient_against_differences(norm, axes):
    """d/dx of sum(dy . y) by central differences of the 64-bit formula, and through autograd with a broadcast gradient.  The differences are good to
    1e-6 of the derivative's scale (steps of 1e-4 of inputs of order 1: the third derivative's term is 1e-8, rounding 1e-12 / 1e-4); dx is rounded to fp16."""
    n, h, dim = 6, 2, 32
    gen = torch.Generator(device=DEV).manual_seed(11)
    x = tensors(h, n, dim, torch.float16, "heads", gen)
    dy = tensors(h, n, dim, torch.float16, "heads", gen)
    w = 1.0 + 0.3 * torch.randn(dim, generator=gen, device=DEV)
    b = 0.1 * torch.randn(dim, generator=gen, device=DEV)
    b = b if norm == "layer" else None
    pos = torch.randint(0, 20, (n, axes), generator=gen, device=DEV, dtype=torch.int32)
    rot = kc.Rotary(dim, 20, axes=axes, base=100.0, norm=norm, eps=1e-6)
    turn = turn64(pos, dim, axes, dim, False, 100.0)

    def f(x64, w64, b64):
        return (forward64(x64, w64, b64, turn, norm, 1e-6)[0] * dy.double()).sum((0, 1, 2))

    got = rot.norm_rotate_backward(dy, None, x, None, pos, w, None, b, None)
    eps = 1e-4
    for i, j, c in ((0, 0, 0), (1, 5, 31), (0, 3, 17), (1, 2, 8)):
        up, down = x.double().clone(), x.double().clone()
        up[i, j, c] += eps
        down[i, j, c] -= eps
        want = (f(up, w, b) - f(down, w, b)) / (2 * eps)
        scale = grad64(x, dy, w, turn, norm, 1e-6)[1][i, j, c]
        assert abs(got[0][i, j, c].double() - want) <= 2.0 ** -11 * abs(want) + 2.0 ** -25 + (2.0 ** -18 + 1e-6) * scale
    for c in (0, 13, 31):
        up, down = w.double().clone(), w.double().clone()
        up[c] += eps
        down[c] -= eps
        want = (f(x, up, b) - f(x, down, b)) / (2 * eps)
        assert abs(got[2][c].double() - want) <= 1e-5 * (1.0 + abs(want))
    # through autograd, with a gradient that is broadcast over heads and channels
    xq, xk = x.clone().requires_grad_(True), x.clone().requires_grad_(True)
    wg = w.clone().requires_grad_(True)
    yq, yk = rot.differentiable(xq, xk, pos, wg, wg, b, b)
    (yq.sum() + (yk * dy).sum()).backward()
    one = rot.norm_rotate_backward(torch.ones_like(dy), dy, x, x, pos, w, w, b, b)
    assert torch.equal(xq.grad, one[0]) and torch.equal(xk.grad, one[1]) and torch.allclose(wg.grad, one[2] + one[4], rtol=1e-6)


def test_another_stream():
    q, k, pos, w, b, rot = make(64, "layer", 2, 64, False, 3000, 8, 8, torch.bfloat16, "heads", seed=8)
    ref = rot.norm_rotate(q, k, pos, w[0], w[1], b[0], b[1])
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    outs = [torch.empty_like(t) for t in (q, k)]
    s.wait_stream(torch.cuda.current_stream())
    rot.norm_rotate(q, k, pos, w[0], w[1], b[0], b[1], out_q=outs[0], out_k=outs[1], stream=s)
    s.synchronize()
    assert torch.equal(outs[0], ref[0]) and torch.equal(outs[1], ref[1])


def test_refusals():
    q, k, pos, w, b, rot = make(64, "layer", 2, 64, False, 20, 4, 4, torch.bfloat16, "heads", seed=9)

    def refuses(code, *a, **kw):
        with pytest.raises(hb.HttmError) as e:
            rot.norm_rotate(*a, **kw)
        assert e.value.code == code, str(e.value)

    refuses(-1, None, None, pos)
    refuses(-1, q.float(), k.float(), pos)
    refuses(-1, q, k.half(), pos)
    refuses(-1, q, k[:, :19], pos)
    refuses(-1, q, k, pos[:19].contiguous())
    refuses(-1, q, k, pos.long())
    refuses(-1, q, k, None)
    refuses(-1, q.cpu(), None, pos)
    refuses(-1, q.transpose(1, 2), None, pos)
    refuses(-1, q, k, pos, w[0].bfloat16())
    refuses(-1, q, k, pos, w[0][:32])
    refuses(-1, q[0], None, pos)
    flat = torch.empty(4 * 20 * 64 + 64, dtype=torch.bfloat16, device=DEV)
    refuses(-3, flat[4:4 + 4 * 20 * 64].view(4, 20, 64), None, pos)                       # not 16-byte aligned
    refuses(-3, torch.empty(4, 20, 68, dtype=torch.bfloat16, device=DEV)[..., :64], None, pos)   # rows of 136 bytes
    base = torch.zeros(4 * 20 * 64 + 4096, dtype=torch.bfloat16, device=DEV)
    x, y = base[:5120].view(4, 20, 64), base[1024:6144].view(4, 20, 64)
    refuses(-1, x, None, pos, out_q=y)                                                     # the output overlaps the input
    refuses(-1, q, None, pos, out_q=torch.empty(1, 20, 64, dtype=torch.bfloat16, device=DEV).expand(4, 20, 64))   # a row written four times
    one = q[:1].expand(4, 20, 64)                                                          # a broadcast input is fine
    assert torch.equal(rot.norm_rotate(one, None, pos)[0][3], rot.norm_rotate(q, None, pos)[0][0])
    none = kc.Rotary(64, 40, axes=2, norm="none")
    with pytest.raises(hb.HttmError):
        none.norm_rotate(q, k, pos, w[0])
    rot.close()
    refuses(-1, q, k, pos)


def test_refusals_of_the_gradients():
    q, k, pos, w, b, rot = make(64, "layer", 2, 64, False, 20, 4, 4, torch.bfloat16, "heads", seed=9)

    def refuses(code, *a, **kw):
        with pytest.raises(hb.HttmError) as e:
            rot.norm_rotate_backward(*a, **kw)
        assert e.value.code == code, str(e.value)

    refuses(-1, None, None, None, None, pos)
    refuses(-1, None, k, q, k, pos)                                # no gradient of q's output
    refuses(-1, q.float(), None, q, None, pos)
    refuses(-1, q[:, :19], None, q, None, pos)
    refuses(-1, q, None, q, None, None)
    refuses(-1, q, None, q, None, pos, w[0].double())
    refuses(-1, q, None, q, None, pos, out_q=torch.empty(4, 20, 65, dtype=torch.bfloat16, device=DEV)[..., :63])
    refuses(-1, "q", None, q, None, pos)
    base = torch.zeros(4 * 20 * 64 + 4096, dtype=torch.bfloat16, device=DEV)
    refuses(-1, base[:5120].view(4, 20, 64), None, q, None, pos, out_q=base[1024:6144].view(4, 20, 64))
    assert rot.norm_rotate_backward(q, None, q, None, pos)[1:] == (None,) * 5
    with pytest.raises(TypeError):
        rot.norm_rotate_backward(q)


def test_outputs_made_on_another_stream_are_its_own():
    """New tensors of a call with a stream of its own get no memory that the current stream has still to write to."""
    n, heads, dim = 300, 8, 64
    rotary = kc.Rotary(dim, 1024, norm="rms")
    q = torch.randn(heads, n, dim, device=DEV).to(torch.bfloat16)
    positions = torch.arange(n, dtype=torch.int32, device=DEV)
    want, _ = rotary.norm_rotate(q, None, positions)
    other = torch.cuda.Stream()
    held = [torch.empty_like(q).fill_(1.0) for _ in range(12)]   # blocks of the size that the call will ask for
    torch.cuda._sleep(1)   # (what is used below is loaded)
    torch.cuda.synchronize()
    torch.cuda._sleep(100_000_000)
    for i in range(1, 11):
        held[i].fill_(7.0)
    del held[2:10:2]   # (each between two that stay: free blocks of just that size)
    got, _ = rotary.norm_rotate(q, None, positions, stream=other)
    torch.cuda.synchronize()
    assert torch.equal(got, want)
