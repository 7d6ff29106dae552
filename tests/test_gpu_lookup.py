"""A scene that is kept and images that are looked up in it: the operators together, as run_lookup uses them.  Needs a B200."""
import pytest
import torch

from paper_2511_21317_b200 import binding as hb
from paper_2511_21317_b200 import kv_cache as kc
from paper_2511_21317_b200 import run_lookup, synth

pytestmark = pytest.mark.gpu


def rotate64(st, x, weight, bias, positions):
    """Layer norm of the heads and rotation by (row, column), in 64 bits: x [heads][tokens][64]."""
    x = x.double()
    x = x - x.mean(-1, keepdim=True)
    z = x / torch.sqrt(x.square().mean(-1, keepdim=True) + 1e-5) * weight.double() + bias.double()
    out = torch.empty_like(z)
    f = 100.0 ** (-2.0 * torch.arange(16, dtype=torch.float64, device=x.device) / 32)
    for axis in range(2):
        t = positions[:, axis].double()[:, None] * f
        a, b = z[..., 32 * axis:32 * axis + 16], z[..., 32 * axis + 16:32 * axis + 32]
        out[..., 32 * axis:32 * axis + 16] = a * t.cos() - b * t.sin()
        out[..., 32 * axis + 16:32 * axis + 32] = a * t.sin() + b * t.cos()
    return out


@pytest.mark.parametrize("page", [16, 128])
def test_images_see_the_scene_and_themselves(page):
    wl = synth.WORKLOADS["tiny"]
    st = run_lookup.Lookup(wl, layers=2, images=3, page_size=page)
    st.encode()
    y = st.lookup()
    torch.cuda.synchronize()
    assert st.ctx.query(hb.Q_DEVICE_STATUS) == 0 and st.rotary.status() == 0 and st.image_batch.status() == 0
    # the images' layers in 64 bits, on the scene's keys and values as the caches hold them.  Per layer q, k, v and the attention's output are
    # rounded to bf16 (2^-8 each), which moves scores of size up to 8 by 8 x 2 x 2^-8 = 2^-4 at worst and by a few hundredths as a rule; the
    # attention is a small part of x (weights of 0.02), so a hundredth of x's size is a wide bound on what is left.
    x = st.x_images.double()
    n, per = wl.n_tokens, wl.tokens_per_frame
    for layer in range(2):
        h = (x.float() * torch.rsqrt(x.float().pow(2).mean(-1, keepdim=True) + 1e-6)).double()
        q, k, v = (h @ st.w_qkv[layer].double().T).view(-1, 3, 16, 64).permute(1, 2, 0, 3)
        w = st.norms[layer]
        q, k = (rotate64(st, t, w[s + "_weight"], w[s + "_bias"], st.pos_images) for t, s in ((q, "q"), (k, "k")))
        pages = -(-n // page)
        ks, vs = (p[:pages].permute(1, 0, 2, 3).reshape(16, pages * page, 64)[:, :n].double() for p in (st.caches[layer].k_pages, st.caches[layer].v_pages))
        out = []
        for i in range(3):
            at = slice(i * per, (i + 1) * per)
            p = torch.softmax(q[:, at] @ torch.cat([ks, k[:, at]], 1).transpose(1, 2) / 8, -1)
            out.append(p @ torch.cat([vs, v[:, at]], 1))
        x = x + torch.cat(out, 1).permute(1, 0, 2).reshape(3 * per, 1024) @ st.w_o[layer].double().T
    err = (y.double() - x).abs().max().item() / x.square().mean().sqrt().item()
    assert err <= 1e-2 * 4, err   # (the largest of 800 000 elements; x itself is held in bf16 and is up to 4 times its mean size)
    st.close()


def test_without_a_scene_an_image_attends_to_itself_as_a_dense_layer_does():
    """Attention over the cache of one sequence and no prefix is dense attention over its tokens."""
    wl = synth.Workload("one", 1, 11, 13, 1, 4, 4, 0.5, 0.5, heads=4, seed=3)
    q, k, v = (hb.bf16_from_bits(t, "cuda:0") for t in synth.make_qkv(wl))
    n = wl.n_tokens
    with hb.Httm(hb.HttmConfig.of(wl)) as ctx:
        dense = ctx.dense_attention(q, k, v).float()
    pools = [torch.full((-(-n // 16), 4, 16, 64), float("nan"), dtype=torch.bfloat16, device="cuda:0") for _ in range(2)]
    cache = kc.KvCache(*pools)
    batch = kc.CacheBatch(4, 4, 64, 16, len(pools[0]), causal=False).set([list(range(len(pools[0])))], [n], [n])
    cache.append(batch, k, v)
    out = cache.attention(batch, q).float()
    # both round the weights and the output to bf16, each by 2^-8 of the size of what is summed
    bound = 2.0 ** -7 * (dense.abs() + torch.softmax(q.float() @ k.float().transpose(1, 2) / 8, -1).matmul(v.float().abs()).permute(1, 0, 2).reshape(n, 256))
    assert ((out - dense).abs() <= bound).all()


def test_the_command_runs(capsys, monkeypatch):
    monkeypatch.setattr("sys.argv", ["run_lookup", "--workload", "tiny", "--layers", "2", "--images", "2", "--steps", "1"])
    assert run_lookup.main() == 0
    assert '"finite": true' in capsys.readouterr().out
