"""The whole step with the dense half in 8 bits and positions: norms, products, rotation,
attention and the MoE layer together, as a program uses them."""

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_2608_15018_amd as s2  # noqa: E402
from paper_2608_15018_amd import verify_step  # noqa: E402


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


KW = dict(layers=3, hidden=256, ffn=256, n_experts=8, top_k=2, n_heads=8, n_kv_heads=2, head_dim=64, seqs=3, nodes=9,
          max_tokens=200, page_size=16, dense="fp8")


def test_accepted_tokens_are_those_of_one_prompt():
    """Depths in a tree are positions in the prompt that its accepted path becomes."""
    torch.manual_seed(0)
    hidden, prompts, nodes = 256, [37, 5, 70], 9
    m, ref = verify_step.VerifyStack(**KW), verify_step.VerifyStack(**KW)
    g = torch.Generator().manual_seed(3)
    ids = ints([0, 1, 2])
    xs = [[torch.randn((n, hidden), device="cuda")] for n in prompts]
    x0 = torch.cat([x[0] for x in xs])
    given = x0.clone()
    y = m.prefill(x0, ids, ints([0, 37, 42, 112]))
    assert torch.equal(x0, given)  # the residual stream is the call's own
    ys = [[y[a:b]] for a, b in ((0, 37), (37, 42), (42, 112))]
    for _ in range(3):
        parent, path, accept = verify_step.draw_trees(3, nodes, g)
        x = torch.randn((3 * nodes, hidden), device="cuda")
        y = m.verify(x, ids, ints([0, 9, 18, 27]), parent.cuda())
        m.commit(ids, path.cuda(), accept.cuda())
        for s in range(3):
            at = path[s][:accept[s]].long().cuda() + s * nodes
            xs[s].append(x[at])
            ys[s].append(y[at])
    xs, ys = [torch.cat(x) for x in xs], [torch.cat(t) for t in ys]
    lens = [len(x) for x in xs]
    assert m.cache.length.tolist() == lens
    off = [0, lens[0], lens[0] + lens[1], sum(lens)]
    want = ref.prefill(torch.cat(xs), ids, ints(off))
    err = (torch.cat(ys) - want).norm(dim=1) / want.norm(dim=1)
    # A row's codes are off by at most 2^-4 of an element (rms 2^-5.8 or so) where a sum's last
    # bit falls the other way, which is rare; otherwise bf16 roundings of 2^-9 add up.  A wrong
    # position, slot or mask is of the order of 1.
    assert err.max() < 0.15 and err.mean() < 0.03, (err.max(), err.mean())


def test_a_layer_against_its_parts_in_32_bits():
    """One layer's first half, from the library's own 8-bit weights: norm, projection, rotation,
    attention, projection, with torch in 32 bits.  Three roundings to 8 bits on the way (2^-4 of
    an element at most, a third of that in the mean square) are those of the norm's rows and
    the attention's output, which the reference makes too."""
    torch.manual_seed(1)
    m = verify_step.VerifyStack(**dict(KW, layers=1))
    Hq, Hkv, D = m.heads
    x = torch.randn((50, 256), device="cuda")
    a = s2.add_norm(x, m.norm, out_dtype=s2.E4M3)
    spread = lambda r, k: r.codes.float() * r.scales.t().repeat_interleave(128, 1)[:, :k]  # noqa: E731
    full = lambda w: w.codes.float() * w.scales.repeat_interleave(128, 0)[:w.codes.shape[0]].repeat_interleave(128, 1)[:, :w.codes.shape[1]]  # noqa: E731
    qkv = (spread(a, 256) @ full(m.qkv[0]).t()).bfloat16().float().view(50, -1, D)
    q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
    angle = torch.arange(50, device="cuda").double()[:, None] * m.inv_freq.double()
    c, s = angle.cos().float()[:, None], angle.sin().float()[:, None]

    def turn(t):
        u, w = t[..., :D // 2], t[..., D // 2:]
        return torch.cat((u * c - w * s, w * c + u * s), -1).bfloat16().float()

    q, k = turn(q), turn(k).repeat_interleave(Hq // Hkv, 1)
    score = torch.einsum("ihd,jhd->hij", q.cpu(), k.cpu()) * D ** -0.5
    score.masked_fill_(torch.ones(50, 50).triu(1).bool(), float("-inf"))
    o = torch.einsum("hij,jhd->ihd", score.softmax(-1), v.cpu().repeat_interleave(Hq // Hkv, 1)).cuda().bfloat16()
    o8 = s2.quantize(o.reshape(50, -1).contiguous())
    want = x + (spread(o8, Hq * D) @ full(m.out[0]).t())
    m._moe = lambda l, h: torch.zeros((50, 256), device="cuda")
    got = m.prefill(x, ints([0]), ints([0, 50]))
    err = float((got - want).norm() / (want - x).norm())
    assert err < 2 ** -5, err


def test_command_runs(capsys):
    verify_step.main(["--layers", "2", "--seqs", "3", "--nodes", "8", "--steps", "2", "--prompt", "100", "--dense", "fp8"])
    out = capsys.readouterr().out
    assert "prefill: 3 prompts" in out and "step 1: verified 24 drafted tokens" in out


def test_the_default_is_as_before():
    with pytest.raises(ValueError):
        verify_step.VerifyStack(**dict(KW, dense="fp4"))
    m = verify_step.VerifyStack(**dict(KW, dense="bf16"))
    assert isinstance(m.qkv[0], torch.Tensor) and m.qkv[0].dtype == torch.bfloat16
