"""The whole step: drafted trees verified over prompts in the cache, the accepted path
kept, and again; the outputs are those of the accepted tokens run as one prompt."""

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from paper_2608_15018_amd import verify_step  # noqa: E402


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def test_accepted_tokens_are_those_of_one_prompt():
    torch.manual_seed(0)
    hidden, prompts, nodes = 256, [37, 5, 70], 9
    kw = dict(layers=3, hidden=hidden, ffn=256, n_experts=8, top_k=2, n_heads=8, n_kv_heads=2,
              head_dim=64, seqs=3, nodes=nodes, max_tokens=200, page_size=16)
    m, ref = verify_step.VerifyStack(**kw), verify_step.VerifyStack(**kw)
    g = torch.Generator().manual_seed(3)
    ids = ints([0, 1, 2])
    xs = [[torch.randn((n, hidden), device="cuda")] for n in prompts]
    off = ints([0, 37, 42, 112])
    y = m.prefill(torch.cat([x[0] for x in xs]), ids, off)
    ys = [[y[a:b]] for a, b in ((0, 37), (37, 42), (42, 112))]
    for _ in range(3):
        parent, path, accept = verify_step.draw_trees(3, nodes, g)
        x = torch.randn((3 * nodes, hidden), device="cuda")
        y = m.verify(x, ids, ints([0, 9, 18, 27]), parent.cuda())
        m.commit(ids, path.cuda(), accept.cuda())
        assert not m.cache.status[:3].any()
        for s in range(3):
            at = path[s][:accept[s]].long().cuda() + s * nodes
            xs[s].append(x[at])
            ys[s].append(y[at])
    xs, ys = [torch.cat(x) for x in xs], [torch.cat(t) for t in ys]
    lens = [len(x) for x in xs]
    assert m.cache.length.tolist() == lens
    off = [0, lens[0], lens[0] + lens[1], sum(lens)]
    want = ref.prefill(torch.cat(xs), ids, ints(off))
    assert ref.cache.length.tolist() == lens
    got = torch.cat(ys)
    # Sums of different order in bf16 layers: each rounds at 2^-9 a few times, and later
    # layers carry that on.  A wrong mask, slot or position is of the order of 1.
    err = (got - want).norm(dim=1) / want.norm(dim=1)
    assert err.max() < 0.05 and err.mean() < 0.01, (err.max(), err.mean())
    # What the caches hold is the same too.
    for s in range(3):
        a = [m.cache.table[s, j // 16] for j in range(lens[s])]
        b = [ref.cache.table[s, j // 16] for j in range(lens[s])]
        ka = torch.stack([m.cache.k[2, a[j], :, j % 16] for j in range(lens[s])]).float()
        kb = torch.stack([ref.cache.k[2, b[j], :, j % 16] for j in range(lens[s])]).float()
        assert ((ka - kb).norm() / kb.norm()) < 0.02


def test_command_runs(capsys):
    verify_step.main(["--layers", "2", "--seqs", "3", "--nodes", "8", "--steps", "2", "--prompt", "100"])
    out = capsys.readouterr().out
    assert "prefill: 3 prompts" in out and "step 1: verified 24 drafted tokens" in out
