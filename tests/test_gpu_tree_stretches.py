"""Tree attention over batches that give every workgroup several tiles of 128 keys: sums and
maxima carried from tile to tile, stretches that end one row block and begin the next, row
blocks whose parts several workgroups leave.  Up to 512 workgroups share the tiles evenly."""

import numpy as np
import pytest

from tests.test_gpu_attention import check, run_tree, tree_reference

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

GROUPS = 512


def units(heads, lengths, counts, f32, most):
    """(sequence, kv head, row block, 128 keys) of a call."""
    Hq, Hkv, D = heads
    G = Hq // Hkv
    block = (16 if G * most <= 16 else 32) if f32 else 16 if G * most <= 16 else 256 if D == 64 else 128
    return sum(Hkv * -(-t * G // block) * -(-(n + t) // 128) for n, t in zip(lengths, counts) if t)


def run(dtype, heads, lengths, counts, per_group, **kw):
    most = max(counts)
    assert units(heads, lengths, counts, dtype == "f32", most) >= per_group * GROUPS
    return run_tree(dtype, heads, kw.pop("P", 32), lengths, counts, max_nodes=most, **kw)


def ragged(seed, n, lo, hi, few, many):
    r = np.random.default_rng(seed)
    return r.integers(lo, hi, n).tolist(), r.integers(few, many + 1, n).tolist()


# At most 16 rows (bf16, fp32), then more (bf16 D = 64 and 128, fp32): 4 to 8 tiles a workgroup.
CASES = [("bf16", (8, 8, 128), 1, 1), ("bf16", (8, 8, 64), 1, 5), ("bf16", (16, 8, 128), 3, 8), ("f32", (8, 8, 128), 1, 2), ("f32", (8, 8, 64), 1, 9),
         ("bf16", (16, 8, 128), 3, 20), ("bf16", (16, 8, 64), 4, 20), ("f32", (16, 8, 64), 1, 20), ("f32", (16, 8, 128), 1, 14)]


@pytest.mark.parametrize("dtype,heads,few,many", CASES)
def test_several_tiles_a_workgroup(dtype, heads, few, many):
    lengths, counts = ragged(1, 30, 900, 2100, few, many)
    run(dtype, heads, lengths, counts, 4, seed=31)


@pytest.mark.parametrize("dtype,heads,few,many", CASES)
def test_long_and_short_sequences_together(dtype, heads, few, many):
    """Stretches that hold whole short sequences between the end of one long one and the start of the next."""
    lengths, counts = ragged(2, 60, 0, 300, few, many)
    lengths[7], lengths[8], lengths[30], lengths[59] = 9100, 4097, 8191, 7000
    counts[3] = counts[40] = 0
    run(dtype, heads, lengths, counts, 1, seed=32, poison=True)


BF16_CASES = [c for c in CASES if c[0] == "bf16"]
F32_CASES = [c for c in CASES if c[0] == "f32"]


@pytest.mark.parametrize("dtype,heads,few,many", BF16_CASES)
def test_large_scores_over_several_tiles(dtype, heads, few, many):
    lengths, counts = ragged(3, 24, 1100, 2400, few, many)
    run(dtype, heads, lengths, counts, 4, seed=33, qscale=40.0, scale=0.5)


def rising(cache, lengths):
    """Coordinate 0 of the cached keys rises by 1 every 64 tokens."""
    P = cache.page_size
    for s, n in enumerate(lengths):
        for j in range(-(-n // P)):
            cache.k[0, int(cache.table[s, j]), :, :, 0] = (torch.arange(j * P, j * P + P, device="cuda") // 64).to(cache.dtype)


@pytest.mark.parametrize("dtype,heads,few,many", BF16_CASES)
def test_rising_maxima_over_several_tiles(dtype, heads, few, many):
    """Each tile outweighs all before it by far, so every step moves the maximum and rescales the sums."""
    lengths, counts = ragged(4, 24, 1100, 2400, few, many)
    cache, att, args, _, _ = run(dtype, heads, lengths, counts, 4, seed=34)
    layer, q, seqs, off, par = args
    rising(cache, lengths)
    q[:, :, 0] = 30.0
    want = tree_reference(cache, 0, q, lengths, counts, par.tolist(), heads[2] ** -0.5)
    check(att(*args), want, dtype)


@pytest.mark.parametrize("dtype,heads,few,many", F32_CASES)
def test_rising_maxima_of_exact_scores(dtype, heads, few, many):
    """The same in fp32, with scores that are whole numbers: those of hundreds would carry errors of 2^-24 of
    themselves, and the weights the same relative ones, past the tolerance."""
    lengths, counts = ragged(4, 24, 1100, 2400, few, many)
    cache, att, args, _, _ = run(dtype, heads, lengths, counts, 4, seed=34, scale=0.125)
    layer, q, seqs, off, par = args
    cache.k.zero_()
    rising(cache, lengths)
    q[:, :, 0] = 64.0
    want = tree_reference(cache, 0, q, lengths, counts, par.tolist(), 0.125)
    check(att(*args), want, dtype)


def test_one_long_sequence_of_many_tiles_a_workgroup():
    run("bf16", (8, 8, 128), [70000], [1], 8, seed=35, P=256)
    run("bf16", (4, 1, 64), [140000], [5], 2, seed=36, P=64)
    run("f32", (4, 1, 64), [140000], [4], 2, seed=37, P=64)


@pytest.mark.parametrize("dtype,heads,T", [("bf16", (2, 1, 64), 3), ("bf16", (32, 1, 64), 3), ("f32", (2, 1, 64), 3)])
def test_a_length_of_no_sense_among_others(dtype, heads, T):
    """A table whose rows could hold 2^31 - 16 tokens, and a length word that says so: its own rows get something,
    the other sequences' what they should."""
    import paper_2608_15018_amd as s2
    from tests.test_gpu_attention import DT, ints

    Hq, Hkv, D = heads
    g = torch.Generator(device="cuda").manual_seed(41)
    cache = s2.KVCache(1, Hkv, D, 64, 16, 3, (1 << 27) - 1, dtype=DT[dtype])
    cache.k.normal_(generator=g), cache.v.normal_(generator=g)
    lengths = [150, 0, 333]
    cache.reserve(ints([0, 2]), ints([150 + T, 333 + T]))
    cache.length.copy_(ints(lengths))
    q = torch.randn((3 * T, Hq, D), generator=g, device="cuda").to(DT[dtype])
    par = [-1, 0, 1] * 3
    att = s2.TreeAttention(cache, Hq, 3, T)
    sane = att(0, q[:2 * T], ints([0, 2]), ints([0, T, 2 * T]), ints(par[:2 * T]))
    for wrong in (2**31 - 1, 2**31 - 17, 2**31 - 16 - T):
        cache.length[1] = wrong
        got = att(0, torch.cat([q[:T], q[2 * T:], q[T:2 * T]]), ints([0, 1, 2]), ints([0, T, 2 * T, 3 * T]), ints(par))
        torch.cuda.synchronize()
        for a, b in ((got[:T], sane[:T]), (got[2 * T:], sane[T:])):
            check(a, b.double().cpu().numpy(), dtype)
