"""Attention of trees of drafts over the cache (score_tree) against the oracle, which takes every draft's path by itself.

Tolerance, elementwise, from the arithmetic: the output is rounded to bf16 (half a step, 2^-8 of the value), and the
softmax weights may be before the product with V (2^-8 of each, so 2^-8 of a = sum p |v| / sum p); scores, weights'
sums and products in fp32 are 1e-4 of a at most (128 terms of 2^-24 each in a score of up to 30).  The logarithm of
the sum: the same 1e-4, and 2^-22 of itself."""

import numpy as np
import pytest
import torch

import paper_2605_14037_amd as spkv
from paper_2605_14037_amd.inputs import to_numpy_f32
from tests.test_gpu_branch import Both

pytestmark = pytest.mark.gpu


def random_tree(rng, n, late=0.6):
    return [-1 if i == 0 or rng.random() < 0.05 else min(i - 1, int(i * rng.random() ** late)) for i in range(n)]


CHAIN = lambda rng, n: [i - 1 for i in range(n)]          # noqa: E731
STAR = lambda rng, n: [-1] * n                            # noqa: E731
BROOM = lambda rng, n: [i - 1 if i < n // 2 else n // 2 - 1 for i in range(n)]      # noqa: E731


class Trees(Both):
    def drafts(self, counts, shape=random_tree, seed=0):
        rng = np.random.default_rng(seed)
        self.counts = counts
        self.k, self.v, self.f = self.rows(sum(counts))
        self.q = torch.randn(sum(counts), self.shape[1], self.shape[3], generator=self.g, device="cuda").bfloat16()
        self.parents = torch.tensor([p for n in counts for p in shape(rng, n)], dtype=torch.int32, device="cuda")

    def score(self, logits=True, **kw):
        return self.cache.score_tree(self.k, self.v, self.q, self.parents, self.cu(self.counts),
                                     util_logits=self.f if logits else None, want_lse=True, **kw)

    def reference(self):
        """Outputs, logarithms of the sums, and the same mean of the values' sizes."""
        args = (to_numpy_f32(self.f), to_numpy_f32(self.q), self.parents.tolist(), self.counts)
        k, v = to_numpy_f32(self.k), to_numpy_f32(self.v)
        out, lse = self.oracle.score_tree(k, v, *args)
        kept = self.oracle._vbuf
        self.oracle._vbuf = [np.abs(x) for x in kept]
        size, _ = self.oracle.score_tree(k, np.abs(v), *args)
        self.oracle._vbuf = kept
        return out, lse, size

    def check_tree(self, got=None, rows=None, **kw):
        out, lse = self.score(**kw) if got is None else got
        ref, ref_lse, size = self.reference()
        out, lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
        pick = slice(None) if rows is None else rows
        err = np.abs(out - ref)[pick]
        bound = (2.0 ** -8 * (np.abs(ref) + size) + 1e-4 * size + 1e-30)[pick]
        assert np.isfinite(out[pick]).all()
        assert (err <= bound).all(), f"{int((err > bound).sum())} of {err.size} outside, worst {np.max(err / bound):.2f} of the bound"
        assert (np.abs(lse - ref_lse) <= 1e-4 + 2.0 ** -22 * np.abs(ref_lse))[pick].all(), np.abs(lse - ref_lse)[pick].max()


# sequences' lengths: none, below, at and above the window, below and above a half-page and a page
LENGTHS = [0, 1, 33, 127, 128, 129, 700]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq,hk,most", [(2, 2, 13), (8, 2, 4), (8, 2, 8), (12, 4, 17), (8, 2, 16), (8, 2, 31), (8, 2, 64), (8, 1, 64), (16, 1, 50),
                                        (3, 1, 64), (2, 2, 64)])
def test_trees_of_every_width(hq, hk, most, d):
    """Groups of 1 to 16 heads; 13 to 1024 columns, so every kernel, and blocks of columns that end inside one."""
    x = Trees(7, hq=hq, hk=hk, d=d, seed=most + d + hq, keep=0.5)
    x.append(LENGTHS)
    for counts in ([most, 1, max(1, most // 2), 0, most, 2, most - 1], [0, 0, 0, 0, 0, 0, most]):
        x.drafts(counts, seed=most)
        x.check_tree()


@pytest.mark.parametrize("window", [1, 2, 5, 16, 63, 64, 100])
@pytest.mark.parametrize("shape", [CHAIN, STAR, BROOM, random_tree], ids=["chain", "star", "broom", "random"])
def test_paths_and_windows(shape, window):
    """Paths longer than the window, whose early drafts are seen by their gates; the ring's end by the drafts' depths."""
    x = Trees(4, d=64, window=window, seed=window, keep=0.5)
    x.append([0, 20, window, 300])
    for counts in ([64, 40, 7, 64], [3, 1, 8, 8], [33, 32, 31, 1]):
        x.drafts(counts, shape, seed=window)
        x.check_tree()


@pytest.mark.parametrize("tau", [0.0, 0.3, 1.0])
@pytest.mark.parametrize("sinks", [0, 6])
def test_thresholds_and_sinks(tau, sinks):
    """All, some, none past the gate; sinks by position, among the drafts too."""
    x = Trees(4, d=64, window=4, tau=tau, sinks=sinks, seed=3, context=9000)
    x.append([0, 2, 3, 200])
    x.drafts([20, 20, 20, 20], CHAIN)
    x.check_tree()
    x.cache.set_tau(0.6)                                  # what is in the ring, and the drafts, by the new threshold
    x.oracle.set_tau(0.6)
    x.check_tree()


def test_without_logits():
    x = Trees(3, d=128, window=20, seed=4)
    x.append([100, 0, 7])
    x.drafts([20, 20, 1], CHAIN)
    x.check_tree(logits=False)
    x.drafts([21, 1, 1], CHAIN)
    with pytest.raises(spkv.SPKVError, match="invalid"):
        x.score(logits=False)
    x.check_tree()


def test_parents_that_are_no_parents():
    """Themselves, later ones, negative ones, ones far out of range: behind the newest token."""
    x = Trees(2, d=64, seed=5)
    x.append([200, 10])
    x.drafts([12, 12])
    x.parents = torch.tensor([5, 1, 0, -7, 2, 1 << 30, -(1 << 31), 6, 12, 9, 64, 10] * 2, dtype=torch.int32, device="cuda")
    x.check_tree()


@pytest.mark.parametrize("n,hq", [(3, 8), (16, 8), (16, 2)])
def test_a_chain_is_what_score_chunk_computes(n, hq):
    x = Trees(3, hq=hq, d=128, seed=6)
    x.append([500, 3, 130])
    x.drafts([n, n, n], CHAIN)
    out, lse = x.score()
    ref, ref_lse = x.cache.score_chunk(x.k, x.v, x.q, x.cu([n] * 3), want_lse=True)
    _, _, size = x.reference()
    err = (out.double() - ref.double()).abs().cpu().numpy()
    assert (err <= 2 * (2.0 ** -8 * (ref.abs().double().cpu().numpy() + size) + 1e-4 * size)).all()
    assert float((lse - ref_lse).abs().max()) < 2e-4


@pytest.mark.parametrize("hq,hk,d,lengths,counts", [
    (8, 2, 128, [9000], [60]), (8, 2, 128, [9000], [4]), (8, 2, 128, [5000, 1, 40, 3000, 300], [16, 16, 16, 16, 16]),
    (8, 8, 64, [6000, 17, 2500], [30, 7, 64]), (16, 1, 64, [7000, 7000], [33, 64])])
def test_long_lists_in_ranges(hq, hk, d, lengths, counts):
    x = Trees(len(lengths), hq=hq, hk=hk, d=d, window=100, seed=7, context=20000, keep=0.6)
    x.append(lengths)
    x.drafts(counts)
    x.check_tree()
    x.check_tree(sm_scale=0.0)


@pytest.mark.parametrize("hq,hk,d,lengths,counts", [
    (8, 8, 64, [9500, 10000, 500, 0, 128], [64, 40, 33, 9, 50]), (32, 8, 128, [9900, 31, 9700], [16, 16, 9]), (16, 16, 128, [9600, 1], [37, 64]),
    (48, 16, 64, [33, 9600, 200], [21, 13, 1])])
def test_lists_long_enough_for_copies_of_their_own(hq, hk, d, lengths, counts):
    """33 to 64 columns over 130 thousand pairs and more; short, empty and window-only sequences among them."""
    x = Trees(len(lengths), hq=hq, hk=hk, d=d, window=128, seed=hq + d, context=11000, keep=0.9)
    x.append(lengths)
    x.drafts(counts)
    x.check_tree()
    x.check_tree(sm_scale=0.0)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n,hq,hk", [(1, 8, 2), (4, 8, 2), (8, 8, 2), (13, 8, 2), (16, 8, 2), (29, 8, 2), (32, 8, 2), (50, 8, 2), (64, 8, 2), (64, 8, 1),
                                     (64, 2, 2)])
def test_one_long_list_and_many_short_ones(n, hq, hk, d):
    """A list in ranges that meet in a join; many lists that are a workgroup's each, drafts and results with them."""
    one = Trees(1, hq=hq, hk=hk, d=d, window=77, seed=n + d, keep=0.9)
    one.append([2900])
    one.drafts([n], seed=n)
    one.check_tree()
    many = Trees(26, hq=hq, hk=hk, d=d, window=77, seed=n + d, keep=0.5, context=500)
    many.append([0, 1, 31, 32, 33, 64, 65, 77, 78, 100, 160, 161, 200, 256, 300] + [b + 60 for b in range(11)])
    for most in (n, max(1, n - 3)):
        many.drafts([most if b % 3 else max(1, most - b) for b in range(26)], seed=n)
        many.check_tree()
    many.check_tree(sm_scale=0.0)


@pytest.mark.parametrize("n,hq,hk,d,lengths", [
    (n, 8, 2, d, lengths) for n in (4, 8, 13, 29, 64) for d, lengths in ((64, [2900]), (128, [25 * b for b in range(26)]))
] + [(13, 8, 2, 128, [2900]), (33, 16, 16, 64, [9600, 1])])
def test_scales_that_the_caller_chooses(n, hq, hk, d, lengths):
    """Every width, in ranges and whole, and long lists."""
    x = Trees(len(lengths), hq=hq, hk=hk, d=d, window=77, seed=n + d, keep=0.9, context=11000)
    x.append(lengths)
    x.drafts([n if b % 5 == 0 else 1 for b in range(len(lengths))], seed=n)
    scale = float(np.float32(0.3 * d ** -0.5))
    default, x.oracle.scale = x.oracle.scale, scale
    x.check_tree(sm_scale=scale)
    x.oracle.scale = default                              # (none, and what is none: the default)
    x.check_tree(sm_scale=-scale)


@pytest.mark.parametrize("batch", [1, 26])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n", [4, 8, 12, 30, 64])
def test_odd_values_in_ranges_and_in_whole_lists(n, d, batch):
    """Values that are not finite, in drafts and in ring keys that only the drafts near the newest token see."""
    x = Trees(batch, hq=8, hk=2, d=d, window=30, seed=n + d, keep=0.9)
    lengths = [2900] if batch == 1 else [7 * b for b in range(batch)]
    k, v, f = x.rows(sum(lengths))
    last = sum(lengths) - 30                                  # the last sequence's window: its gates off, its oldest values odd
    f[last:] -= 100
    v[last], v[last + 1, :, 3], k[last + 2, 1] = float("inf"), float("nan"), float("nan")
    x.cache.append(k, v, f, x.cu(lengths))
    v[last:last + 2], k[last + 2] = 0, 0                      # (drafts three deep and more do not see them)
    x.oracle.append(to_numpy_f32(k), to_numpy_f32(v), to_numpy_f32(f), x.cu(lengths))
    counts = [n] * batch
    x.drafts(counts, lambda r, m: [i - 1 for i in range(m - 1)] + [-1])
    x.f -= 100
    top = n * (batch - 1)
    bad = top + n - 2                                         # the chain's last draft; the last draft of all hangs elsewhere
    x.v[bad, :, 5] = float("-inf")
    out, lse = x.score()
    for r in (top, top + 1, bad, top + n - 1):
        assert not bool(torch.isfinite(out[r]).all()), r
    x.v[bad] = 0
    x.check_tree(got=(out, lse), rows=[r for r in range(n * batch) if r not in (top, top + 1, top + 2, bad, top + n - 1)])


@pytest.mark.parametrize("long", [False, True])
@pytest.mark.parametrize("n", [40, 64])
def test_odd_values_among_short_and_long_lists(n, long):
    """Ring keys that some drafts see, and drafts, that are not finite, in a short list beside short and long ones."""
    x = Trees(2, hq=8, hk=8, d=128, window=120, seed=n, keep=0.95, context=20000)
    x.append([19000 if long else 500, 0])
    k, v, f = x.rows(120)
    f = f - 100                                           # these leave the ring for good
    v[:3], v[3, 1], k[4, 2] = float("nan"), float("inf"), float("nan")
    x.cache.append(k, v, f, [0, 0, 120])
    k[4], v[:4] = 0, 0                                    # drafts below depth 5 do not see them
    x.oracle.append(to_numpy_f32(k), to_numpy_f32(v), to_numpy_f32(f), [0, 0, 120])
    x.drafts([n, n], lambda r, m: [i - 1 for i in range(m - 8)] + [10] * 8)
    x.f -= 100
    x.v[n - 4, :, 3], x.k[2 * n - 2], x.v[2 * n - 3, :, 64:] = float("nan"), float("nan"), float("-inf")
    out, lse = x.score()
    for r in (n - 4, n, n + 1, 2 * n - 2, 2 * n - 3):
        assert not bool(torch.isfinite(out[r]).all()), r
    x.v[n - 4], x.k[2 * n - 2], x.v[2 * n - 3] = 0, 0, 0
    clean = [r for r in range(2 * n) if r not in (n - 4, 2 * n - 2, 2 * n - 3) and not n <= r < n + 5]
    x.check_tree(got=(out, lse), rows=clean)


def test_more_pairs_than_a_launch_takes():
    x = Trees(200, hq=8, hk=4, d=64, window=20, seed=8, context=200)
    x.append([b % 50 for b in range(200)])
    x.drafts([b % 5 for b in range(200)])
    x.check_tree()
    wide = Trees(40, hq=64, hk=16, d=64, window=20, seed=9, context=100)
    wide.append([b % 30 for b in range(40)])
    wide.drafts([64 if b % 7 == 0 else 1 for b in range(40)])
    wide.check_tree()


def test_the_cache_is_left_as_it_was():
    x = Trees(3, d=64, window=50, seed=10)
    x.append([300, 0, 77])
    x.drafts([64, 5, 9])
    x.score()
    x.check(attend=False)
    # one path of every tree is accepted: what a chain of its drafts would have left
    parents, paths, at = x.parents.tolist(), [], 0
    for n in (64, 5, 9):
        path, i = [], n - 1
        while i >= 0:
            path.insert(0, at + i)
            i = parents[at + i]
        paths.append(path)
        at += n
    rows = [r for p in paths for r in p]
    counts = [len(p) for p in paths]
    x.cache.append_rows(x.k, x.v, x.f, torch.tensor(rows, dtype=torch.int32, device="cuda"), x.cu(counts))
    x.oracle.append(to_numpy_f32(x.k)[rows], to_numpy_f32(x.v)[rows], to_numpy_f32(x.f)[rows], x.cu(counts))
    x.check(attend=False)
    # the last draft of every path attends now as it did in the tree
    last = [p[-1] for p in paths]
    y = Trees(3, d=64, window=50, seed=10)
    y.append([300, 0, 77])
    y.k, y.v, y.f, y.q, y.parents, y.counts = x.k, x.v, x.f, x.q, x.parents, x.counts
    out, lse = y.score()
    again, again_lse = x.cache.decode_attention(x.q[last].contiguous(), want_lse=True)
    ref, _, size = y.reference()
    err = (out[last].double() - again.double()).abs().cpu().numpy()
    assert (err <= 2 * (2.0 ** -8 * (np.abs(ref[last]) + size[last]) + 1e-4 * size[last])).all()
    assert float((lse[last] - again_lse).abs().max()) < 2e-4


@pytest.mark.parametrize("n,hq", [(4, 8), (7, 8), (12, 8), (30, 8), (64, 8)])
def test_values_that_are_not_finite_stay_on_their_paths(n, hq):
    """In a draft: its descendants see it, no other draft does.  In the ring's oldest key: drafts near the newest token do."""
    x = Trees(2, hq=hq, d=128, window=40, seed=n, keep=0.0)
    x.append([40, 25])
    rng = np.random.default_rng(n)
    x.drafts([n, n], lambda r, m: random_tree(rng, m))
    bad = n // 3
    x.v[bad, :, 5] = float("inf")
    x.v[n + bad, :, ::3] = float("nan")
    x.k[n + bad, 0] = float("nan")
    parents = x.parents.tolist()
    clean = []
    for b in range(2):
        hit = {bad}
        for i in range(bad + 1, n):
            if parents[b * n + i] in hit:
                hit.add(i)
        clean += [b * n + i for i in range(n) if i not in hit]
    out, lse = x.score()
    rows = torch.tensor(sorted(set(range(2 * n)) - set(clean)), device="cuda")
    assert not bool(torch.isfinite(out[rows][:, :, 5 if n == 0 else slice(None)]).all(-1).any())
    x.v[bad], x.v[n + bad], x.k[n + bad] = 0, 0, 0        # (the clean rows do not see them)
    x.check_tree(got=(out, lse), rows=clean)


@pytest.mark.parametrize("n", [4, 8, 12, 30, 64])
def test_a_ring_key_that_some_drafts_see(n):
    """The window's oldest pairs are not finite and their gates off: drafts deep enough do not see them."""
    x = Trees(1, hq=8, d=64, window=10, seed=n, keep=0.0)
    k, v, f = x.rows(10)
    v[:2] = float("nan")
    x.cache.append(k, v, f, [0, 10])
    v = v.clone()
    v[:2] = 0
    x.oracle.append(to_numpy_f32(k), to_numpy_f32(v), to_numpy_f32(f), [0, 10])
    x.drafts([n], CHAIN)                                  # draft i sees keys i + 1 .. 9
    out, lse = x.score()
    assert not bool(torch.isfinite(out[0]).all(-1).any())
    x.check_tree(got=(out, lse), rows=list(range(1 if n < 2 else 1, n)))


def test_rows_behind_the_last_draft_stay():
    x = Trees(2, d=64, seed=11)
    x.append([100, 9])
    x.drafts([5, 3])
    out = torch.full((20, 8, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((20, 8), 7.0, device="cuda")
    x.check_tree(got=x.cache.score_tree(x.k, x.v, x.q, x.parents, [0, 5, 8], util_logits=x.f, out=out[:8], lse=lse[:8]))
    assert bool((out[8:] == 7).all()) and bool((lse[8:] == 7).all())
    assert x.cache.score_tree(x.k, x.v, x.q, x.parents, [0, 0, 0]) is None


def test_trees_in_a_graph():
    """Replays take other trees, other drafts, and lists that have grown since."""
    x = Trees(3, d=64, window=30, seed=12, keep=0.5, context=9000)
    x.append([200, 0, 31])
    x.drafts([9, 4, 13])
    x.check_tree()
    out, lse = torch.zeros_like(x.q), torch.zeros(26, 8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        x.score(out=out, lse=lse)
    mine = (x.k, x.v, x.f, x.q, x.parents)
    for turn in range(4):
        x.drafts([9, 4, 13], [random_tree, CHAIN, STAR, BROOM][turn], seed=turn)
        for to, src in zip(mine, (x.k, x.v, x.f, x.q, x.parents)):
            to.copy_(src)
        graph.replay()
        torch.cuda.synchronize()
        x.check_tree(got=(out, lse))
        x.check_tree()
        x.append([700 * turn + 1, 5, 1])
        x.fork([-1, -1, 0 if turn == 2 else -1])


@pytest.mark.parametrize("n", [4, 8, 16, 40])
def test_windows_of_thousands(n):
    """Rings of more half-pages than a wave's lanes hold gates of; long paths past none of it."""
    x = Trees(3, hq=8, hk=2, d=64, window=2600, seed=n, keep=0.3, context=6000)
    x.append([5000, 2599, 100])
    for shape in (random_tree, CHAIN):
        x.drafts([n, n, max(1, n // 2)], shape, seed=n)
        x.check_tree()


def test_trees_behind_shared_prompts():
    """Joined with the attention over a shared prompt, for sequences that hold a window of their own tokens or more."""
    shape = dict(d=128, window=40, keep=0.4, seed=30)
    prompts, own, all_of_it = Trees(2, **shape), Trees(3, **shape), Trees(3, **shape)
    prompts.append([500, 90])
    continues = [1, 0, 0]
    all_of_it.fork(continues, prompts)
    lengths = [40, 41, 200]
    k, v, f = own.rows(sum(lengths))
    for x in (own, all_of_it):
        x.cache.append(k, v, f, x.cu(lengths))
        x.oracle.append(to_numpy_f32(k), to_numpy_f32(v), to_numpy_f32(f), x.cu(lengths))
    own.drafts([30, 12, 1])
    for name in ("k", "v", "f", "q", "parents", "counts"):
        setattr(all_of_it, name, getattr(own, name))
    all_of_it.check_tree()
    out, lse = own.score()
    sharing = spkv.PrefixSharing(prompts.cache, continues)
    out, lse = own.cache.prefix_attention(sharing, own.q, own.cu([30, 12, 1]), out, lse, appended=False)
    ref, ref_lse, size = all_of_it.reference()
    # (what is joined has been rounded once already)
    assert (np.abs(out.double().cpu().numpy() - ref) <= 2 * (2.0 ** -8 * (np.abs(ref) + size) + 1e-4 * size)).all()
    assert (np.abs(lse.double().cpu().numpy() - ref_lse) <= 2e-4).all()


def test_turns_of_drafts_and_beams():
    """As they are used together: sequences taken over from where their prompts were fed, trees scored, paths accepted, beams that
    take each other's places, a slot given back and taken again."""
    rng = np.random.default_rng(31)
    shape = dict(d=64, window=50, keep=0.4, sinks=2, seed=31)
    prompts, x = Trees(2, **shape), Trees(6, **shape)
    prompts.append([333, 40])
    x.fork([0, 0, 0, 1, 1, 1], prompts)
    beams = [[0, 0, 2, 4, 4, 4], [1, 0, 2, 3, 5, 3], [-1, 2, 1, -2, 3, -1], [0, 0, 0, 0, 4, 5], [5, 4, 3, 2, 1, 0]]
    for turn, after in enumerate(beams):
        counts = [int(c) for c in rng.integers(1, 30, 6)]
        x.drafts(counts, seed=turn)
        x.check_tree()
        parents, rows, accepted, at = x.parents.tolist(), [], [], 0
        for n in counts:
            i, path = int(rng.integers(0, n)), []
            while i >= 0:
                path.insert(0, at + i)
                i = parents[at + i]
            accepted.append(len(path))
            rows += path
            at += n
        x.cache.append_rows(x.k, x.v, x.f, torch.tensor(rows, dtype=torch.int32, device="cuda"), x.cu(accepted))
        x.oracle.append(to_numpy_f32(x.k)[rows], to_numpy_f32(x.v)[rows], to_numpy_f32(x.f)[rows], x.cu(accepted))
        x.fork(after)
        x.check(attend=turn != 2)
        if turn == 2:                                     # the slot that was given back
            x.fork([-1, -1, -1, 0, -1, -1], prompts)
            x.check()


def test_two_caches_on_two_streams():
    xs = [Trees(2, d=64, seed=20 + i) for i in range(2)]
    for x in xs:
        x.append([800, 100])
        x.drafts([20, 9])
    torch.cuda.synchronize()
    got = []
    streams = [torch.cuda.Stream() for _ in xs]
    for _ in range(3):
        got = []
        for x, s in zip(xs, streams):
            with torch.cuda.stream(s):
                got.append(x.score())
    torch.cuda.synchronize()
    for x, g in zip(xs, got):
        x.check_tree(got=g)


def test_refusals():
    x = Trees(2, d=64, window=100, seed=13)
    x.append([10, 10])
    x.drafts([64, 1])
    k, v, q, p, f = x.k, x.v, x.q, x.parents, x.f
    with pytest.raises(spkv.SPKVError, match="invalid"):
        x.cache.score_tree(k, v, q, p, [0, 65, 65], util_logits=f)
    with pytest.raises(spkv.SPKVError, match="invalid"):
        x.cache.score_tree(k, v, q, p, [1, 64, 65], util_logits=f)
    for args in ((k[:64], v, q, p), (k, v.float(), q, p), (k, v, q[:, :4], p), (k, v, q, p.long()), (k, v, q, p[:64]), (k, v, q, p.cpu())):
        with pytest.raises(ValueError):
            x.cache.score_tree(*args, [0, 64, 65], util_logits=f)
    x.check_tree()
