"""Attention over shared prompts against the definition in 64 bits: every row for itself, the keys it sees -- of the
prompt and of its own sequence -- by position and gate.

Tolerances.  With p the exact weights: bf16 weights are off by 2^-8 of themselves, the sequence's own part is
rounded to bf16 (2^-8 again) before it is joined, scores are fp32 sums of D exact products (delta = (D + 8)
2^-24 times the largest sum of |q_d k_d| times the scale), sums run over at most n / 32 + 40 fp32 steps.  An output is
off by half a step of bf16 of itself and by (2 * 2^-8 + 2 delta + that) of sum p |v|; lse by delta, that and its own
rounding.  The 2-norm of a whole output stays under the harness's bound, for which errors of many keys are
independent."""

import math

import pytest
import torch

import paper_2605_14037_amd as spkv
from tests.harness import REL_L2_MAX

pytestmark = pytest.mark.gpu


class Setup:
    """A cache of prompts, a cache of sequences that continue them, and the same tokens on the host."""

    def __init__(self, prompts, own, member, hq, hk, d, window=128, tau=0.5, keep=0.3, seed=0, sinks=0, extra=64, v_gain=1.0):
        self.hq, self.hk, self.d, self.w, self.tau, self.sinks = hq, hk, d, window, tau, sinks
        self.theta = math.log(tau / (1 - tau))
        self.g = torch.Generator(device="cuda").manual_seed(1000 + seed)
        mu = {0.0: -40.0, 1.0: 40.0}.get(keep, torch.special.ndtri(torch.tensor(float(keep))).item()) + self.theta
        self.mu = mu
        self.member, self.batch = list(member), len(own)

        def cache(counts):
            pool = sum(max(0, n + extra - window) for n in counts) * hk
            return spkv.SPKVCache(len(counts), hq, hk, d, max_context=max(max(counts), 1) + extra,
                                  max_total_kept_tokens=pool, window=window, tau=tau)

        self.prefix, self.cache = cache(prompts), cache(own)
        if sinks:
            self.prefix.set_option(spkv.OPT_SINK_TOKENS, sinks)
        self.prompt = [[], [], []]
        self.own = [[], [], []]
        self._feed(self.prefix, self.prompt, prompts)
        self.held = [0] * self.batch
        self.append(own)
        self.sharing = spkv.PrefixSharing(self.prefix, self.member)

    def randn(self, *shape):
        return torch.randn(*shape, generator=self.g, device="cuda")

    def tokens(self, counts):
        n = sum(counts)
        return self.randn(n, self.hk, self.d).bfloat16(), self.randn(n, self.hk, self.d).bfloat16(), self.randn(n, self.hk) + self.mu

    def _feed(self, cache, lists, counts, kvf=None):
        kvf = self.tokens(counts) if kvf is None else kvf
        cu = [sum(counts[:b]) for b in range(len(counts) + 1)]
        cache.append(*kvf, cu)
        for t, into in zip(kvf, lists):
            parts = [t[cu[b]:cu[b + 1]].double().cpu() for b in range(len(counts))]
            into[:] = [torch.cat([a, b]) for a, b in zip(into, parts)] if into else parts
        return cu

    def append(self, counts):
        self._feed(self.cache, self.own, counts)
        self.held = [a + n for a, n in zip(self.held, counts)]

    def reference(self, q, counts, own_part=None, appended=True):
        """Exact output, lse and bounds of the rows of a call that brought `counts` tokens."""
        q = q.double().cpu()
        scale, group = self.d ** -0.5, self.hq // self.hk
        theta = torch.tensor(self.theta, dtype=torch.float64).float().double()
        out, lse, size, delta, steps = [], [], [], 0.0, 0
        row = 0
        for b in range(self.batch):
            for i in range(counts[b]):
                place = self.held[b] - (counts[b] if appended else 0) + i
                ks, vs, oks = [], [], []
                p = self.member[b]
                if p >= 0:
                    k, v, f = (t[p] for t in self.prompt)
                    s = torch.arange(len(k))
                    oks.append((len(k) + place - s < self.w)[:, None] | (f >= theta) | (s < self.sinks)[:, None])
                    ks.append(k)
                    vs.append(v)
                if own_part is None:
                    k, v, f = (t[b][:place + 1] for t in self.own)
                    s = torch.arange(len(k))
                    oks.append((place - s < self.w)[:, None] | (f >= theta))
                    ks.append(k)
                    vs.append(v)
                K = torch.cat(ks) if ks else torch.zeros(0, self.hk, self.d, dtype=torch.float64)
                V = torch.cat(vs) if vs else K
                ok = torch.cat(oks) if oks else torch.zeros(0, self.hk, dtype=torch.bool)
                qr = q[row].reshape(self.hk, group, self.d)
                x = torch.einsum("hgd,shd->hgs", qr, K) * scale
                if len(K):
                    big = torch.einsum("hgd,shd->hgs", qr.abs(), K.abs()) * scale
                    delta = max(delta, (self.d + 8) * 2.0 ** -24 * big.max().item())
                x = x.masked_fill(~ok.t()[:, None], -math.inf)
                z = torch.logsumexp(x, -1) if len(K) else torch.full((self.hk, group), -math.inf, dtype=torch.float64)
                steps = max(steps, len(K) // 32 + 40)
                if own_part is not None:
                    oo, oz = own_part[0][row].double().cpu(), own_part[1][row].double().cpu()
                    oz = oz.reshape(self.hk, group)
                    both = torch.logaddexp(z, oz)
                    part = torch.exp(oz - both).nan_to_num(0.0)[..., None] * oo.reshape(self.hk, group, self.d).nan_to_num(0.0)
                    z = both
                else:
                    part = torch.zeros(self.hk, group, self.d, dtype=torch.float64)
                w = torch.exp(x - z[..., None]).nan_to_num(0.0)
                out.append((torch.einsum("hgs,shd->hgd", w, V) + part).reshape(self.hq, self.d))
                size.append((torch.einsum("hgs,shd->hgd", w, V.abs()) + part.abs()).reshape(self.hq, self.d))
                lse.append(z.reshape(-1))
                row += 1
        return torch.stack(out), torch.stack(lse), torch.stack(size), delta, steps * 2.0 ** -24

    def check(self, got, got_lse, ref, label=""):
        out, lse, size, delta, sums = ref
        assert torch.isfinite(got).all(), label
        diff = (got.double().cpu() - out).abs()
        over = diff - (2.0 ** -8 * out.abs() + (2 * 2.0 ** -8 + 2 * delta + sums) * size)
        assert over.max() <= 0, f"{label}: off by {diff.flatten()[over.argmax()]:.3e}"
        assert (got.double().cpu() - out).norm() <= REL_L2_MAX * out.norm(), label
        if got_lse is not None:
            got_lse, some = got_lse.double().cpu(), torch.isfinite(lse)
            assert torch.equal(got_lse[~some], lse[~some])
            bound = delta + sums + 2.0 ** -22 * (1 + lse[some].abs())
            assert ((got_lse[some] - lse[some]).abs() <= bound).all(), label

    def decode(self, want_lse=True):
        q = self.randn(self.batch, self.hq, self.d).bfloat16()
        got = self.cache.decode_attention_shared(self.sharing, q, want_lse=want_lse)
        out, lse = got if want_lse else (got, None)
        self.check(out, lse, self.reference(q, [1] * self.batch), "decode")
        return q, out, lse


@pytest.mark.parametrize("window", [16, 100, 128])
@pytest.mark.parametrize("keep", [0.0, 0.3, 1.0])
@pytest.mark.parametrize("hq,hk,d", [(8, 2, 64), (8, 2, 128), (6, 2, 64), (16, 1, 128)])
def test_decode_around_the_window(hq, hk, d, keep, window):
    """Prompts of one token up to several pages, sequences of one token up to longer than the window."""
    w = window
    prompts = [1, 5, w - 1, w, w + 1, w + 31, 900]
    own = [1, 2, w - 1, w, w + 1, w + 7, 3 * w]
    s = Setup(prompts, own * 2, [0, 1, 2, 3, 4, 5, 6, 6, 5, 4, 3, 2, 1, 0], hq, hk, d, window=w, keep=keep)
    s.decode()
    for _ in range(2):
        s.append([1] * 14)
        s.decode(want_lse=False)


@pytest.mark.parametrize("batch,hq,hk,d", [
    (1, 4, 4, 128), (1, 32, 8, 128), (3, 10, 2, 128), (8, 32, 8, 128), (9, 32, 8, 128), (16, 8, 2, 64), (17, 8, 2, 64),
    (32, 8, 2, 128), (33, 16, 4, 128), (64, 8, 2, 128), (65, 8, 2, 64), (150, 8, 2, 128), (40, 24, 3, 64), (21, 13, 1, 64)])
def test_decode_columns(batch, hq, hk, d):
    """One to many columns of one prompt: every width of a workgroup, full and partly filled, several blocks."""
    s = Setup([2000], [1 + (7 * b) % 150 for b in range(batch)], [0] * batch, hq, hk, d, keep=0.25, seed=batch)
    s.decode()


@pytest.mark.parametrize("batch", [1, 3, 6, 12, 40])
def test_long_lists_and_wide_windows(batch):
    """More pages than are sent for beforehand (256), and more of the ring than a wave keeps the gates of."""
    s = Setup([24000], [1 + 5 * b for b in range(batch)], [0] * batch, 8, 2, 64, keep=0.95, seed=batch)
    s.decode()
    s = Setup([6000], [1 + 500 * b for b in range(batch)], [0] * batch, 8, 2, 64, keep=0.3, window=5000, seed=batch, extra=20000)
    s.decode()


def test_decode_of_uneven_prompts():
    """Prompts of unlike lengths and numbers of sequences, some empty, some that nobody continues, none."""
    member = [3, 0, -1, 0, 0, 5, 3, 0, 2, 0, 0, 0, 1, 0, -1, 0]
    s = Setup([3000, 0, 70, 431, 900, 1], [1 + 11 * b for b in range(16)], member, 8, 2, 128, keep=0.4, seed=3)
    q, out, lse = s.decode()
    alone, alone_lse = s.cache.decode_attention(q, want_lse=True)
    out, lse = s.cache.prefix_attention(s.sharing, q, None, alone, alone_lse)
    s.check(out, lse, s.reference(q, [1] * 16), "joined")
    for b in (2, 12, 14):                                # no prompt, an empty one: the sequence's own, bit for bit
        assert torch.equal(out[b], alone[b]) and torch.equal(lse[b], alone_lse[b])
    s.sharing[2] = s.member[2] = 4
    s.decode()
    s.sharing.prefix_of[:] = [-1] * 16
    s.member = [-1] * 16
    s.decode()


def test_decode_with_sinks_threshold_and_release():
    s = Setup([700, 300], [5, 40, 1], [0, 1, 0], 8, 2, 64, tau=0.3, keep=0.2, sinks=3)
    s.decode()
    s.prefix.set_tau(0.3)
    s.prefix.release_sequence(1)                         # the prompt of sequence 1 is gone: its own tokens alone
    for t in s.prompt:
        t[1] = t[1][:0]
    s.decode()


@pytest.mark.parametrize("own", [[3000, 1, 700], [2900, 2900, 2900]])
def test_long_sequences_of_their_own(own):
    """Longer than what rides in the prompts' launch."""
    s = Setup([700, 300], own, [0, 1, 0], 8, 2, 64, keep=0.9)
    s.decode()


def test_more_sequences_than_travel_with_the_launch():
    s = Setup([200, 90, 1], [1 + b % 37 for b in range(300)], [b % 3 for b in range(300)], 2, 1, 64)
    s.decode()


def test_many_small_prompts():
    n = 270
    s = Setup([1 + 9 * p for p in range(n)], [1 + p % 5 for p in range(n)], list(range(n))[::-1], 8, 2, 64, keep=0.5)
    s.decode()


@pytest.mark.parametrize("hq,hk,d,counts", [
    (32, 8, 128, [1, 0, 3, 1]), (8, 2, 64, [16, 2, 0, 7]), (8, 2, 128, [40, 150, 129, 1]), (8, 2, 64, [300, 0, 0, 5]),
    (13, 1, 64, [31, 5, 2, 1]), (16, 1, 128, [20, 20, 20, 20])])
@pytest.mark.parametrize("shared", [True, False], ids=["one", "three"])
def test_questions(hq, hk, d, counts, shared):
    """Several tokens a sequence: the own part from prefill_attention, joined with the prompts'."""
    member = [0, 0, 0, 0] if shared else [2, 0, 1, 2]
    s = Setup([1100, 150, 2300], [1, 130, 0, 60], member, hq, hk, d, keep=0.3, seed=sum(counts), extra=320)
    k, v, f = s.tokens(counts)
    q = s.randn(sum(counts), hq, d).bfloat16()
    cu = [sum(counts[:b]) for b in range(5)]
    own, own_lse = s.cache.prefill_attention(k, v, f, q, cu, want_lse=True)
    for t, into in zip((k, v, f), s.own):
        into[:] = [torch.cat([into[b], t[cu[b]:cu[b + 1]].double().cpu()]) for b in range(4)]
    s.held = [a + n for a, n in zip(s.held, counts)]
    out, lse = s.cache.prefix_attention(s.sharing, q, cu, own, own_lse)
    s.check(out, lse, s.reference(q, counts), "all keys")
    s.check(out, lse, s.reference(q, counts, (own, own_lse)), "given the own part")
    again, again_lse = s.cache.prefix_attention(s.sharing, q, cu, own, own_lse, out=own, lse=own_lse)
    assert again is own and torch.equal(own, out) and torch.equal(own_lse, lse)


def test_drafts_that_are_not_appended():
    s = Setup([500, 40], [3, 200, 90], [0, 1, 0], 8, 2, 128, window=64)
    counts = [2, 4, 1]
    k, v, f = s.tokens(counts)
    q = s.randn(7, 8, 128).bfloat16()
    cu = [0, 2, 6, 7]
    own, own_lse = s.cache.score_chunk(k, v, q, cu, want_lse=True)
    out, lse = s.cache.prefix_attention(s.sharing, q, cu, own, own_lse, appended=False)
    s.check(out, lse, s.reference(q, counts, (own, own_lse), appended=False), "drafts")


def test_rows_that_see_nothing():
    """No key of the own sequence (lse -infinity, whatever the values), none of the prompt, neither."""
    s = Setup([40], [200, 200, 1, 1], [0, -1, 0, -1], 8, 2, 64, window=16, keep=0.0)      # nothing kept: seen up to place 15
    q = s.randn(4, 8, 64).bfloat16()
    own = s.randn(4, 8, 64).bfloat16()
    own_lse = s.randn(4, 8)
    own[2:] = float("nan")
    own_lse[2:] = -math.inf
    out, lse = s.cache.prefix_attention(s.sharing, q, None, own, own_lse)
    assert torch.equal(out[:2], own[:2])                 # gates off and far: the own part
    assert (lse[:2] - own_lse[:2]).abs().max() <= 2.0 ** -20 and torch.equal(lse[1], own_lse[1])
    ref = s.reference(q, [1] * 4, (own, own_lse))
    got = out[2:3].double().cpu()
    assert (got - ref[0][2:3]).abs().max() <= (3 * 2.0 ** -8) * ref[2][2:3].max() and torch.isfinite(got).all()
    s.append([40] * 4)
    own_lse[:] = -math.inf
    own[:] = float("nan")
    s.sharing.prefix_of[:] = [0] * 4
    out, lse = s.cache.prefix_attention(s.sharing, q, None, own, own_lse)
    assert (out == 0).all() and (lse == -math.inf).all()


@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
def test_what_no_row_sees_does_not_show(bad):
    """Infinities and NaN in values and keys whose gate is off, behind the window of all rows, and behind list ends."""
    s = Setup([0], [60, 80], [0, 0], 8, 2, 64, window=32, keep=0.0, extra=400)
    k, v, f = s.tokens([300])
    f = s.randn(300, 2)
    f[270:, :] = -9.0
    f[280] = 9.0
    k[281:290], v[270:275], v[290:] = bad, bad, bad
    s._feed(s.prefix, s.prompt, [300], (k, v, f))
    for t in s.prompt[:2]:
        t[0] = t[0].nan_to_num(0.0, 0.0, 0.0)
    s.decode()


def test_pages_that_held_something_else():
    """A prompt in pages and a ring that held infinities before."""
    s = Setup([0], [5, 9], [0, 0], 8, 2, 128, keep=0.5, extra=1500)
    k, v, f = s.tokens([1000])
    s.prefix.append(torch.full_like(k, float("inf")), torch.full_like(v, float("nan")), f.abs() + 1, [0, 1000])
    s.prefix.release_sequence(0)
    s._feed(s.prefix, s.prompt, [333])
    s.decode()


def test_same_as_the_whole_sequence_in_one_cache():
    """Prompt and own tokens appended to one sequence each: the same attention, up to both calls' roundings."""
    s = Setup([1500, 200], [30, 250, 128], [0, 0, 1], 32, 8, 128, seed=9)
    whole = spkv.SPKVCache(3, 32, 8, 128, max_context=2000, max_total_kept_tokens=3 * 8 * 2000)
    parts = [[torch.cat([s.prompt[i][p], s.own[i][b]]) for b, p in enumerate(s.member)] for i in range(3)]
    n = [len(x) for x in parts[0]]
    k, v, f = (torch.cat(x).cuda() for x in parts)
    whole.append(k.bfloat16(), v.bfloat16(), f.float().contiguous(), [0, n[0], n[0] + n[1], sum(n)])
    q, out, lse = s.decode()
    one, one_lse = whole.decode_attention(q, want_lse=True)
    assert (out.float() - one.float()).norm() <= 2 * REL_L2_MAX * one.float().norm()
    assert (lse - one_lse).abs().max() <= 1e-4


def test_streams_and_small_workspaces():
    s = Setup([2500], [10] * 20, [0] * 20, 8, 2, 128)
    q, out, lse = s.decode()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = s.cache.decode_attention_shared(s.sharing, q)
    side.synchronize()
    assert torch.equal(again, out)
    slot = 20 * 8 * 130 * 4                              # bytes of one range of every list
    slots = min(255, (96 << 20) // slot)
    tables = s.sharing.workspace_bytes(20) - -(-slots * slot // 256) * 256
    ws = torch.empty(tables + 3 * slot, dtype=torch.uint8, device="cuda")
    few = s.cache.decode_attention_shared(s.sharing, q, workspace=ws)
    assert (few.float() - out.float()).norm() <= 2 * REL_L2_MAX * out.float().norm()
    with pytest.raises(spkv.SPKVError):
        s.cache.decode_attention_shared(s.sharing, q, workspace=ws[:tables + slot - 1])


def test_captured_steps_replay_as_sequences_grow():
    """Append and shared attention captured once, replayed while the own sequences leave the prompt's window."""
    s = Setup([600, 77], [3, 30, 31], [0, 1, 0], 8, 2, 64, window=40, keep=0.3, extra=200)
    k, v, f = s.tokens([1, 1, 1])
    q = s.randn(3, 8, 64).bfloat16()
    out = torch.empty_like(q)
    lse = torch.empty(3, 8, device="cuda")
    ws = torch.empty(s.sharing.workspace_bytes(3), dtype=torch.uint8, device="cuda")
    cu = s.cache.make_cu([0, 1, 2, 3])
    s.decode()                                           # reads the lengths
    s.cache.safe_steps()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.cache.append(k, v, f, cu)
        s.cache.decode_attention_shared(s.sharing, q, out=out, lse=lse, workspace=ws)
    for step in range(45):
        if step > 0:                                     # the captured call itself counted one
            s.cache.advance(1)
        for t, new in zip((k, v, f), s.tokens([1, 1, 1])):
            t.copy_(new)
        q.copy_(s.randn(3, 8, 64).bfloat16())
        graph.replay()
        torch.cuda.synchronize()
        for t, into in zip((k, v, f), s.own):
            into[:] = [torch.cat([into[b], t[b:b + 1].double().cpu()]) for b in range(3)]
        s.held = [n + 1 for n in s.held]
        s.check(out, lse, s.reference(q, [1] * 3), f"replay {step}")


@pytest.mark.parametrize("bad", [float("inf"), -float("inf"), float("nan")])
@pytest.mark.parametrize("hq,hk,d,batch", [(4, 4, 64, 3), (8, 2, 128, 7), (8, 2, 128, 14), (16, 2, 64, 15), (16, 1, 128, 20)])
def test_what_one_row_sees_does_not_show_in_another(hq, hk, d, batch, bad):
    """Keys with their gate off that are still inside the window of some sequences, their values not finite: the
    sequences that see them get them, the others what they would without."""
    own = [1 + (5 * b) % 60 for b in range(batch)]
    s = Setup([0], own, [0] * batch, hq, hk, d, window=48, keep=0.0, extra=400, seed=batch)
    k, v, f = s.tokens([300])
    f = s.randn(300, hk) - 9.0
    f[290:] += 18.0
    there = [260, 275, 281]
    for i, at in enumerate(there):
        v[at, :, 5 * i::7] = bad
    s._feed(s.prefix, s.prompt, [300], (k, v, f))
    q = s.randn(batch, hq, d).bfloat16()
    out, lse = s.cache.decode_attention_shared(s.sharing, q, want_lse=True)
    got = out.clone()
    for b in range(batch):
        for i, at in enumerate(there):
            if 300 + own[b] - 1 - at < 48:
                x = got[b, :, 5 * i::7]
                assert not torch.isfinite(x).any(), (b, at)      # (weights in two parts: an infinity may come out as a NaN)
                x.zero_()
    assert torch.isfinite(got).all()
    s.prompt[1][0] = s.prompt[1][0].nan_to_num(0.0, 0.0, 0.0)
    ref = s.reference(q, [1] * batch)
    for b in range(batch):
        for i, at in enumerate(there):
            if 300 + own[b] - 1 - at < 48:
                ref[0][b, :, 5 * i::7] = 0.0
    s.check(got, lse, ref, "finite part")


def test_a_query_that_is_not_a_number_shows():
    """... in its own rows alone, in the output and in lse, whether or not the sequence has keys of its own."""
    s = Setup([500, 40], [3, 80, 7, 1], [0, 0, 1, 0], 8, 2, 64)
    q, out, lse = s.decode()
    q[1, 3, 5] = float("nan")
    bad, bad_lse = s.cache.decode_attention_shared(s.sharing, q, want_lse=True)
    assert torch.isnan(bad[1, 3]).all() and torch.isnan(bad_lse[1, 3])
    bad[1, 3], bad_lse[1, 3] = out[1, 3], lse[1, 3]
    assert torch.equal(bad, out) and torch.equal(bad_lse, lse)
    own, own_lse = s.randn(4, 8, 64).bfloat16(), s.randn(4, 8)
    own_lse[2] = -math.inf
    bad, bad_lse = s.cache.prefix_attention(s.sharing, q, None, own, own_lse)
    assert torch.isnan(bad[1, 3]).all() and torch.isnan(bad_lse[1, 3])
    assert torch.isfinite(bad[0]).all() and torch.isfinite(bad[2:]).all()
    own_lse[0, 2] = float("nan")
    bad, bad_lse = s.cache.prefix_attention(s.sharing, q, None, own, own_lse)
    assert torch.isnan(bad[0, 2]).all() and torch.isnan(bad_lse[0, 2])


@pytest.mark.parametrize("asking", [64, 65])
@pytest.mark.parametrize("appended", [True, False], ids=["appended", "drafts"])
def test_questions_of_many_sequences(asking, appended):
    """Up to 64 sequences with rows and a prompt travel with the launches, more by tables; others have neither."""
    batch = 90
    counts = [0 if b % 7 == 3 else 1 + (5 * b) % 9 for b in range(batch)]
    member, n = [], 0
    for b in range(batch):
        use = counts[b] > 0 and n < asking
        member.append((0, 2, 1)[b % 3] if use else -1 if b % 2 else 3)
        n += use
    assert n == asking
    s = Setup([700, 90, 300, 0], [(11 * b) % 60 for b in range(batch)], member, 8, 2, 64, window=64, keep=0.3, seed=asking)
    cu = [sum(counts[:b]) for b in range(batch + 1)]
    k, v, f = s.tokens(counts)
    q = s.randn(cu[-1], 8, 64).bfloat16()
    if appended:
        own, own_lse = s.cache.prefill_attention(k, v, f, q, cu, want_lse=True)
        s.held = [a + n for a, n in zip(s.held, counts)]
    else:
        own, own_lse = s.cache.score_chunk(k, v, q, cu, want_lse=True)
    out, lse = s.cache.prefix_attention(s.sharing, q, cu, own, own_lse, appended=appended)
    s.check(out, lse, s.reference(q, counts, (own, own_lse), appended=appended), "given the own part")
    for b in range(batch):
        if member[b] in (-1, 3):
            assert torch.equal(out[cu[b]:cu[b + 1]], own[cu[b]:cu[b + 1]]) and torch.equal(lse[cu[b]:cu[b + 1]], own_lse[cu[b]:cu[b + 1]])


def test_questions_without_any_prompt():
    """No sequence continues a prompt, or only an empty one: the own part, bit for bit."""
    s = Setup([0, 50], [5, 9, 1], [-1, 0, -1], 8, 2, 128)
    own, own_lse = s.randn(11, 8, 128).bfloat16(), s.randn(11, 8)
    out, lse = s.cache.prefix_attention(s.sharing, s.randn(11, 8, 128).bfloat16(), [0, 3, 10, 11], own, own_lse)
    assert torch.equal(out, own) and torch.equal(lse, own_lse)
