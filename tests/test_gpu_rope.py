"""qk_norm_rope and its gradients against the definition in 64 bits.

Tolerances, from the arithmetic: with u = 2^-24 an output is off by its own rounding, half a step of its
type relative to itself, and by the fp32 work before it: 16 squares added in a lane and up to three
exchanges, the square root's reciprocal, two products (together under 24 u of the element), cosine and
sine to 4 u, two products and a sum: under 32 u of |a| + |b|, the normed elements of the pair.  The
backward pass has twice that of |g w| + |x| r^2 mean|g w x|.  A weight's gradient adds up products that
are off by 40 u, 8 rows at most in a lane at the sizes here, then 5 exchanges, 32 rows of partial sums and 5 more:
under 128 u of the sum of the products' magnitudes."""

import pytest
import torch

import paper_2605_14037_amd as spkv

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def _turn(rope, positions):
    """cos, sin [tokens, 1, pairs] in 64 bits."""
    n = rope.rot_dim // 2
    pos = positions.reshape(rope.n_axes, -1).double().cpu()
    f = torch.tensor(list(rope._freq)[:n], dtype=torch.float64)
    ax = torch.tensor(list(rope._axis)[:n], dtype=torch.long)
    phi = pos[ax].t() * f
    return torch.cos(phi)[:, None], torch.sin(phi)[:, None]


def _index(rope):
    n = rope.rot_dim // 2
    i = torch.arange(n)
    return (2 * i, 2 * i + 1) if rope.adjacent else (i, i + n)


def _rotate(rope, x, cos, sin):
    a, b = _index(rope)
    y = x.clone()
    y[..., a] = x[..., a] * cos - x[..., b] * sin
    y[..., b] = x[..., a] * sin + x[..., b] * cos
    return y


def _pair_size(rope, x):
    """|a| + |b| in the place of both elements of every pair, |x| elsewhere."""
    a, b = _index(rope)
    y = x.abs()
    y[..., a] = y[..., b] = x[..., a].abs() + x[..., b].abs()
    return y


def _norm(x, w, eps):
    return x if eps is None else x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * w


def _forward(rope, x, w, positions, eps):
    """(result, bound of the fp32 work)"""
    n = _norm(x.double().cpu(), None if w is None else w.double().cpu(), eps)
    return _rotate(rope, n, *_turn(rope, positions)), 32 * U * _pair_size(rope, n)


def _check(got, ref, err, label):
    got, h = got.detach(), HALF[got.dtype]
    diff = (got.double().cpu() - ref).abs()
    over = diff - (h * ref.abs() + (1 + h) * err)
    assert torch.isfinite(got).all(), label
    assert over.max() <= 0, f"{label}: off by {diff.flatten()[over.argmax()]:.3e}, allowed {(diff - over).flatten()[over.argmax()]:.3e}"


def _inputs(t, hq, hk, d, dtype, seed=0, gain=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    qkv = (gain * torch.randn(t, hq + 2 * hk, d, generator=g, device="cuda")).to(dtype)
    w = 1.0 + 0.3 * torch.randn(2, d, generator=g, device="cuda")
    return qkv, qkv[:, :hq], qkv[:, hq:hq + hk], qkv[:, hq + hk:], w[0].contiguous(), w[1].contiguous(), g


ROPES = [dict(), dict(rot_dim=16), dict(rot_dim=48), dict(rot_dim=0), dict(adjacent=True), dict(adjacent=True, rot_dim=2),
         dict(adjacent=True, rot_dim=30), dict(sections=True), dict(axis=True, adjacent=True, rot_dim=60)]


def _rope(d, rot_dim=None, adjacent=False, sections=False, axis=False):
    n = (d if rot_dim is None else rot_dim) // 2
    kw = {}
    if sections:
        kw["sections"] = [n // 4, 3 * n // 8, n - n // 4 - 3 * n // 8]
    if axis:
        kw["axis"] = [i % 3 for i in range(n)]
    return spkv.Rope(d, rot_dim=rot_dim, theta=1e6, adjacent=adjacent, **kw)


def _positions(rope, t, g, most=1 << 20):
    p = torch.randint(0, most, (rope.n_axes, t), generator=g, device="cuda", dtype=torch.int32)
    return p[0].contiguous() if rope.n_axes == 1 else p


@pytest.mark.parametrize("rope", ROPES, ids=str)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("t,hq,hk,d", [(1, 32, 8, 128), (5, 8, 2, 64), (67, 3, 3, 64), (131, 5, 1, 128)])
def test_forward(t, hq, hk, d, dtype, rope):
    rope = _rope(d, **rope)
    qkv, q, k, v, qw, kw, g = _inputs(t, hq, hk, d, dtype)
    pos = _positions(rope, t, g)
    for eps in (1e-6, None):
        w = dict(q_weight=qw, k_weight=kw, eps=eps) if eps is not None else {}
        qo, ko, vo = spkv.qk_norm_rope(q, k, pos, rope, v=v, **w)
        assert qo.is_contiguous() and ko.is_contiguous() and torch.equal(vo, v)
        _check(qo, *_forward(rope, q, qw, pos, eps), "q")
        _check(ko, *_forward(rope, k, kw, pos, eps), "k")
        two = spkv.qk_norm_rope(q, k, pos, rope, **w)
        assert len(two) == 2 and torch.equal(two[0], qo) and torch.equal(two[1], ko)


@pytest.mark.parametrize("rope", ROPES, ids=str)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("t,hq,hk,d", [(1, 32, 8, 128), (5, 8, 2, 64), (67, 3, 3, 64), (1003, 5, 1, 128)])
def test_backward(t, hq, hk, d, dtype, rope):
    rope = _rope(d, **rope)
    qkv, q, k, v, qw, kw, g = _inputs(t, hq, hk, d, dtype)
    pos = _positions(rope, t, g)
    dq, dk, dv = (torch.randn(t, h, d, generator=g, device="cuda").to(dtype) for h in (hq, hk, hk))
    cos, sin = _turn(rope, pos)
    for eps in (1e-6, None):
        grad = torch.full_like(qkv, float("nan"))
        into = (grad[:, :hq], grad[:, hq:hq + hk], grad[:, hq + hk:])
        w = dict(q=q, k=k, q_weight=qw, k_weight=kw, eps=eps) if eps is not None else {}
        got_w = spkv.qk_norm_rope_backward(dq, dk, pos, rope, dv=dv, out=into, **w)
        assert torch.equal(into[2], dv) and len(got_w) == (2 if eps is not None else 0)
        for i, (x, wt, dy, name) in enumerate(((q, qw, dq, "q"), (k, kw, dk, "k"))):
            y = _rotate(rope, dy.double().cpu(), cos, -sin)
            size = _pair_size(rope, dy.double().cpu())
            if eps is None:
                _check(into[i], y, 32 * U * size, "d" + name)
                continue
            x, wt = x.double().cpu(), wt.double().cpu()
            r = 1 / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
            ref = r * (y * wt - x * r * r * (y * wt * x).mean(-1, keepdim=True))
            around = r * (size * wt.abs() + x.abs() * r * r * (size * (wt * x).abs()).mean(-1, keepdim=True))
            _check(into[i], ref, 64 * U * around, "d" + name)
            _check(got_w[i], (y * x * r).sum((0, 1)), 128 * U * (size * (x * r).abs()).sum((0, 1)), "weight of " + name)
        dense = spkv.qk_norm_rope_backward(dq, dk, pos, rope, dv=dv, **w)
        for a, b in zip(dense[:3], into):
            assert torch.equal(a, b)
        assert all(torch.equal(a, b) for a, b in zip(dense[3:], got_w))     # fixed order: the same bits


def test_many_rows_take_longer_tiles():
    """Sizes at which a tile takes more passes, forwards and backwards (and a workgroup several tiles)."""
    rope = _rope(64, sections=True)
    for t in (1500, 12001):
        qkv, q, k, v, qw, kw, g = _inputs(t, 24, 8, 64, torch.bfloat16)
        pos = _positions(rope, t, g, 5000)
        qo, ko, vo = spkv.qk_norm_rope(q, k, pos, rope, qw, kw, 1e-5, v=v)
        _check(qo, *_forward(rope, q, qw, pos, 1e-5), "q")
        _check(ko, *_forward(rope, k, kw, pos, 1e-5), "k")
        assert torch.equal(vo, v)
        dq, dk, dqw, dkw = spkv.qk_norm_rope_backward(q, k, pos, rope, q=q, k=k, q_weight=qw, k_weight=kw, eps=1e-5)
        cos, sin = _turn(rope, pos)
        for x, wt, got, got_w in ((q, qw, dq, dqw), (k, kw, dk, dkw)):
            x, wt = x.double().cpu(), wt.double().cpu()
            r = 1 / torch.sqrt((x * x).mean(-1, keepdim=True) + 1e-5)
            y, size = _rotate(rope, x, cos, -sin), _pair_size(rope, x)
            around = r * (size * wt.abs() + x.abs() * r * r * (size * (wt * x).abs()).mean(-1, keepdim=True))
            _check(got, r * (y * wt - x * r * r * (y * wt * x).mean(-1, keepdim=True)), 64 * U * around, "dx")
            rows = -(-t * 32 // (64 * 1024)) + 8                     # of a lane, at most
            _check(got_w, (y * x * r).sum((0, 1)), (128 + rows) * U * (size * (x * r).abs()).sum((0, 1)), "weight")


@pytest.mark.parametrize("hq,hk", [(1, 1), (2, 1)])
def test_few_heads_bring_many_tokens_to_a_tile(hq, hk):
    rope = _rope(128)
    qkv, q, k, v, qw, kw, g = _inputs(40003, hq, hk, 128, torch.bfloat16)
    pos = _positions(rope, 40003, g)
    qo, ko = spkv.qk_norm_rope(q, k, pos, rope, qw, kw, 1e-6)
    _check(qo, *_forward(rope, q, qw, pos, 1e-6), "q")
    _check(ko, *_forward(rope, k, kw, pos, 1e-6), "k")


@pytest.mark.parametrize("positions", [[0, 1, -1, -77777], [2 ** 31 - 1, -2 ** 31, 2 ** 30 + 1, 123456789]])
def test_far_and_negative_positions(positions):
    """cos and sin of the reference are of pos * f in 64 bits: 2^31 * 2^-53 rad of its own."""
    rope = _rope(128)
    qkv, q, k, v, qw, kw, g = _inputs(4, 4, 2, 128, torch.float32)
    pos = torch.tensor(positions, dtype=torch.int32, device="cuda")
    qo, ko = spkv.qk_norm_rope(q, k, pos, rope)
    for got, x in ((qo, q), (ko, k)):
        ref, err = _forward(rope, x, None, pos, None)
        _check(got, ref, err + 2.0 ** -21 * _pair_size(rope, x.double().cpu()), "far")


def test_strides_and_places():
    """Heads before tokens, one key head for all (stride 0), in place, another stream."""
    rope = _rope(64, rot_dim=32)
    t, hq, hk, d = 37, 6, 3, 64
    g = torch.Generator(device="cuda").manual_seed(3)
    q = torch.randn(hq, t, d, generator=g, device="cuda").bfloat16().transpose(0, 1)
    k = torch.randn(t, 1, d, generator=g, device="cuda").bfloat16().expand(t, hk, d)
    pos = _positions(rope, t, g)
    qw = 1 + 0.1 * torch.randn(d, generator=g, device="cuda")
    qo, ko = spkv.qk_norm_rope(q, k, pos, rope, q_weight=qw, eps=0.0)
    one = torch.ones(d, device="cuda")
    _check(qo, *_forward(rope, q, qw, pos, 0.0), "q")
    _check(ko, *_forward(rope, k, one, pos, 0.0), "k")
    with pytest.raises(spkv.SPKVError):
        spkv.qk_norm_rope(q, k, pos, rope, out=(qo, k))                 # rows that share their elements
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    buf = torch.cat([q, k], 1).contiguous()
    with torch.cuda.stream(side):
        views = (buf[:, :hq], buf[:, hq:])
        spkv.qk_norm_rope(*views, pos, rope, q_weight=qw, eps=0.0, out=views)
    side.synchronize()
    assert torch.equal(views[0], qo) and torch.equal(views[1], ko)
    dq = spkv.qk_norm_rope_backward(qo, ko, pos, rope, q=q, k=k, q_weight=qw, eps=0.0)
    x = torch.cat([q, k], 1).contiguous()
    gq, gk = qo.clone(), ko.clone()
    again = spkv.qk_norm_rope_backward(gq, gk, pos, rope, q=x[:, :hq], k=x[:, hq:], q_weight=qw, eps=0.0, out=(gq, gk))
    assert torch.equal(gq, dq[0]) and torch.equal(gk, dq[1])
    assert torch.equal(again[0], dq[2]) and torch.equal(again[1], dq[3])


def test_rows_keep_to_themselves():
    """Rows of zeros stay zeros; a row with NaN or infinity spoils no other."""
    rope = _rope(128)
    qkv, q, k, v, qw, kw, g = _inputs(9, 4, 2, 128, torch.bfloat16)
    pos = _positions(rope, 9, g)
    clean = spkv.qk_norm_rope(q, k, pos, rope, qw, kw, 1e-6)
    q[2, 1], q[3, 0, 5], k[4, 1, 127], q[6, 3] = 0.0, float("nan"), float("inf"), 0.0
    qo, ko = spkv.qk_norm_rope(q, k, pos, rope, qw, kw, 1e-6)
    assert (qo[2, 1] == 0).all() and (qo[6, 3] == 0).all()
    assert qo[3, 0].isnan().all() and ko[4, 1].isnan().any()
    qo[2, 1], qo[3, 0], ko[4, 1], qo[6, 3] = clean[0][2, 1], clean[0][3, 0], clean[1][4, 1], clean[0][6, 3]
    assert torch.equal(qo, clean[0]) and torch.equal(ko, clean[1])
    dy, dk = torch.ones_like(qo), torch.ones_like(ko)
    dq, dk, _, _ = spkv.qk_norm_rope_backward(dy, dk, pos, rope, q=q, k=k, q_weight=qw, k_weight=kw, eps=1e-6)
    assert torch.isfinite(dq[2, 1]).all() and dq[3, 0].isnan().all()
    bad = torch.zeros(9, 4, dtype=torch.bool, device="cuda")
    bad[3, 0] = True
    assert torch.isfinite(dq[~bad]).all()


def test_no_tokens():
    rope, z = _rope(64), torch.zeros(0, 4, 64, dtype=torch.bfloat16, device="cuda")
    pos = torch.zeros(0, dtype=torch.int32, device="cuda")
    assert spkv.qk_norm_rope(z, z[:, :2], pos, rope, eps=1e-6)[0].shape == (0, 4, 64)
    _, _, dqw, dkw = spkv.qk_norm_rope_backward(z, z[:, :2], pos, rope, q=z, k=z[:, :2], eps=1e-6)
    assert (dqw == 0).all() and (dkw == 0).all()


@pytest.mark.parametrize("what", ["x", "weight"])
def test_gradient_against_differences(what):
    """Central differences of the operator itself along random directions, fp32.  L = sum(dy * y) is added up in
    64 bits, so a difference is off from that of the definition in 64 bits by the outputs' errors, 40 u of
    sum |dy| (|a| + |b|) at most, over the step; and that from the gradient by step^2 / 6 of the third derivative (of
    x / |x| along a unit of its size: 15 of the same sum, four times that for rows shorter than one) and
    64 u of the gradient's own."""
    rope = _rope(64, sections=True)
    t, hq, hk, d, eps, step = 11, 6, 2, 64, 1e-2, 2.0 ** -8
    qkv, q, k, v, qw, kw, g = _inputs(t, hq, hk, d, torch.float32, seed=5)
    pos = _positions(rope, t, g)
    dy = [torch.randn(t, h, d, generator=g, device="cuda") for h in (hq, hk)]
    q, k = q.contiguous(), k.contiguous()
    got = spkv.qk_norm_rope_backward(*dy, pos, rope, q=q, k=k, q_weight=qw, k_weight=kw, eps=eps)
    for trial in range(4):
        moved = [q, k] if what == "x" else [qw, kw]
        u = [torch.randn(m.shape, generator=g, device="cuda").sign() for m in moved]

        def loss(sign, wide):
            m = [a + sign * step * b for a, b in zip(moved, u)]
            xs, ws = (m, [qw, kw]) if what == "x" else ([q, k], m)
            if wide:
                y = [_rotate(rope, _norm(x.double().cpu(), w.double().cpu(), eps), *_turn(rope, pos)) for x, w in zip(xs, ws)]
                return sum((a * b.double().cpu()).sum() for a, b in zip(y, dy))
            y = spkv.qk_norm_rope(*xs, pos, rope, *ws, eps)
            return sum((a.double() * b.double()).sum().cpu() for a, b in zip(y, dy))

        along = sum((a.double() * b.double()).sum().cpu() for a, b in zip(got[:2] if what == "x" else got[2:], u))
        diff, wide = ((loss(1, w) - loss(-1, w)) / (2 * step) for w in (False, True))
        size = sum((_pair_size(rope, _norm(x.double().cpu(), w.double().cpu(), eps)) * b.double().cpu().abs()).sum()
                   for x, w, b in zip((q, k), (qw, kw), dy))
        rounding = 2 * 40 * U * size / (2 * step)
        assert (diff - wide).abs() <= rounding
        assert (wide - along).abs() <= (10 * step * step + 2.0 ** -18) * size


def test_captured_calls_replay():
    """A graph of both directions replayed on new inputs, with eager calls between the replays."""
    rope = _rope(128)
    t, hq, hk, d = 130, 8, 2, 128
    qkv, q, k, v, qw, kw, g = _inputs(t, hq, hk, d, torch.bfloat16)
    pos = _positions(rope, t, g)
    out = [torch.empty(t, h, d, dtype=torch.bfloat16, device="cuda") for h in (hq, hk, hk)]
    grad = torch.empty_like(qkv)
    into = (grad[:, :hq], grad[:, hq:hq + hk], grad[:, hq + hk:])
    ws = torch.empty(1024 * 2 * d * 4, dtype=torch.uint8, device="cuda")

    def both():
        spkv.qk_norm_rope(q, k, pos, rope, qw, kw, 1e-6, v=v, out=out)
        return spkv.qk_norm_rope_backward(out[0], out[1], pos, rope, q=q, k=k, q_weight=qw, k_weight=kw, eps=1e-6,
                                          dv=out[2], out=into, workspace=ws)

    both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        dw = both()
    for _ in range(4):
        qkv.copy_(torch.randn(qkv.shape, generator=g, device="cuda").bfloat16())
        pos.copy_(_positions(rope, t, g))
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in (*out, grad, *dw)]
        want_w = both()
        torch.cuda.synchronize()
        for a, b in zip(got, (*out, grad, *want_w)):
            assert torch.equal(a, b)


@pytest.mark.parametrize("dtype,d,adjacent,t", [
    (torch.bfloat16, 128, False, 14001), (torch.float32, 64, True, 14001), (torch.bfloat16, 128, False, 22003),
    (torch.float32, 64, True, 23003)], ids=["bf16", "fp32", "bf16-longer", "fp32-longer"])
def test_more_than_the_caches_hold(dtype, d, adjacent, t):
    """Calls that move more than the last cache holds take other loads, and other stores where what they write alone is more:
    the same bits as in pieces.  Weights' gradients, as sums in another order, differ by the errors of both: under 136 u of
    the products' magnitudes each."""
    hq, hk, piece = 32, 8, 2000
    rope = _rope(d, adjacent=adjacent)
    qkv, q, k, v, qw, kw, g = _inputs(t, hq, hk, d, dtype)
    dy = torch.randn(t, hq + 2 * hk, d, generator=g, device="cuda").to(dtype)
    dq, dk, dv = dy[:, :hq], dy[:, hq:hq + hk], dy[:, hq + hk:]
    pos = _positions(rope, t, g)
    norm = dict(q_weight=qw, k_weight=kw, eps=1e-6)
    whole = spkv.qk_norm_rope(q, k, pos, rope, v=v, **norm)
    back = spkv.qk_norm_rope_backward(dq, dk, pos, rope, q=q, k=k, dv=dv, **norm)
    sums = [torch.zeros(d, dtype=torch.float64, device="cuda") for _ in range(2)]
    for at in range(0, t, piece):
        s = slice(at, min(at + piece, t))
        for x, y in zip(whole, spkv.qk_norm_rope(q[s], k[s], pos[s].contiguous(), rope, v=v[s], **norm)):
            assert torch.equal(x[s], y)
        part = spkv.qk_norm_rope_backward(dq[s], dk[s], pos[s].contiguous(), rope, q=q[s], k=k[s], dv=dv[s], **norm)
        for x, y in zip(back[:3], part):
            assert torch.equal(x[s], y)
        for x, y in zip(sums, part[3:]):
            x += y
    for x, y, heads, grad in ((sums[0], back[3], q, dq), (sums[1], back[4], k, dk)):
        # |g| <= |a| + |b| of its pair: the magnitudes' sum is at least that of the products
        r = torch.rsqrt(heads.float().pow(2).mean(-1, keepdim=True) + 1e-6)
        size = (_pair_size(rope, grad.float()) * heads.float().abs() * r).double().sum((0, 1))
        assert ((x - y).abs() <= 2 * 136 * U * size).all()
