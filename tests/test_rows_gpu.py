"""Rows between the projection and the attention on the GPU, through the C ABI, against the fp64 oracle: norms per head and rotation
(tl_rotate_rows), rows written to the pool (tl_pool_write_rows), rows that move (tl_pool_move_rows), and all of it in front of
the attention.  Every value is held to the bound that oracle.rows_oracle.rows derives for it."""
import math

import numpy as np
import pytest
import torch

from oracle import rows_oracle as ro
from oracle import tokenlake_oracle as orc
from paper_2508_17219_amd import binding as B
from tests import tl_harness as H

pytestmark = pytest.mark.gpu

DEV = "cuda"
KIND = {"bf16": torch.bfloat16, "fp32": torch.float32}


def _say(msg):
    print("[case] " + msg, flush=True)


def _freqs(rot, base=1e6):
    return float(base) ** (-np.arange(0, rot, 2, dtype=np.float64) / rot)


def _rope(freqs, interleaved=False, factor=1.0):
    return B.tl_rope_of(torch.from_numpy(B.tl_rope_steps(freqs).view(np.int64)).to(DEV), interleaved, factor)


def _randn(seed, *shape, kind=torch.bfloat16):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(shape, generator=g).to(kind).to(DEV)


def _out(n, heads, guard=0):
    return torch.full((n + guard, heads, 128), float("nan"), dtype=torch.bfloat16, device=DEV)


def _np(t):
    return t.double().cpu().numpy()


def _check(got, want, tol, what):
    got = _np(got)
    assert np.array_equal(np.isnan(got), np.isnan(want)), what
    bad = ~(np.abs(got - want) <= tol) & ~np.isnan(want)
    assert not bad.any(), "%s: %d values off, first at %s: %r for %r" % (what, bad.sum(), np.argwhere(bad)[0], got[bad][0], want[bad][0])


def _weights(seed):
    return (1 + 0.3 * _randn(seed, 128, kind=torch.float32)), (1 + 0.3 * _randn(seed + 1, 128, kind=torch.float32))


@pytest.mark.parametrize("n,q_heads,kv_heads,rot,interleaved,kind,norm", [
    (1, 64, 8, 128, False, "bf16", True), (1, 1, 1, 128, True, "bf16", True), (2, 8, 2, 64, False, "bf16", False),
    (3, 7, 1, 16, False, "bf16", True), (5, 28, 4, 96, False, "fp32", True), (17, 8, 1, 112, True, "bf16", True),
    (33, 32, 8, 128, False, "bf16", True), (64, 3, 3, 32, True, "fp32", False), (100, 16, 16, 48, False, "bf16", True),
    (257, 8, 2, 128, False, "fp32", True), (9, 33, 11, 80, True, "bf16", False)])
def test_rotate_rows_every_value(n, q_heads, kv_heads, rot, interleaved, kind, norm):
    _say("rotate %d %d/%d rot %d %s %s norm %s" % (n, q_heads, kv_heads, rot, interleaved, kind, norm))
    heads, factor = q_heads + 2 * kv_heads, 1.0 if norm else 1.2
    fused = _randn(n, n, heads, 128, kind=KIND[kind]) * 3
    q, k, v = fused[:, :q_heads], fused[:, q_heads:q_heads + kv_heads], fused[:, q_heads + kv_heads:]
    before = fused.clone()
    pos = torch.from_numpy(np.random.default_rng(n).integers(0, 200000, n).astype(np.int32)).to(DEV)
    qw, kw = _weights(n) if norm else (None, None)
    qo, ko, vo = _out(n, q_heads, 1), _out(n, kv_heads, 1), _out(n, kv_heads, 1)
    freqs = _freqs(rot)
    B.tl_rotate_rows(_rope(freqs, interleaved, factor), pos, q, k, v, qo[:n], ko[:n], vo[:n], qw, kw, 1e-5)
    torch.cuda.synchronize()
    p = pos.cpu().numpy()
    for name, x, w, o in (("q", q, qw, qo), ("k", k, kw, ko)):
        want, tol = ro.rows(_np(x), p, freqs, interleaved, factor, None if w is None else _np(w), 1e-5)
        _check(o[:n], want, tol, name)
    assert torch.equal(vo[:n], v.to(torch.bfloat16))
    for o in (qo, ko, vo):
        assert torch.isnan(o[n:].float()).all()               # rows behind the last are left
    assert torch.equal(fused, before)


def test_rotate_rows_of_one_tensor_alone_norm_alone_and_copies():
    _say("parts of a call")
    n, freqs = 6, _freqs(128)
    q, k = _randn(1, n, 4, 128), _randn(2, n, 2, 128)
    pos = torch.arange(n, dtype=torch.int32, device=DEV) * 1000
    qw, kw = _weights(3)
    rope = _rope(freqs)
    want = {}
    whole = [_out(n, 4), _out(n, 2), _out(n, 2)]
    B.tl_rotate_rows(rope, pos, q, k, k, *whole, qw, kw)
    one = _out(n, 4)
    B.tl_rotate_rows(rope, pos, q, q_out=one, q_weight=qw)
    assert torch.equal(one, whole[0])
    one = _out(n, 2)
    B.tl_rotate_rows(rope, pos, k=k, k_out=one, k_weight=kw)
    assert torch.equal(one, whole[1])
    one = _out(n, 2)
    B.tl_rotate_rows(None, None, v=k, v_out=one)
    assert torch.equal(one, k)
    # no rotation: the norm alone, on the queries alone; keys go through
    qo, ko = _out(n, 4), _out(n, 2)
    B.tl_rotate_rows(None, None, q, k, None, qo, ko, None, qw, None, 1e-3)
    w, tol = ro.rows(_np(q), None, weight=_np(qw), eps=1e-3)
    _check(qo, w, tol, "norm alone")
    assert torch.equal(ko, k)
    # position 0 and a factor of 1 leave every bit
    B.tl_rotate_rows(rope, torch.zeros_like(pos), q, q_out=qo)
    assert torch.equal(qo, q)
    # no tokens
    B.tl_rotate_rows(rope, pos[:0], q[:0], q_out=qo[:0])


def test_rotate_rows_at_every_position():
    """Angles of far positions are as exact as near ones: 2^31 - 1 radians, negative positions, the ends of the range."""
    _say("far positions")
    p = np.array([0, 1, -1, 2, 1 << 24, (1 << 24) + 1, 10 ** 6 + 7, -10 ** 6, 2 ** 31 - 1, -2 ** 31, 2 ** 31 - 2, 12345678], np.int64)
    freqs = np.concatenate([_freqs(124, 1e4), [0.0, -0.5]])
    x = _randn(5, len(p), 2, 128)
    for interleaved in (False, True):
        out = _out(len(p), 2)
        B.tl_rotate_rows(_rope(freqs, interleaved), torch.from_numpy(p.astype(np.int32)).to(DEV), x, q_out=out)
        want, tol = ro.rows(_np(x), p, freqs, interleaved)
        _check(out, want, tol, "interleaved" if interleaved else "halves")


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotate_rows_angle_is_the_nearest_of_32_bits(interleaved):
    """Angles of a few 2^-32 of a turn, which a sine shows to the bit: off by 2^-33 of a turn for the phase, and by what a sine of that size is rounded
    by: half a step of bf16 (with what the first of two roundings adds), 2^-20 of it for 32 bits."""
    _say("small angles, " + ("neighbours" if interleaved else "halves"))
    parts = [0, 1, (1 << 31) - 1, 1 << 31, (1 << 31) + 1, (1 << 32) - 1]
    steps = np.array([(j << 32) + f for j in (0, 1, 2, 3, 5, 9) for f in parts] + [0] * 28, np.uint64)
    rope = B.tl_rope_of(torch.from_numpy(steps.view(np.int64)).to(DEV), interleaved)
    positions = [1, -1, 2, -3]
    x = torch.zeros(len(positions), 1, 128, device=DEV)
    (x[..., 0::2] if interleaved else x[..., :64]).fill_(1)
    out = _out(len(positions), 1)
    B.tl_rotate_rows(rope, torch.tensor(positions, dtype=torch.int32, device=DEV), x, q_out=out)
    got = _np(out)[:, 0]
    got = got[:, 1::2] if interleaved else got[:, 64:]
    turn = 2 * math.pi / 2.0 ** 32
    want = np.array(positions)[:, None] * (steps.astype(np.float64) / 2.0 ** 32)[None] * turn
    tol = 0.5 * turn + (np.abs(want) + 0.5 * turn) * (2.0 ** -8 * (1 + 2.0 ** -9) + 2.0 ** -20)
    bad = np.abs(got - want) > tol
    assert not bad.any(), (np.argwhere(bad)[0], got[bad][0] / turn, want[bad][0] / turn)


def test_rotate_rows_strides_orders_and_starts():
    """Heads in front of tokens, tokens and heads that repeat (stride 0), tensors that start between 16-byte boundaries, outputs too."""
    _say("strides")
    n, h, freqs = 13, 5, _freqs(96)
    pos = torch.arange(n, dtype=torch.int32, device=DEV) + 77
    rope = _rope(freqs)
    for kind in ("bf16", "fp32"):
        base = _randn(7, n * h * 128 + 9, kind=KIND[kind])
        views = {"heads first": base[:n * h * 128].view(h, n, 128).transpose(0, 1), "one token": base[3:3 + h * 128].view(1, h, 128).expand(n, h, 128),
                 "one head": base[1:1 + n * 128].view(n, 1, 128).expand(n, h, 128), "off by one": base[1:1 + n * h * 128].view(n, h, 128),
                 "off by seven": base[7:7 + n * h * 128].view(n, h, 128), "every other": base.new_zeros(0)}
        wide = _randn(8, 2 * n, h + 3, 128, kind=KIND[kind])
        views["every other"] = wide[::2, 1:1 + h]
        for what, x in views.items():
            want, tol = ro.rows(_np(x), pos.cpu().numpy(), freqs)
            for off in (0, 3):
                flat = torch.full((n * h * 128 + 16,), float("nan"), dtype=torch.bfloat16, device=DEV)
                out = flat[off:off + n * h * 128].view(n, h, 128)
                B.tl_rotate_rows(rope, pos, x, q_out=out)
                _check(out, want, tol, "%s %s out+%d" % (kind, what, off))
                assert torch.isnan(flat[:off].float()).all() and torch.isnan(flat[off + n * h * 128:].float()).all()


def test_rotate_rows_in_place_and_the_overlaps_that_are_refused():
    _say("in place")
    n, freqs = 50, _freqs(128)
    qw, kw = _weights(4)
    pos = torch.arange(n, dtype=torch.int32, device=DEV) * 3
    rope = _rope(freqs)
    q, k, v = _randn(1, n, 12, 128), _randn(2, n, 3, 128), _randn(3, n, 3, 128)
    want = [_out(n, 12), _out(n, 3), _out(n, 3)]
    B.tl_rotate_rows(rope, pos, q, k, v, *want, qw, kw)
    got = [q.clone(), k.clone(), v.clone()]
    B.tl_rotate_rows(rope, pos, *got, *got, qw, kw)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    buf = torch.zeros(2 * n, 12, 128, dtype=torch.bfloat16, device=DEV)
    for x, o in ((buf[:n], buf[1:n + 1]), (buf[1:n + 1], buf[:n])):
        with pytest.raises(B.TokenLakeError) as e:
            B.tl_rotate_rows(rope, pos, x, q_out=o)
        assert e.value.status == B.TL_EINVAL


def test_rotate_rows_values_out_of_the_ordinary():
    """Rows of zeros, squares beyond 32 bits, infinities and NaN: the norm's own formula, and no head disturbs another."""
    _say("extremes")
    x = _randn(9, 8, 3, 128, kind=torch.float32)
    x[0] = 0
    x[1] *= 1e25
    x[2] *= 1e-25
    x[3, 1, 5] = float("inf")
    x[4, 0, 64] = float("nan")
    x[5] = 3e38
    x[6, 2, :64] = -2e30
    w = _weights(5)[0]
    out = _out(8, 3)
    B.tl_rotate_rows(None, None, x, q_out=out, q_weight=w)
    with np.errstate(invalid="ignore"):
        want, tol = ro.rows(_np(x), None, weight=_np(w))
    finite = np.isfinite(_np(x)).all(-1)
    got = _np(out)
    assert (np.abs(got - want) <= tol)[finite].all()
    assert np.isnan(got[3, 1, 5]) and (np.delete(got[3, 1], 5) == 0).all() and np.isnan(got[4, 0]).all()
    # values keep their bits, NaN payloads among them
    bits = torch.randint(-32768, 32768, (8, 3, 128), generator=torch.Generator().manual_seed(1)).to(torch.int16).to(DEV)
    v = bits.view(torch.bfloat16)
    vo = _out(8, 3)
    B.tl_rotate_rows(None, None, v=v, v_out=vo)
    assert torch.equal(vo.view(torch.int16), bits)
    # 32-bit values all over the range, those below the normal numbers too, are rounded to the nearest, ties to even, like torch does
    for step in (345679, 2731):
        f = (torch.arange(0, 8 * 3 * 128, device=DEV, dtype=torch.int32).view(8, 3, 128) * step).view(torch.float32)
        f = torch.where(torch.isfinite(f), f, torch.zeros_like(f))
        B.tl_rotate_rows(None, None, v=f, v_out=vo)
        assert torch.equal(vo, f.to(torch.bfloat16))


@pytest.mark.parametrize("kind", ["bf16", "fp32"])
@pytest.mark.parametrize("size,eps", [(2.0 ** 62, 1e38), (1e18, 3.4e38), (1e19, 3.4028234e38), (1e25, 3e38), (3e38, 3.4e38), (1e25, 1e-6), (1e-3, 1e30),
                                      (2.0 ** -64, 2.0 ** -126), (2.0 ** -60, 2.0 ** -110), (0.0, 2.0 ** -126)])
def test_the_norm_holds_for_every_eps(size, eps, kind):
    """Any positive normal eps counts, beside squares beyond 32 bits and squares below the normal numbers too."""
    _say("norm %s of %g with eps %g" % (kind, size, eps))
    x = (_randn(17, 5, 3, 128, kind=torch.float32).clamp(-1, 1) * size).to(KIND[kind])
    w = _weights(18)[0]
    out = _out(5, 3)
    B.tl_rotate_rows(None, None, x, q_out=out, q_weight=w, eps=eps)
    want, tol = ro.rows(_np(x), None, weight=_np(w), eps=eps)
    _check(out, want, tol, "norm")


def test_rotate_rows_offsets_beyond_32_bits():
    """Tokens 2^31 values apart, and more tokens than one launch takes (their inputs one row, repeated)."""
    _say("long strides")
    far = torch.empty(2 * (1 << 31) + 256, dtype=torch.bfloat16, device=DEV).as_strided((3, 2, 128), (1 << 31, 128, 1))
    x = _randn(1, 3, 2, 128)
    far.copy_(x)
    pos = torch.tensor([5, 6, 7], dtype=torch.int32, device=DEV)
    freqs = _freqs(128)
    a, b = _out(3, 2), _out(3, 2)
    B.tl_rotate_rows(_rope(freqs), pos, far, q_out=a)
    B.tl_rotate_rows(_rope(freqs), pos, x, q_out=b)
    assert torch.equal(a, b)
    del far
    _say("many tokens")
    n = (1 << 25) + 5
    x = _randn(2, 1, 1, 128)
    pos = torch.arange(n, dtype=torch.int32, device=DEV)
    out = torch.empty((n, 1, 128), dtype=torch.bfloat16, device=DEV)
    B.tl_rotate_rows(_rope(freqs), pos, x.expand(n, 1, 128), q_out=out)
    at = torch.tensor([0, 1, (1 << 25) - 1, 1 << 25, (1 << 25) + 1, n - 1], device=DEV)
    want, tol = ro.rows(np.repeat(_np(x), len(at), 0), at.cpu().numpy(), freqs)
    _check(out[at], want, tol, "many tokens")
    again = out[-70000:].clone()
    few = torch.empty_like(again)
    B.tl_rotate_rows(_rope(freqs), pos[-70000:], x.expand(70000, 1, 128), q_out=few)
    assert torch.equal(few, again)


@pytest.mark.parametrize("mb,kind,norm", [(90, "bf16", True), (110, "bf16", True), (260, "bf16", True), (290, "fp32", False), (280, "bf16", False)])
def test_rows_of_large_calls_are_the_rows_of_small_ones(mb, kind, norm):
    """Calls on either side of what the cache behind HBM holds, whole and in place, to the bits of calls of a few hundred tokens."""
    _say("%d MB" % mb)
    q_heads, kv_heads = 9, 3
    n = mb * 1000000 // ((q_heads + 2 * kv_heads) * 128 * (4 if kind == "bf16" else 6))
    g = torch.Generator(device=DEV).manual_seed(mb)
    x = torch.randn(n, q_heads + 2 * kv_heads, 128, generator=g, device=DEV).to(KIND[kind])
    q, k, v = x[:, :q_heads], x[:, q_heads:q_heads + kv_heads], x[:, q_heads + kv_heads:]
    pos = torch.randint(0, 1 << 20, (n,), generator=g, device=DEV, dtype=torch.int32)
    qw, kw = _weights(mb) if norm else (None, None)
    rope = _rope(_freqs(128))
    outs = [torch.empty((n, h, 128), dtype=torch.bfloat16, device=DEV) for h in (q_heads, kv_heads, kv_heads)]
    B.tl_rotate_rows(rope, pos, q, k, v, *outs, qw, kw)
    for first in (0, 1000, n // 2 + 1, n - 333):
        part = slice(first, first + 333)
        few = [torch.empty((333, h, 128), dtype=torch.bfloat16, device=DEV) for h in (q_heads, kv_heads, kv_heads)]
        B.tl_rotate_rows(rope, pos[part], q[part], k[part], v[part], *few, qw, kw)
        assert all(torch.equal(a[part], b) for a, b in zip(outs, few))
    if kind == "bf16":
        again = [t.contiguous() for t in (q, k, v)]
        B.tl_rotate_rows(rope, pos, *again, *again, qw, kw)
        assert all(torch.equal(a, b) for a, b in zip(outs, again))


@pytest.mark.parametrize("n,q_heads,kv_heads", [(2, 46337, 1), (3, 50000, 1), (61, 65536, 1), (2, 1, 23200), (3, 2, 65536), (1, 65536, 65536)])
def test_rotate_rows_of_as_many_heads_as_there_may_be(n, q_heads, kv_heads):
    """Tens of thousands of heads beside few (one token's, repeated): the calls return, and every token's rows are what a call of 8 heads gives."""
    _say("%d tokens of %d/%d heads" % (n, q_heads, kv_heads))
    freqs = _freqs(128)
    rope, (qw, kw) = _rope(freqs), _weights(n)
    pos = torch.arange(n, dtype=torch.int32, device=DEV) * 1009 + 5
    few = _randn(q_heads, 8, 128)

    def spread(heads):
        return few.repeat(-(-heads // 8), 1)[:heads].view(1, heads, 128).expand(n, heads, 128)

    outs = [_out(n, q_heads), _out(n, kv_heads), _out(n, kv_heads)]
    B.tl_rotate_rows(rope, pos, spread(q_heads), spread(kv_heads), spread(kv_heads), *outs, qw, kw)
    want_q, want_k = _out(n, 8), _out(n, 8)
    eight = few.view(1, 8, 128).expand(n, 8, 128)
    B.tl_rotate_rows(rope, pos, eight, eight, None, want_q, want_k, None, qw, kw)
    for got, want, heads in zip(outs, (want_q, want_k, eight), (q_heads, kv_heads, kv_heads)):
        for first in range(8):
            part = got[:, first::8]
            assert torch.equal(part, want[:, first:first + 1].expand(part.shape))
    w, tol = ro.rows(_np(eight), pos.cpu().numpy(), freqs, weight=_np(qw))
    _check(want_q, w, tol, "queries")


def _in_parts(rope, pos, q, k, v, qw, kw, part=2000):
    """What tl_rotate_rows makes of the rows, by calls of a few tokens."""
    outs = [None if t is None else torch.empty((t.shape[0], t.shape[1], 128), dtype=torch.bfloat16, device=DEV) for t in (q, k, v)]
    for first in range(0, pos.shape[0], part):
        at = slice(first, first + part)
        B.tl_rotate_rows(rope, pos[at], *(None if t is None else t[at] for t in (q, k, v, *outs)), qw, kw)
    return outs


@pytest.mark.parametrize("rot,interleaved", [(128, False), (128, True), (96, False), (96, True), (0, False)])
@pytest.mark.parametrize("mb,kind", [(70, "fp32"), (120, "bf16"), (120, "fp32"), (290, "bf16"), (290, "fp32")])
def test_large_calls_of_every_order_are_small_ones(mb, kind, rot, interleaved):
    """Both orders of pairs, all dimensions or some, both types, on each side of what the cache keeps: to the bits of small calls, every row."""
    _say("%d MB %s rot %d %s" % (mb, kind, rot, interleaved))
    q_heads, kv_heads = 9, 3
    n = mb * 1000000 // ((q_heads + 2 * kv_heads) * 128 * (4 if kind == "bf16" else 6))
    g = torch.Generator(device=DEV).manual_seed(mb + rot)
    x = torch.randn(n, q_heads + 2 * kv_heads, 128, generator=g, device=DEV).to(KIND[kind])
    q, k, v = x[:, :q_heads], x[:, q_heads:q_heads + kv_heads], x[:, q_heads + kv_heads:]
    pos = torch.randint(0, 1 << 20, (n,), generator=g, device=DEV, dtype=torch.int32)
    qw, kw = _weights(mb)
    rope = _rope(_freqs(rot), interleaved, 1.1) if rot else None
    outs = [torch.empty((n, h, 128), dtype=torch.bfloat16, device=DEV) for h in (q_heads, kv_heads, kv_heads)]
    B.tl_rotate_rows(rope, pos, q, k, v, *outs, qw, kw)
    assert all(torch.equal(a, b) for a, b in zip(outs, _in_parts(rope, pos, q, k, v, qw, kw)))
    few = slice(n - 40, n)
    for t, w, o in ((q, qw, outs[0]), (k, kw, outs[1])):
        _check(o[few], *ro.rows(_np(t[few]), pos[few].cpu().numpy(), _freqs(rot) if rot else None, interleaved, 1.1 if rot else 1.0, _np(w)), "rows")


@pytest.mark.parametrize("kind", ["bf16", "fp32"])
def test_norms_of_rows_out_of_the_ordinary_in_both_types(kind):
    """Infinities, NaN and squares beyond 32 bits, through the sum of squares of each type; no head disturbs another."""
    _say("extremes of " + kind)
    x = _randn(19, 7, 5, 128, kind=torch.float32)
    x[1] *= 1e25
    x[2] = 3e38
    x[3, 1, 5] = float("inf")
    x[3, 2, 127] = -float("inf")
    x[4, 0, 64] = float("nan")
    x[5, 3, :64] = -2e30
    x[6, 4, 3], x[6, 4, 70] = float("inf"), float("nan")
    x = x.to(KIND[kind])
    w = _weights(20)[0]
    out = _out(7, 5)
    B.tl_rotate_rows(None, None, x, q_out=out, q_weight=w, eps=1e-6)
    with np.errstate(invalid="ignore"):
        want, tol = ro.rows(_np(x), None, weight=_np(w), eps=1e-6)
    got, finite = _np(out), np.isfinite(_np(x)).all(-1)
    assert finite.sum() == 7 * 5 - 4 and (np.abs(got - want) <= tol)[finite].all()
    for token, head, at in ((3, 1, 5), (3, 2, 127)):
        assert np.isnan(got[token, head, at]) and (np.delete(got[token, head], at) == 0).all()
    assert np.isnan(got[4, 0]).all() and np.isnan(got[6, 4]).all()


def test_rotate_rows_in_several_launches():
    """16384 heads beside one: 112 tokens to a launch.  Three launches, the tokens on both sides of each border, queries, keys and values."""
    _say("several launches")
    n, q_heads, freqs = 250, 16384, _freqs(128)
    rope, (qw, kw) = _rope(freqs), _weights(21)
    pos = torch.arange(n, dtype=torch.int32, device=DEV) * 77 - 500
    heads = torch.arange(q_heads, device=DEV) % 5
    few = _randn(22, n, 5, 128)
    q, k, v = _randn(23, 1, 5, 128)[:, heads].expand(n, q_heads, 128), few[:, :1], few[:, 1:2]
    outs = [_out(n, q_heads, 1), _out(n, 1, 1), _out(n, 1, 1)]
    B.tl_rotate_rows(rope, pos, q, k, v, *(o[:n] for o in outs), qw, kw)
    want = _in_parts(rope, pos, _randn(23, 1, 5, 128).expand(n, 5, 128), k, v, qw, kw, part=7)
    assert all(torch.equal(outs[0][at, :], want[0][at][heads]) for at in range(n))
    assert torch.equal(outs[1][:n], want[1]) and torch.equal(outs[2][:n], v)
    assert all(torch.isnan(o[n:].float()).all() for o in outs)
    _check(want[0], *ro.rows(_np(_randn(23, 1, 5, 128).expand(n, 5, 128)), pos.cpu().numpy(), freqs, weight=_np(qw)), "queries")


# ---- the pool -----------------------------------------------------------------------------
def _pool(n_slots, seg_len, kv_heads, seed=11):
    k, v = _randn(seed, n_slots, seg_len, kv_heads, 128), _randn(seed + 1, n_slots, seg_len, kv_heads, 128)
    return B.tl_pool_create(n_slots, seg_len, kv_heads, 128, k, v), k, v


@pytest.mark.parametrize("n,q_heads,kv_heads,rot,interleaved,kind,norm,dense", [
    (1, 8, 1, 128, False, "bf16", True, False), (16, 64, 8, 128, False, "bf16", True, True), (77, 0, 2, 64, True, "fp32", True, False),
    (130, 6, 3, 96, False, "bf16", False, True), (200, 4, 4, 0, False, "fp32", False, False)])
def test_write_rows_is_rotate_rows_at_the_reserved_places(n, q_heads, kv_heads, rot, interleaved, kind, norm, dense):
    _say("write %d %d/%d" % (n, q_heads, kv_heads))
    C = 64
    pool, pk, pv = _pool(12, C, kv_heads)
    B.tl_pool_adopt(pool, [1, 2], [7, 3], [C, 50])
    counts = [n - n // 3, n // 3]
    need = [-(-max(0, counts[0] - 14) // C), -(-counts[1] // C)]
    _, rows = B.tl_pool_reserve_batch(pool, [2, None], [list(range(10, 10 + need[0])), list(range(20, 20 + need[1]))], counts)
    rows = torch.from_numpy(rows).to(DEV)
    fused = _randn(n, n, q_heads + 2 * kv_heads, 128, kind=KIND[kind])
    q, k, v = (fused[:, a:b] for a, b in ((0, q_heads), (q_heads, q_heads + kv_heads), (q_heads + kv_heads, q_heads + 2 * kv_heads)))
    pos = torch.arange(n, dtype=torch.int32, device=DEV) * 31
    qw, kw = _weights(n) if norm else (None, None)
    rope = _rope(_freqs(rot), interleaved) if rot else None
    q = q if q_heads else None
    qo, ko, vo = (_out(n, q_heads) if q_heads else None), _out(n, kv_heads), _out(n, kv_heads)
    B.tl_rotate_rows(rope, pos, q, k, v, qo, ko, vo, qw, kw)
    want_k, want_v = pk.clone(), pv.clone()
    want_k.view(-1, kv_heads, 128)[rows.long()] = ko
    want_v.view(-1, kv_heads, 128)[rows.long()] = vo
    outs = [_out(n, q_heads) if q_heads else None] + ([_out(n, kv_heads), _out(n, kv_heads)] if dense else [None, None])
    B.tl_pool_write_rows(pool, rope, pos, rows, k, v, q, *outs, qw, kw)
    torch.cuda.synchronize()
    assert torch.equal(pk, want_k) and torch.equal(pv, want_v)           # the rows, and nothing but them
    for a, b in zip(outs, (qo, ko, vo)):
        assert a is None or torch.equal(a, b)
    B.tl_pool_destroy(pool)


def test_write_rows_of_a_padded_batch():
    """Rows outside the pool are not written, whatever they are; their outputs are."""
    _say("padded batch")
    C, n_slots, hkv = 64, 3, 2
    pool, pk, pv = _pool(n_slots, C, hkv)
    rows = torch.tensor([5, -1, 191, 192, 2 ** 31 - 1, -2 ** 31, 64], dtype=torch.int32, device=DEV)
    n = len(rows)
    k, v, q = _randn(1, n, hkv, 128), _randn(2, n, hkv, 128), _randn(3, n, 4, 128)
    pos = torch.arange(n, dtype=torch.int32, device=DEV)
    rope = _rope(_freqs(128))
    qo, ko, vo = _out(n, 4), _out(n, hkv), _out(n, hkv)
    B.tl_rotate_rows(rope, pos, q, k, v, qo, ko, vo)
    want_k, want_v = pk.clone(), pv.clone()
    keep = torch.tensor([0, 2, 6], device=DEV)
    want_k.view(-1, hkv, 128)[rows[keep].long()], want_v.view(-1, hkv, 128)[rows[keep].long()] = ko[keep], vo[keep]
    got = _out(n, 4)
    B.tl_pool_write_rows(pool, rope, pos, rows, k, v, q, got)
    assert torch.equal(pk, want_k) and torch.equal(pv, want_v) and torch.equal(got, qo)
    with pytest.raises(B.TokenLakeError):
        B.tl_pool_write_rows(pool, rope, pos[:3], rows[:3], pk.view(-1, hkv, 128)[:3], v[:3])     # rows of the pool itself
    B.tl_pool_destroy(pool)


def test_write_and_move_in_a_pool_beyond_32_bits():
    """Slots 4 GiB and more into the pool."""
    _say("large pool")
    C, hkv, n_slots = 512, 8, 4200                     # 2.2e9 values each of keys and values
    k_pool = torch.zeros((n_slots, C, hkv, 128), dtype=torch.bfloat16, device=DEV)
    v_pool = torch.zeros_like(k_pool)
    pool = B.tl_pool_create(n_slots, C, hkv, 128, k_pool, v_pool)
    rows = torch.tensor([n_slots * C - 1, 4100 * C + 3, 17], dtype=torch.int32, device=DEV)
    k, v = _randn(1, 3, hkv, 128), _randn(2, 3, hkv, 128)
    rope, pos = _rope(_freqs(128)), torch.tensor([9, 10, 11], dtype=torch.int32, device=DEV)
    ko, vo = _out(3, hkv), _out(3, hkv)
    B.tl_rotate_rows(rope, pos, None, k, v, None, ko, vo)
    B.tl_pool_write_rows(pool, rope, pos, rows, k, v)
    flat_k, flat_v = k_pool.view(-1, hkv, 128), v_pool.view(-1, hkv, 128)
    assert torch.equal(flat_k[rows.long()], ko) and torch.equal(flat_v[rows.long()], vo)
    dst = torch.tensor([18, n_slots * C - 2, 4100 * C + 5], dtype=torch.int32, device=DEV)
    B.tl_pool_move_rows(pool, None, rows, dst)
    assert torch.equal(flat_k[dst.long()], ko) and torch.equal(flat_v[dst.long()], vo)
    assert int((flat_v != 0).any(-1).any(-1).sum()) == 6
    B.tl_pool_destroy(pool)


@pytest.mark.parametrize("n,kv_heads,rot,interleaved", [(1, 1, 128, False), (50, 8, 128, True), (333, 3, 64, False), (700, 5, 96, True)])
def test_move_rows_turns_keys_and_copies_values(n, kv_heads, rot, interleaved):
    _say("move %d rows of %d heads" % (n, kv_heads))
    C, n_slots = 64, 40
    pool, pk, pv = _pool(n_slots, C, kv_heads)
    rng = np.random.default_rng(n)
    places = rng.permutation(n_slots * C)
    src, dst = places[:n].astype(np.int32), places[n:2 * n].astype(np.int32)
    shift = rng.integers(-100000, 100000, n).astype(np.int32)
    shift[0] = 0
    in_place = rng.random(n) < 0.2
    dst = np.where(in_place, src, dst).astype(np.int32)
    freqs = _freqs(rot)
    k0, v0 = pk.clone(), pv.clone()
    B.tl_pool_move_rows(pool, _rope(freqs, interleaved, 1.5), *(torch.from_numpy(a).to(DEV) for a in (src, dst, shift)))
    torch.cuda.synchronize()
    flat = lambda t: t.view(-1, kv_heads, 128)  # noqa: E731
    want, tol = ro.rows(_np(flat(k0)[torch.from_numpy(src).long().to(DEV)]), shift, freqs, interleaved)
    _check(flat(pk)[torch.from_numpy(dst).long().to(DEV)], want, tol, "keys")
    assert torch.equal(flat(pk)[dst[0].item()], flat(k0)[src[0].item()])           # by nothing: as it was
    want_v = flat(v0).clone()
    want_v[torch.from_numpy(dst).long().to(DEV)] = flat(v0)[torch.from_numpy(src).long().to(DEV)]
    assert torch.equal(flat(pv), want_v)
    rest = torch.ones(n_slots * C, dtype=torch.bool, device=DEV)
    rest[torch.from_numpy(dst).long().to(DEV)] = False
    assert torch.equal(flat(pk)[rest], flat(k0)[rest])
    # entries outside the pool are left out
    k0 = pk.clone()
    bad = torch.tensor([-1, 0, n_slots * C, 1], dtype=torch.int32, device=DEV)
    to = torch.tensor([0, -1, 1, n_slots * C], dtype=torch.int32, device=DEV)
    B.tl_pool_move_rows(pool, _rope(freqs), bad, to, torch.ones_like(bad))
    B.tl_pool_move_rows(pool, _rope(freqs), bad[:0], to[:0], bad[:0])
    assert torch.equal(pk, k0)
    B.tl_pool_destroy(pool)


@pytest.mark.parametrize("kv_heads,seg_len,n", [(8, 64, 20000), (8, 256, 33001), (2, 512, 140001)])
def test_moves_of_many_rows_are_moves_of_a_few(kv_heads, seg_len, n):
    """The same on either side of the cache's size; rows of a large move in the order of the slots and scattered."""
    _say("move %d rows" % n)
    n_slots = 2 * n // seg_len + 2
    g = torch.Generator(device=DEV).manual_seed(n)
    pk, pv = (torch.randn(n_slots, seg_len, kv_heads, 128, generator=g, device=DEV).bfloat16() for _ in "kv")
    k0, v0 = pk.clone(), pv.clone()
    pool = B.tl_pool_create(n_slots, seg_len, kv_heads, 128, pk, pv)
    order = torch.randperm(n_slots * seg_len, generator=g, device=DEV).to(torch.int32)
    src, dst = order[:n].contiguous(), order[n:2 * n].sort().values
    shift = torch.randint(-5000, 5000, (n,), generator=g, device=DEV, dtype=torch.int32)
    rope = _rope(_freqs(128))
    B.tl_pool_move_rows(pool, rope, src, dst, shift)
    big_k, big_v = pk.clone(), pv.clone()
    pk.copy_(k0), pv.copy_(v0)
    for first in range(0, n, n // 3 + 1):
        part = slice(first, min(n, first + n // 3 + 1))
        B.tl_pool_move_rows(pool, rope, src[part], dst[part], shift[part])
    assert torch.equal(pk, big_k) and torch.equal(pv, big_v)
    at = torch.tensor([0, 1, n // 2, n - 1], device=DEV)
    flat = pk.view(-1, kv_heads, 128)
    want, tol = ro.rows(_np(k0.view(-1, kv_heads, 128)[src[at].long()]), shift[at].cpu().numpy(), _freqs(128))
    _check(flat[dst[at].long()], want, tol, "keys")
    assert torch.equal(pv.view(-1, kv_heads, 128)[dst.long()], v0.view(-1, kv_heads, 128)[src.long()])
    B.tl_pool_destroy(pool)


@pytest.mark.parametrize("mb,kind,rot,interleaved,queries,dense", [
    (60, "bf16", 96, False, True, True), (120, "bf16", 128, False, True, False), (120, "bf16", 64, True, False, True), (120, "fp32", 96, False, True, True),
    (120, "fp32", 128, True, False, False), (300, "bf16", 96, False, True, True), (300, "bf16", 128, True, True, False), (300, "fp32", 128, False, False, True),
    (300, "fp32", 64, True, True, True)])
def test_large_writes_are_rotated_rows_at_their_places(mb, kind, rot, interleaved, queries, dense):
    """Writes on each side of what the cache keeps: the pool's rows, all of them, and the outputs to the bits of small calls of tl_rotate_rows."""
    _say("write %d MB %s rot %d %s" % (mb, kind, rot, interleaved))
    q_heads, kv_heads, C = (5 if queries else 0), 3, 64
    size = 2 if kind == "bf16" else 4
    n = mb * 1000000 // (128 * (q_heads * (size + 2) + 2 * kv_heads * (size + 2 + (2 if dense else 0)))) + 1
    g = torch.Generator(device=DEV).manual_seed(mb + rot)
    x = torch.randn(n, q_heads + 2 * kv_heads, 128, generator=g, device=DEV).to(KIND[kind])
    q, k, v = x[:, :q_heads] if queries else None, x[:, q_heads:q_heads + kv_heads], x[:, q_heads + kv_heads:]
    pos = torch.randint(0, 1 << 20, (n,), generator=g, device=DEV, dtype=torch.int32)
    qw, kw = _weights(mb)
    rope = _rope(_freqs(rot), interleaved)
    n_slots = n // C + 3
    pk, pv = (torch.randn(n_slots, C, kv_heads, 128, generator=g, device=DEV, dtype=torch.bfloat16) for _ in "kv")
    rows = torch.randperm(n_slots * C, generator=g, device=DEV)[:n].to(torch.int32)
    rows[5] = -1
    want_q, want_k, want_v = _in_parts(rope, pos, q, k, v, qw if queries else None, kw)
    want_pk, want_pv = pk.clone(), pv.clone()
    there = rows >= 0
    want_pk.view(-1, kv_heads, 128)[rows[there].long()], want_pv.view(-1, kv_heads, 128)[rows[there].long()] = want_k[there], want_v[there]
    pool = B.tl_pool_create(n_slots, C, kv_heads, 128, pk, pv)
    outs = [_out(n, q_heads) if queries else None] + ([_out(n, kv_heads), _out(n, kv_heads)] if dense else [None, None])
    B.tl_pool_write_rows(pool, rope, pos, rows, k, v, q, *outs, qw if queries else None, kw)
    torch.cuda.synchronize()
    assert torch.equal(pk, want_pk) and torch.equal(pv, want_pv)
    assert all(a is None or torch.equal(a, b) for a, b in zip(outs, (want_q, want_k, want_v)))
    B.tl_pool_destroy(pool)


@pytest.mark.parametrize("n,rot,interleaved", [(20000, 64, False), (20000, 128, True), (33001, 64, False), (33001, 96, True), (33001, 112, False), (33001, 0, False)])
def test_large_moves_of_every_order_are_moves_of_a_few(n, rot, interleaved):
    """Some dimensions and neighbouring pairs on both sides of the cache's size, a part of the rows in place."""
    _say("move %d rows rot %d %s" % (n, rot, interleaved))
    kv_heads, C = 8, 64
    n_slots = 2 * n // C + 2
    g = torch.Generator(device=DEV).manual_seed(n + rot)
    pk, pv = (torch.randn(n_slots, C, kv_heads, 128, generator=g, device=DEV, dtype=torch.bfloat16) for _ in "kv")
    k0, v0 = pk.clone(), pv.clone()
    pool = B.tl_pool_create(n_slots, C, kv_heads, 128, pk, pv)
    order = torch.randperm(n_slots * C, generator=g, device=DEV).to(torch.int32)
    src, dst = order[:n].contiguous(), order[n:2 * n].contiguous()
    dst[::7] = src[::7]
    shift = torch.randint(-5000, 5000, (n,), generator=g, device=DEV, dtype=torch.int32) if rot else None
    rope = _rope(_freqs(rot), interleaved) if rot else None
    B.tl_pool_move_rows(pool, rope, src, dst, shift)
    big_k, big_v = pk.clone(), pv.clone()
    pk.copy_(k0), pv.copy_(v0)
    for first in range(0, n, 1000):
        part = slice(first, first + 1000)
        B.tl_pool_move_rows(pool, rope, src[part], dst[part], None if shift is None else shift[part])
    assert torch.equal(pk, big_k) and torch.equal(pv, big_v)
    flat = lambda t: t.view(-1, kv_heads, 128)  # noqa: E731
    at = torch.tensor([0, 1, 7, n // 2, n - 1], device=DEV)
    want, tol = ro.rows(_np(flat(k0)[src[at].long()]), np.zeros(5) if shift is None else shift[at].cpu().numpy(), _freqs(rot) if rot else None, interleaved)
    _check(flat(pk)[dst[at].long()], want, tol, "keys")
    assert torch.equal(flat(pv)[dst.long()], flat(v0)[src.long()])
    B.tl_pool_destroy(pool)


def test_writes_and_moves_in_several_launches():
    """A pool of 32768 heads: 63 tokens to a launch.  70 rows are written and moved, and those of neighbouring places stay."""
    _say("several launches to the pool")
    kv_heads, C, n = 32768, 64, 70
    freqs = _freqs(128)
    rope, kw = _rope(freqs), _weights(24)[1]
    pk = torch.zeros(3, C, kv_heads, 128, dtype=torch.bfloat16, device=DEV)
    pv = torch.zeros_like(pk)
    pool = B.tl_pool_create(3, C, kv_heads, 128, pk, pv)
    flat_k, flat_v = pk.view(-1, kv_heads, 128), pv.view(-1, kv_heads, 128)
    heads = torch.arange(kv_heads, device=DEV) % 5
    one_k, one_v = _randn(25, 1, 5, 128), _randn(26, 1, 5, 128)
    pos, rows = torch.arange(n, dtype=torch.int32, device=DEV) * 13, torch.arange(n, dtype=torch.int32, device=DEV) + 1
    rows[64] = -1
    B.tl_pool_write_rows(pool, rope, pos, rows, one_k[:, heads].expand(n, kv_heads, 128), one_v[:, heads].expand(n, kv_heads, 128), k_weight=kw)
    want = _in_parts(rope, pos, None, one_k.expand(n, 5, 128), None, None, kw)[1]
    for i in range(n):
        if i != 64:
            assert torch.equal(flat_k[i + 1], want[i][heads]) and torch.equal(flat_v[i + 1], one_v[0][heads]), i
    assert not flat_k[0].any() and not flat_k[65].any() and not flat_k[n + 1:].any() and not flat_v[65].any()
    # to places behind them, the last row in place
    src = torch.arange(n, dtype=torch.int32, device=DEV) + 1
    dst = torch.arange(n, dtype=torch.int32, device=DEV) + 100
    dst[69] = src[69]
    B.tl_pool_move_rows(pool, rope, src, dst, torch.full_like(src, 1000))
    turned = _in_parts(rope, torch.full_like(src, 1000), None, want, None, None, None)[1]
    for i in (0, 1, 61, 62, 63, 65, 68, 69):
        assert torch.equal(flat_k[dst[i].long()], turned[i][heads]) and torch.equal(flat_v[dst[i].long()], one_v[0][heads]), i
    assert not flat_k[164].any() and not flat_k[0].any() and not flat_v[99].any()
    B.tl_pool_destroy(pool)


# ---- streams, graphs ----------------------------------------------------------------------
def test_rows_on_another_stream_and_in_a_graph():
    """One call captured with its positions, rows and places in buffers that change between replays, two graphs over the same
    operands, eager work in between; and the same calls on a stream of their own."""
    _say("streams and graphs")
    C, hkv, hq, n = 64, 2, 8, 21
    pool, pk, pv = _pool(8, C, hkv)
    rope = _rope(_freqs(128))
    qw, kw = _weights(1)
    x = _randn(1, n, hq + 2 * hkv, 128)
    q, k, v = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]
    pos, rows = torch.zeros(n, dtype=torch.int32, device=DEV), torch.arange(n, dtype=torch.int32, device=DEV)
    dst, shift = rows + 6 * C, torch.full((n,), -40, dtype=torch.int32, device=DEV)
    qo, go = _out(n, hq), _out(n, hq)

    def step(out):
        B.tl_pool_write_rows(pool, rope, pos, rows, k, v, q, out, None, None, qw, kw)
        B.tl_pool_move_rows(pool, rope, rows, dst, shift)

    step(qo)
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for g in graphs:
        with torch.cuda.graph(g):
            step(go)
    for turn in range(4):
        new = _randn(100 + turn, n, hq + 2 * hkv, 128)
        x.copy_(new)
        pos.fill_(1000 * turn + 3)
        rows.copy_(torch.randperm(5 * C, generator=torch.Generator().manual_seed(turn))[:n].to(torch.int32))
        pk.zero_(), pv.zero_()
        graphs[turn % 2].replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (pk, pv, go)]
        pk.zero_(), pv.zero_(), go.zero_()
        step(go)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (pk, pv, go)))
    # the same on another stream, in order behind what that stream does
    want = [t.clone() for t in (pk, pv, go)]
    pk.zero_(), pv.zero_(), go.zero_()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        torch.cuda._sleep(1000000)
        step(go)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, (pk, pv, go)))
    pk.zero_(), pv.zero_(), go.zero_()
    torch.cuda.synchronize()
    B.tl_pool_write_rows(pool, rope, pos, rows, k, v, q, go, None, None, qw, kw, stream=side.cuda_stream)
    B.tl_pool_move_rows(pool, rope, rows, dst, shift, stream=side.cuda_stream)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, (pk, pv, go)))
    B.tl_pool_destroy(pool)


def test_binding_refuses_shapes_and_kinds():
    _say("refusals on the device")
    n = 4
    q, k = _randn(1, n, 4, 128), _randn(2, n, 2, 128)
    pos = torch.arange(n, dtype=torch.int32, device=DEV)
    rope, w = _rope(_freqs(128)), _weights(1)[0]
    qo, ko = _out(n, 4), _out(n, 2)
    for bad in (dict(q=q.half(), q_out=qo), dict(q=q, q_out=qo.float()), dict(q=q, k=k.float(), q_out=qo, k_out=ko), dict(q=q, q_out=qo, q_weight=w.bfloat16())):
        with pytest.raises(TypeError):
            B.tl_rotate_rows(rope, pos, **bad)
    with pytest.raises(TypeError):
        B.tl_rotate_rows(rope, pos.long(), q, q_out=qo)
    for bad in (dict(q=q[..., :64], q_out=qo), dict(q=q.flatten(1), q_out=qo), dict(q=q.transpose(1, 2), q_out=qo), dict(q=q, q_out=qo[:2]),
                dict(q=q, q_out=ko), dict(q=q, q_out=_out(n, 8)[:, :4]), dict(q=q[:0], k=k, q_out=qo[:0], k_out=ko), dict(q=q, k=k[:0], q_out=qo, k_out=ko[:0]), dict(q=q, k=k[:3], q_out=qo, k_out=ko), dict(q=q, q_out=qo, q_weight=w[:64]),
                dict(k=k, v=q, k_out=ko, v_out=qo), dict(q=q.cpu(), q_out=qo), dict(q=q, q_out=qo.cpu()),
                dict(q=torch.zeros(n, 4, 256, dtype=torch.bfloat16, device=DEV)[..., ::2], q_out=qo)):
        with pytest.raises(ValueError):
            B.tl_rotate_rows(rope, pos, **bad)
    for bad in (pos[:3], pos.cpu(), torch.arange(2 * n, dtype=torch.int32, device=DEV)[::2]):
        with pytest.raises(ValueError):
            B.tl_rotate_rows(rope, bad, q, q_out=qo)
    with pytest.raises(B.TokenLakeError):
        B.tl_rotate_rows(rope, None, q, q_out=qo)
    # dense tensors of any shape will do where only the elements count
    flat = torch.empty(n, 4 * 128, dtype=torch.bfloat16, device=DEV)
    B.tl_rotate_rows(rope, pos.view(1, n), q, q_out=flat)
    B.tl_rotate_rows(rope, pos, q, q_out=qo)
    assert torch.equal(flat.view(n, 4, 128), qo)
    pool, pk, pv = _pool(3, 64, 2)
    with pytest.raises(B.TokenLakeError):
        B.tl_pool_write_rows(pool, rope, pos, pos, q, q)             # 4 heads into a pool of 2
    with pytest.raises(ValueError):
        B.tl_pool_write_rows(pool, rope, pos, pos[:2], k, k)
    for bad in ((pos, pos[:2], pos), (pos[:2], pos, pos), (pos, pos, pos[:2]),
                (pos, pos.cpu(), pos), (torch.arange(8, dtype=torch.int32, device=DEV)[::2], pos, pos)):
        with pytest.raises(ValueError):
            B.tl_pool_move_rows(pool, rope, *bad)
    with pytest.raises(TypeError):
        B.tl_pool_move_rows(pool, rope, pos, pos.long(), pos)
    with pytest.raises(B.TokenLakeError):
        B.tl_pool_move_rows(pool, rope, pos, pos)
    B.tl_pool_destroy(pool)


def test_outputs_are_filled_in_the_order_that_their_shape_says():
    """An output of another order ([heads, n, 128]: heads in front of tokens) is refused, each of the three; other shapes with the same order get the same bits."""
    _say("orders of outputs")
    n, hq, hkv = 10, 4, 2
    q, k, v = _randn(1, n, hq, 128), _randn(2, n, hkv, 128), _randn(3, n, hkv, 128)
    rope, pos = _rope(_freqs(128)), torch.arange(n, dtype=torch.int32, device=DEV)
    want = [_out(n, hq), _out(n, hkv), _out(n, hkv)]
    B.tl_rotate_rows(rope, pos, q, k, v, *want)
    pool, pk, pv = _pool(2, 64, hkv)
    for which, heads in enumerate((hq, hkv, hkv)):
        for shape in ((heads, n, 128), (n, 128, heads), (heads, n * 128)):
            outs = [_out(n, hq), _out(n, hkv), _out(n, hkv)]
            outs[which] = torch.zeros(shape, dtype=torch.bfloat16, device=DEV)
            with pytest.raises(ValueError, match="qkv"[which] + "_out"):
                B.tl_rotate_rows(rope, pos, q, k, v, *outs)
            with pytest.raises(ValueError, match="qkv"[which] + "_out"):
                B.tl_pool_write_rows(pool, rope, pos, pos, k, v, q, *outs)
        for shape in ((n, heads * 128), (1, n, heads * 128), (2, n // 2, heads, 128), (n * heads, 128), (n * heads * 128,)):
            outs = [_out(n, hq), _out(n, hkv), _out(n, hkv)]
            outs[which] = outs[which].view(shape)
            B.tl_rotate_rows(rope, pos, q, k, v, *outs)
            assert all(torch.equal(a.view(b.shape), b) for a, b in zip(outs, want))
    B.tl_pool_destroy(pool)


# ---- together, in front of the attention ---------------------------------------------------
class _Model:
    """A layer's projections of sessions, and the norms and rotation that the oracle holds their rows to."""

    def __init__(self, hq, hkv, seed):
        self.hq, self.hkv, self.seed = hq, hkv, seed
        self.freqs = _freqs(128, 1e4)
        self.qw, self.kw = _weights(seed)
        self.rope = _rope(self.freqs)

    def raw(self, session, first, n):
        g = torch.Generator().manual_seed(self.seed * 1000003 + session * 100003 + first)
        return torch.randn(n, self.hq + 2 * self.hkv, 128, generator=g).to(torch.bfloat16)

    def check(self, raw, pos, q, k, v):
        """Queries, keys and values as the attention reads them, each value against the oracle."""
        x, hq, hkv = raw.double().numpy(), self.hq, self.hkv
        _check(q, *ro.rows(x[:, :hq], pos, self.freqs, weight=_np(self.qw)), "queries")
        _check(k, *ro.rows(x[:, hq:hq + hkv], pos, self.freqs, weight=_np(self.kw)), "keys")
        assert np.array_equal(_np(v), x[:, hq + hkv:])


def _bits(t):
    return t.contiguous().view(torch.int16).cpu().numpy().view(np.uint16)


def test_sessions_prefill_decode_and_move_with_rows_from_the_projection():
    """Sessions as a server runs them, from the projection's rows on: a chunk's queries, keys and values go through
    tl_pool_write_rows (queries and the self block's keys and values dense, rows to the reserved places), the attention reads them; tokens
    are decoded with their own key in the pool already; then the first session's beginning is dropped, its rest moves to
    the front, keys turned back, and it goes on.  Every value that the attention reads is held to the oracle's of the raw
    rows, and its result to the oracle's attention over what it read."""
    _say("sessions from projection to attention")
    hq, hkv, C, n_slots = 8, 2, 64, 40
    m = _Model(hq, hkv, 7)
    pk = torch.full((n_slots, C, hkv, 128), float("nan"), dtype=torch.bfloat16, device=DEV)
    pv = torch.full_like(pk, float("nan"))
    pool = B.tl_pool_create(n_slots, C, hkv, 128, pk, pv)
    scale = 1 / math.sqrt(128)
    S = 3
    chain, total, hist = [[] for _ in range(S)], [0] * S, [(np.zeros((0, hkv, 128), np.uint16),) * 2 for _ in range(S)]
    nid = [100]

    def reserve(counts):
        tails, ids = [], []
        for s in range(S):
            tail = chain[s][-1] if total[s] % C else None
            need = -(-max(0, counts[s] - (C - total[s] % C if tail is not None else 0)) // C)
            tails.append(tail), ids.append(list(range(nid[0], nid[0] + need)))
            nid[0] += need
        _, rows = B.tl_pool_reserve_batch(pool, tails, ids, counts)
        for s in range(S):
            chain[s] += ids[s]
        return torch.from_numpy(rows).to(DEV)

    def ptr(xs):
        return np.concatenate([[0], np.cumsum(xs)]).astype(np.int32)

    def attend(plan, q, kn, vn, causal):
        info = B.tl_plan_get_info(plan)
        part = torch.full((max(1, info.n_partial_rows), hq, 128), float("nan"), device=DEV)
        lsep = torch.full((max(1, info.n_partial_rows), hq), float("nan"), device=DEV)
        out, lse = torch.full((info.n_tokens, hq, 128), float("nan"), device=DEV), torch.full((info.n_tokens, hq), float("nan"), device=DEV)
        B.tl_segment_attn(pool, plan, q, scale, part, lsep)
        if causal:
            B.tl_causal_block(plan, q, kn, vn, scale, part, lsep)
        B.tl_merge(plan, part, lsep, out, False, lse)
        torch.cuda.synchronize()
        B.tl_plan_destroy(plan)
        return out, lse

    def turn(counts, own_key_in_pool):
        raw = [m.raw(s, total[s], counts[s]) for s in range(S)]
        x = torch.cat(raw).to(DEV)
        n = x.shape[0]
        at = [total[s] + np.arange(counts[s]) for s in range(S)]
        pos = torch.from_numpy(np.concatenate(at).astype(np.int32)).to(DEV)
        q, k, v = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]
        qo, ko, vo = _out(n, hq), _out(n, hkv), _out(n, hkv)
        if own_key_in_pool:        # decode: the row goes to the pool first, no self block
            rows = reserve(counts)
            plan = B.tl_plan_create(pool, hq, ptr(counts), ptr([len(c) for c in chain]), np.array(sum(chain, []), np.uint64), 0)
            B.tl_pool_write_rows(pool, m.rope, pos, rows, k, v, q, qo, None, None, m.qw, m.kw)
            out, lse = attend(plan, qo, None, None, False)
        else:                      # a chunk: attention over what was there, the self block, and the rows to the pool for later
            plan = B.tl_plan_create(pool, hq, ptr(counts), ptr([len(c) for c in chain]), np.array(sum(chain, []), np.uint64))
            B.tl_rotate_rows(m.rope, pos, q, k, v, qo, ko, vo, m.qw, m.kw)
            out, lse = attend(plan, qo, ko, vo, True)
            rows = reserve(counts)
            B.tl_pool_write_rows(pool, m.rope, pos, rows, k, v, None, None, None, None, None, m.kw)
        flat_k, flat_v = (p.view(-1, hkv, 128)[rows.long()] for p in (pk, pv))
        m.check(torch.cat(raw), pos.cpu().numpy(), qo, flat_k, flat_v)
        if not own_key_in_pool:
            assert torch.equal(ko, flat_k) and torch.equal(vo, flat_v)
        qb, kb, vb = _bits(qo), _bits(flat_k), _bits(flat_v)
        t0 = 0
        for s in range(S):
            t1, past = t0 + counts[s], hist[s][0].shape[0]
            hist[s] = tuple(np.concatenate([a, b[t0:t1]]) for a, b in zip(hist[s], (kb, vb)))
            if counts[s]:
                want_o, want_l = orc.partial_attention(qb[t0:t1], hist[s][0], hist[s][1], scale, n_visible=past + np.arange(counts[s]) + 1)
                assert np.abs(_np(out[t0:t1]) - want_o).max() <= H.TOL_O, s
                assert np.abs(_np(lse[t0:t1]) - want_l).max() <= H.TOL_LSE, s
            t0 = t1
            total[s] += counts[s]

    turn([150, 64, 3], False)
    turn([40, 0, 90], False)
    for _ in range(3):
        turn([1, 1, 1], True)
    turn([5, 70, 1], False)
    # session 0 drops its first 100 tokens: the rest goes to new segments, its keys 100 positions earlier
    drop, keep = 100, total[0] - 100
    slots = B.tl_pool_lookup(pool, chain[0])
    old = (slots[:, None] * C + np.arange(C)).reshape(-1)[drop:drop + keep].astype(np.int32)
    ids = list(range(nid[0], nid[0] + -(-keep // C)))
    nid[0] += len(ids)
    _, new = B.tl_pool_reserve_batch(pool, [None], [ids], [keep])
    B.tl_pool_move_rows(pool, m.rope, torch.from_numpy(old).to(DEV), torch.from_numpy(new).to(DEV), torch.full((keep,), -drop, dtype=torch.int32, device=DEV))
    for i in chain[0]:
        B.tl_pool_release(pool, i)
        B.tl_pool_evict_lru(pool)
    k_old, v_old = hist[0]
    flat = pk.view(-1, hkv, 128)[torch.from_numpy(new).long().to(DEV)]
    _check(flat, *ro.rows(orc.bf16_bits_to_f64(k_old[drop:]), np.full(keep, -drop), m.freqs), "moved keys")
    hist[0] = (_bits(flat), v_old[drop:])
    chain[0], total[0] = ids, keep
    for _ in range(2):
        turn([1, 1, 1], True)
    turn([70, 2, 0], False)
    B.tl_pool_destroy(pool)
