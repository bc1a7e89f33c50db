"""Rows between the projection and the attention, what a CPU can check: the steps of the rotation, the places that
tl_pool_reserve_batch gives, and the calls that are refused (no call here launches anything)."""
import ctypes as C
from decimal import Decimal, getcontext

import numpy as np
import pytest
import torch

from oracle import tokenlake_oracle as orc
from paper_2508_17219_amd import binding as B

FAKE_K, FAKE_V = 0x10000000, 0x20000000          # never dereferenced
N = 3                                           # tokens of the refused calls


def test_steps_are_fractions_of_a_turn():
    getcontext().prec = 80
    two_pi = 2 * Decimal("3.14159265358979323846264338327950288419716939937510582097494459230781640628620899")
    freqs = [1.0, 1e-4, 1e6 ** -0.984375, 0.0, -0.25, 6.283185307179586, 7.5, 123456.789, 2.0 ** -60, 1e-300]
    got = B.tl_rope_steps(freqs)
    for f, step in zip(freqs, got.tolist()):
        turns = Decimal(f) / two_pi
        want = (turns * 2 ** 64) % (2 ** 64)
        off = abs(Decimal(step) - want)
        off = min(off, 2 ** 64 - off)
        assert off <= 1 + 2 * abs(turns), (f, off)           # 64 bits of mantissa: two units of the quotient, one of the rounding
    assert len(B.tl_rope_steps([])) == 0
    for bad in (float("nan"), float("inf")):
        with pytest.raises(B.TokenLakeError) as e:
            B.tl_rope_steps([1.0, bad])
        assert e.value.status == B.TL_EINVAL
    assert B.load_library().tl_rope_steps(None, 2, None) == B.TL_EINVAL
    assert B.load_library().tl_rope_steps(None, -1, None) == B.TL_EINVAL


def _two_pi(bits):
    """2 pi times 2^bits, by Machin's formula."""
    def arctan_of_inverse(x):
        power = total = (1 << (bits + 32)) // x
        n = 1
        while power:
            power //= -x * x
            n += 2
            total += power // n
        return total
    return 8 * (4 * arctan_of_inverse(5) - arctan_of_inverse(239)) >> 32


def test_steps_are_the_nearest_for_every_finite_frequency():
    """Whole turns are taken off exactly, however many a position turns by: from the least number to the largest."""
    two_pi = _two_pi(2400)
    rng = np.random.default_rng(6)
    bits = rng.integers(0, 2 ** 64, 4000, dtype=np.uint64).view(np.float64)
    freqs = np.concatenate([[1.0, 7.5, -0.25, 123456.789, 1e300, -1e300, 1e22, 5e-324, 2.0 ** -1022, np.finfo(np.float64).max, 2 ** 53 + 2.0, 2.0 ** -60, 0.0, -0.0],
                            rng.uniform(-1e6, 1e6, 500), 1e6 ** (-rng.random(500)), 2.0 ** np.arange(-1074, 1024), bits[np.isfinite(bits)]])
    for f, step in zip(freqs.tolist(), B.tl_rope_steps(freqs).tolist()):
        over, under = abs(f).as_integer_ratio()
        scaled = (over << (64 + 64 + 2400)) // (under * two_pi)              # turns times 2^64, 64 bits behind the point (below 2^-1000 off)
        want = (scaled if f >= 0 else -scaled) % (1 << 128)
        off = abs((step << 64) - want)
        off = min(off, (1 << 128) - off)
        assert off <= (1 << 63) + 2, (f, step, off / 2 ** 64)


# ---- places -------------------------------------------------------------------------------
def test_reserved_rows_are_where_the_oracle_appends():
    rng = np.random.default_rng(3)
    for trial in range(20):
        C_, n_slots = int(rng.choice([64, 128])), 24
        pool = B.tl_pool_create(n_slots, C_, 1, 128, FAKE_K, FAKE_V)
        table = orc.SlotTable(n_slots, C_)
        chains, totals, nid = [[] for _ in range(3)], [0, 0, 0], 100
        for step in range(6):
            tails, ids, counts = [], [], []
            for c in range(3):
                n = int(rng.choice([0, 1, 5, C_ - 1, C_, C_ + 1, 2 * C_ + 3]))
                tail = chains[c][-1] if totals[c] % C_ else None
                need = -(-max(0, n - (C_ - totals[c] % C_ if tail is not None else 0)) // C_)
                tails.append(tail), ids.append(list(range(nid, nid + need))), counts.append(n)
                nid += need
            if B.tl_pool_used(pool) + sum(map(len, ids)) > n_slots:
                before = B.tl_pool_used(pool)
                with pytest.raises(B.TokenLakeError) as e:
                    B.tl_pool_reserve_batch(pool, tails, ids, counts)
                assert e.value.status == B.TL_EFULL and B.tl_pool_used(pool) == before
                break
            slots, rows = B.tl_pool_reserve_batch(pool, tails, ids, counts)
            want = np.zeros(sum(counts), np.int64)
            base = 0
            for c in range(3):
                for slot, tok, n, row in table.append(tails[c], ids[c], counts[c]):
                    want[base + row:base + row + n] = slot * C_ + tok + np.arange(n)
                base += counts[c]
                chains[c] += ids[c]
                totals[c] += counts[c]
            assert np.array_equal(rows, want)
            assert np.array_equal(slots, table.lookup([i for x in ids for i in x]))
            every = [i for ch in chains for i in ch]
            at = table.lookup(every)
            assert np.array_equal(B.tl_pool_lookup(pool, every), at) and np.array_equal(B.tl_pool_fills(pool, at), table.fill(at))
        B.tl_pool_destroy(pool)


def test_reserve_refuses_what_append_refuses_and_changes_nothing():
    pool = B.tl_pool_create(4, 64, 1, 128, FAKE_K, FAKE_V)
    B.tl_pool_adopt(pool, [1, 2], [0, 1], [60, 64])
    assert B.tl_pool_put(pool, 2, FAKE_K, FAKE_V, 64, -1, stream=0) == 1      # a second holder
    for tails, ids, counts, status in [([9], [[]], [1], B.TL_ENOTFOUND), ([2], [[3]], [1], B.TL_EINVAL), ([1], [[3]], [4], B.TL_EINVAL),
                                       ([1], [[]], [5], B.TL_EINVAL), ([None], [[1]], [3], B.TL_EINVAL), ([None, None], [[3], [3]], [1, 1], B.TL_EINVAL),
                                       ([1, 1], [[], []], [1, 1], B.TL_EINVAL), ([None], [[3, 4, 5]], [130], B.TL_EFULL)]:
        with pytest.raises(B.TokenLakeError) as e:
            B.tl_pool_reserve_batch(pool, tails, ids, counts)
        assert e.value.status == status, (tails, ids, counts)
        assert B.tl_pool_used(pool) == 2 and list(B.tl_pool_fills(pool, [0, 1, 2, 3])) == [60, 64, 0, 0]
    lib = B.load_library()
    z, one = np.zeros(2, np.int32), np.array([0, 1], np.int32)
    assert lib.tl_pool_reserve_batch(None, 1, z.ctypes.data, None, z.ctypes.data, None, z.ctypes.data, None, None) == B.TL_EINVAL
    assert lib.tl_pool_reserve_batch(pool, -1, z.ctypes.data, None, z.ctypes.data, None, z.ctypes.data, None, None) == B.TL_EINVAL
    assert lib.tl_pool_reserve_batch(pool, 1, None, None, z.ctypes.data, None, z.ctypes.data, None, None) == B.TL_EINVAL
    ids = np.array([7], np.uint64)
    assert lib.tl_pool_reserve_batch(pool, 1, z.ctypes.data, None, one.ctypes.data, ids.ctypes.data, one.ctypes.data, None, None) == B.TL_EINVAL
    assert lib.tl_pool_reserve_batch(pool, 0, None, None, None, None, None, None, None) == B.TL_OK
    # a plan made before is stale, one made behind it sees the tokens
    slots, rows = B.tl_pool_reserve_batch(pool, [1, None], [[5], [6]], [6, 2])
    assert list(slots) == [2, 3] and list(rows) == [60, 61, 62, 63, 128, 129, 192, 193]
    assert list(B.tl_pool_fills(pool, [0, 1, 2, 3])) == [64, 64, 2, 2]
    B.tl_pool_destroy(pool)


def test_a_plan_goes_stale_when_rows_are_reserved():
    """A tail that grows alone, and a new segment: a plan made before is refused in front of any device work, and names the reason."""
    lib = B.load_library()
    for tails, ids, counts in (([10], [[]], [3]), ([None], [[12]], [5])):
        pool = B.tl_pool_create(4, 64, 1, 128, FAKE_K, FAKE_V)
        B.tl_pool_adopt(pool, [10, 11], [0, 1], [20, 64])
        plan = B.tl_plan_create(pool, 1, [0, 3], [0, 2], np.array([11, 10], np.uint64), B.TL_PLAN_SELF_BLOCK)
        B.tl_pool_reserve_batch(pool, tails, ids, counts)
        assert lib.tl_segment_attn(pool, plan, FAKE_K, 0.1, FAKE_K, FAKE_V, None) == B.TL_EINVAL
        assert b"pool has changed" in lib.tl_last_error() and b"reserve" in lib.tl_last_error()
        B.tl_plan_destroy(plan)
        B.tl_pool_destroy(pool)


def test_as_many_rows_as_there_may_be_are_counted():
    """2^31 - 1 rows for a chain: the new segments that they need are told, without overflow."""
    lib = B.load_library()
    pool = B.tl_pool_create(4, 64, 1, 128, FAKE_K, FAKE_V)
    none, new_ptr, row_ptr = np.zeros(1, np.int32), np.zeros(2, np.int32), np.array([0, 2 ** 31 - 1], np.int32)
    rows = np.zeros(1, np.int32)
    assert lib.tl_pool_reserve_batch(pool, 1, none.ctypes.data, None, new_ptr.ctypes.data, None, row_ptr.ctypes.data, None, rows.ctypes.data) == B.TL_EINVAL
    assert b"need exactly 33554432 new segments" in lib.tl_last_error(), lib.tl_last_error()
    B.tl_pool_destroy(pool)


# ---- refusals -----------------------------------------------------------------------------
def _rope(**kw):
    return B.tl_rope(**{**dict(steps_dev=0x5000, rot_dim=64, interleaved=0, factor=1.0), **kw})


def _rows(**kw):
    """3 tokens of 4 query heads on 2, each tensor dense and by itself."""
    d = dict(q=0x100000, k=0x200000, v=0x300000, q_row_stride=512, q_head_stride=128, k_row_stride=256, k_head_stride=128, v_row_stride=256,
             v_head_stride=128, q_heads=4, kv_heads=2, is_bf16=1, eps=1e-6, q_weight=None, k_weight=None, q_out=0x400000, k_out=0x500000, v_out=0x600000)
    return B.tl_qkv(**{**d, **kw})


def _refused(call, what):
    lib = B.load_library()
    assert call(lib) == B.TL_EINVAL
    assert what.encode() in lib.tl_last_error(), lib.tl_last_error()


@pytest.mark.parametrize("rope,what", [
    (dict(rot_dim=0), "rot_dim"), (dict(rot_dim=8), "rot_dim"), (dict(rot_dim=72), "rot_dim"), (dict(rot_dim=144), "rot_dim"), (dict(rot_dim=-16), "rot_dim"),
    (dict(steps_dev=None), "null steps"), (dict(factor=float("nan")), "factor"), (dict(factor=float("inf")), "factor")])
def test_rotations_that_are_refused(rope, what):
    pool = B.tl_pool_create(4, 64, 2, 128, FAKE_K, FAKE_V)
    _refused(lambda lib: lib.tl_rotate_rows(C.byref(_rope(**rope)), C.byref(_rows()), 0x7000, N, None), what)
    _refused(lambda lib: lib.tl_pool_write_rows(pool, C.byref(_rope(**rope)), C.byref(_rows()), 0x7000, 0x8000, N, None), what)
    _refused(lambda lib: lib.tl_pool_move_rows(pool, C.byref(_rope(**rope)), 0x7000, 0x8000, 0x9000, N, None), what)
    B.tl_pool_destroy(pool)


@pytest.mark.parametrize("rows,what", [
    (dict(q=None, k=None, v=None, q_out=None, k_out=None, v_out=None), "no rows"),
    (dict(q=None), "output for q without q"), (dict(v=None), "output for v without v"), (dict(q_out=None), "q without an output"),
    (dict(q_heads=0), "heads of q"), (dict(q_heads=-4), "heads of q"), (dict(q_heads=1 << 20), "heads of q"), (dict(kv_heads=0), "heads of k"),
    (dict(q_weight=0x5000, eps=0.0), "eps"), (dict(k_weight=0x5000, eps=-1.0), "eps"), (dict(q_weight=0x5000, eps=float("nan")), "eps"),
    (dict(q_weight=0x5000, eps=float("inf")), "eps"), (dict(q_weight=0x5000, eps=1e-40), "eps"),
    (dict(q_row_stride=1 << 62), "strides of q"), (dict(k_row_stride=1 << 58), "strides of k"), (dict(v_row_stride=-(1 << 30)), "strides of v"),
    (dict(q_head_stride=1 << 55), "strides of q"), (dict(v_head_stride=-(1 << 62)), "strides of v"),
    # an output over another input, over part of its own, over another output, over its own with other strides or of 32 bits
    (dict(k_out=0x100000 + 512), "overlaps q"), (dict(q_out=0x100000 + 256), "overlaps q"), (dict(k_out=0x600000 + 1024), "outputs of k and v overlap"),
    (dict(q_out=0x100000, q_row_stride=640), "overlaps q"), (dict(q_out=0x100000, is_bf16=0), "overlaps q"),
    (dict(v_out=0x300000, v_row_stride=128, v_head_stride=384), "overlaps v"), (dict(q=0x400000 + 3 * 1024, q_row_stride=-512), "overlaps q")])
def test_rows_that_are_refused(rows, what):
    _refused(lambda lib: lib.tl_rotate_rows(C.byref(_rope()), C.byref(_rows(**rows)), 0x7000, N, None), what)


def test_other_arguments_that_are_refused():
    pool = B.tl_pool_create(4, 64, 2, 128, FAKE_K, FAKE_V)
    rope, rows = _rope(), _rows()
    _refused(lambda lib: lib.tl_rotate_rows(C.byref(rope), None, 0x7000, N, None), "null rows")
    _refused(lambda lib: lib.tl_rotate_rows(C.byref(rope), C.byref(rows), None, N, None), "null positions")
    _refused(lambda lib: lib.tl_rotate_rows(C.byref(rope), C.byref(rows), 0x7000, -1, None), "negative")
    _refused(lambda lib: lib.tl_pool_write_rows(None, C.byref(rope), C.byref(rows), 0x7000, 0x8000, N, None), "null pool")
    _refused(lambda lib: lib.tl_pool_write_rows(pool, C.byref(rope), None, 0x7000, 0x8000, N, None), "null keys")
    _refused(lambda lib: lib.tl_pool_write_rows(pool, C.byref(rope), C.byref(_rows(k=None, k_out=None)), 0x7000, 0x8000, N, None), "null keys")
    _refused(lambda lib: lib.tl_pool_write_rows(pool, C.byref(rope), C.byref(_rows(kv_heads=4)), 0x7000, 0x8000, N, None), "heads, the pool has 2")
    _refused(lambda lib: lib.tl_pool_write_rows(pool, C.byref(rope), C.byref(rows), 0x7000, None, N, None), "null pool rows")
    _refused(lambda lib: lib.tl_pool_write_rows(pool, C.byref(rope), C.byref(rows), None, 0x8000, N, None), "null positions")
    _refused(lambda lib: lib.tl_pool_write_rows(pool, C.byref(rope), C.byref(rows), 0x7000, 0x8000, -1, None), "negative")
    for inside in (dict(k=FAKE_K + 4096), dict(q_out=FAKE_V + 1024), dict(v=FAKE_V - 512)):
        _refused(lambda lib: lib.tl_pool_write_rows(pool, C.byref(rope), C.byref(_rows(**inside)), 0x7000, 0x8000, N, None), "pool's slots")
    _refused(lambda lib: lib.tl_pool_move_rows(None, C.byref(rope), 0x7000, 0x8000, 0x9000, N, None), "null pool")
    _refused(lambda lib: lib.tl_pool_move_rows(pool, C.byref(rope), None, 0x8000, 0x9000, N, None), "null rows")
    _refused(lambda lib: lib.tl_pool_move_rows(pool, C.byref(rope), 0x7000, None, 0x9000, N, None), "null rows")
    _refused(lambda lib: lib.tl_pool_move_rows(pool, C.byref(rope), 0x7000, 0x8000, None, N, None), "shifts")
    _refused(lambda lib: lib.tl_pool_move_rows(pool, C.byref(rope), 0x7000, 0x8000, 0x9000, -1, None), "negative")
    B.tl_pool_destroy(pool)


def test_rows_are_packed_as_the_structure_is_laid_out():
    args = (1, 2, 3, 4, -5, 6, 7, -8, 9, 10, 11, True, 0.5, 12, 13, 14, 15, 16)
    assert B._PACK_QKV(*args) == bytes(B.tl_qkv(*args))


def test_no_tokens_are_no_work():
    lib = B.load_library()
    assert lib.tl_rotate_rows(None, None, None, 0, None) == B.TL_OK
    assert lib.tl_pool_write_rows(None, None, None, None, None, 0, None) == B.TL_OK
    assert lib.tl_pool_move_rows(None, None, None, None, None, 0, None) == B.TL_OK


def test_binding_refuses_tensors_that_are_not_on_a_gpu():
    q, pos = torch.zeros(N, 4, 128, dtype=torch.bfloat16), torch.zeros(N, dtype=torch.int32)
    with pytest.raises(ValueError, match="no rows"):
        B.tl_rotate_rows(None, None)
    with pytest.raises(ValueError, match="device"):
        B.tl_rotate_rows(None, None, q, q_out=q)
    with pytest.raises(ValueError, match="device"):
        B.tl_rope_of(torch.zeros(64, dtype=torch.int64))
    with pytest.raises(TypeError, match="steps"):
        B.tl_rope_of(torch.zeros(64))
    pool = B.tl_pool_create(4, 64, 4, 128, FAKE_K, FAKE_V)
    with pytest.raises(ValueError, match="device"):
        B.tl_pool_write_rows(pool, None, None, pos, q, q)
    with pytest.raises(ValueError, match="device"):
        B.tl_pool_move_rows(pool, None, pos, pos)
    B.tl_pool_destroy(pool)


@pytest.mark.parametrize("n,heads,fits,not_so", [
    (10, 4, [(10, 4, 128), (10, 512), (5120,), (40, 128), (1, 10, 512), (2, 5, 4, 128), (2, 5, 512), (1, 40, 128), (10, 1, 512), (10, 2, 2, 128)],
     [(4, 10, 128), (10, 128, 4), (128, 10, 4), (4, 1280), (2, 4, 5, 128), (4, 5, 2, 128), (20, 256), (10, 4, 64), (10, 4, 2, 128), (0, 4, 128)]),
    (1, 4, [(1, 4, 128), (4, 1, 128), (512,), (4, 128), (1, 512)], [(128, 4), (1, 128, 4), (2, 4, 128)]),
    (5, 1, [(5, 1, 128), (1, 5, 128), (640,), (5, 128)], [(128, 5), (128, 1, 5), (5, 1, 256)]),
    (1, 1, [(1, 1, 128), (128,)], [(64, 2), ()])])
def test_outputs_of_another_order_do_not_fit(n, heads, fits, not_so):
    for shape in fits:
        assert B._in_order(torch.Size(shape), n, heads), shape
    for shape in not_so:
        assert not B._in_order(torch.Size(shape), n, heads), shape
