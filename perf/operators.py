"""The operators between a layer's QKV projection and the attention over the segment pool, as cases to time.

  rotate   norms of queries and keys for each head and their position rotation, values split off: from the projection's rows to
           the dense tensors that the attention reads
  write    the same for rows that go to the pool: keys are normed, turned and written to their places in the slots with the
           values, queries come along to their dense tensor
  move     rows of the pool go to other places and positions: keys are turned by the difference

Shapes are those of the repository's workloads (32 query heads on 8 KV heads, 64 on 8, the tiny 8 on 2, 70B's layer split over 8
GPUs: 8 on 1), its chunk and batch sizes and its segment lengths.
"""
from __future__ import annotations

import math

import torch

own = False

D = 128

# n: tokens, as `chains` runs of consecutive positions; first: positions at which a run starts lie below it; fused: q, k and v
# are views into one projection's rows [n, (q_heads + 2 kv_heads) * 128]; norm: weights for queries and keys; rot: dimensions that
# turn; inter: pairs (2i, 2i + 1) in place of (i, i + rot / 2); factor: on the turned dimensions
_ROTATE = dict(op="rotate", n=1, chains=1, q_heads=32, kv_heads=8, kind="bf16", fused=True, norm=True, rot=128, inter=False,
               base=1e6, factor=1.0, first=32768)
# seg_len: tokens of a slot; dense: the turned keys and the values are wanted as dense tensors too, for the self block; queries: whether they come along
_WRITE = dict(_ROTATE, op="write", seg_len=256, queries=True, dense=False)
# n rows as `chains` runs; shift: by how many positions at most they move
_MOVE = dict(op="move", n=1, chains=1, kv_heads=8, seg_len=256, rot=128, inter=False, base=1e6, shift=32768)


def listed():
    return [
        # One decoded token of the 70B shape: launches and latency.
        dict(_ROTATE, name="rotate_one_token", q_heads=64),
        # The decode configuration's batch of 256 requests far apart.
        dict(_ROTATE, name="rotate_decode_256", n=256, chains=256, q_heads=64, first=131072),
        # Odd sizes: ragged chunks, an odd group, half the dimensions turn, neighbouring pairs, no norm, tensors of their own.
        dict(_ROTATE, name="rotate_partial_pairs", n=1021, chains=5, q_heads=28, kv_heads=4, fused=False, norm=False, rot=64,
             inter=True, base=1e4),
        # The prefill configuration: 16 chunks of 512 tokens.
        dict(_ROTATE, name="rotate_chunks", n=8192, chains=16),
        # A turn of the multi-turn configuration whose projection left its sums in 32 bits; stretched frequencies with a factor.
        dict(_ROTATE, name="rotate_fp32_rows", n=16384, chains=64, kind="fp32", norm=False, base=5e5, factor=1.2),
        # A decode batch of a few users: keys and values to the pool, queries along.
        dict(_WRITE, name="write_decode_16", n=16, chains=16, q_heads=64, seg_len=64, first=131072),
        # The decode configuration's batch.
        dict(_WRITE, name="write_decode_256", n=256, chains=256, q_heads=64, seg_len=64, first=131072),
        # Ragged chunks whose queries go another way: keys and values alone.
        dict(_WRITE, name="write_chunks", n=8191, chains=16, queries=False),
        # A turn of the multi-turn configuration: everything the layer needs in one launch.
        dict(_WRITE, name="write_turn", n=16384, chains=64, dense=True),
        # The end of one conversation moves up by what was dropped in front of it.
        dict(_MOVE, name="move_tail", n=777, chains=1),
        # One of 8 GPUs has one KV head; sessions of a few thousand tokens.
        dict(_MOVE, name="move_one_kv_head", n=20000, chains=8, kv_heads=1, seg_len=64, rot=64, inter=True, base=1e4),
        # The long-context configuration's prefix of 128k tokens.
        dict(_MOVE, name="move_long_prefix", n=131072, chains=4, seg_len=512),
    ]


_HEADS = [(32, 8), (64, 8), (8, 2), (8, 1), (16, 4), (28, 4), (16, 16), (32, 8)]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    most = max(work(c)["bytes"] for c in listed())
    for _ in range(1000):
        hq, hkv = rng.choice(_HEADS)
        common = dict(kv_heads=hkv, rot=rng.choice([128, 128, 128, 96, 64, 32]), inter=rng.random() < 0.3, base=rng.choice([1e4, 5e5, 1e6]))
        op = rng.choice(["rotate", "rotate", "write", "write", "move"])
        n = _log_int(rng, 1, 131072 if op == "move" else 16384)
        common.update(n=n, chains=rng.choice([1, min(n, 16), n if n <= 512 else 64]))
        if op == "move":
            case = dict(_MOVE, seg_len=rng.choice([64, 128, 256, 512]), shift=_log_int(rng, 16, 131072))
        else:
            case = dict(_ROTATE if op == "rotate" else _WRITE, q_heads=hq, kind=rng.choice(["bf16", "bf16", "bf16", "fp32"]), fused=rng.random() < 0.6,
                        norm=rng.random() < 0.6, factor=rng.choice([1.0, 1.0, 1.1]), first=_log_int(rng, 1024, 1048576))
            if op == "write":
                case.update(seg_len=rng.choice([64, 128, 256, 512]), queries=rng.random() < 0.7, dense=rng.random() < 0.4)
        case.update(common)
        if work(case)["bytes"] <= most:
            return case
    raise RuntimeError("no case within the limits")


def work(case):
    n, hkv = case["n"], case["kv_heads"]
    if case["op"] == "move":
        return {"bytes": n * (8 * hkv * D + 12), "flops": n * hkv * D * 4}
    size = 2 if case["kind"] == "bf16" else 4
    hq = case["q_heads"] if case.get("queries", True) else 0
    values = n * (hq + 2 * hkv) * D
    moved = values * (size + 2) + 4 * n + 4 * case["rot"]
    if case["op"] == "write":
        moved += 4 * n + (n * 2 * hkv * D * 2 if case["dense"] else 0)
    if case["norm"]:
        moved += (4 * D if hq else 0) + 4 * D
    return {"bytes": moved, "flops": n * (hq + hkv) * D * (4 + (4 if case["norm"] else 0))}


# ---- inputs ---------------------------------------------------------------------------------------------
def _runs(case, g, dev, first):
    """n tokens as ragged runs: (run of each token, its number in the run, where each run starts)."""
    n, chains = case["n"], case["chains"]
    cut = torch.randperm(n - 1, generator=g, device=dev)[:chains - 1].sort().values + 1 if chains < n else torch.arange(1, n, device=dev)
    begin = torch.cat([torch.zeros(1, dtype=torch.int64, device=dev), cut])
    run = torch.zeros(n, dtype=torch.int64, device=dev)
    run[begin[1:]] = 1
    run = run.cumsum(0)
    start = torch.randint(0, first, (len(begin),), generator=g, device=dev)
    return run, torch.arange(n, device=dev) - begin[run], start


def _places(case, g, dev, run, at, start):
    """A pool row for each token: runs lie in slots of their own, scattered, the first entered in its middle.
    (rows, slots of the pool: enough wherever the runs begin)"""
    C = case["seg_len"]
    token = start[run] % C + at
    slots_of = torch.zeros(int(run[-1]) + 1, dtype=torch.int64, device=dev).scatter_reduce_(0, run, token // C + 1, "amax")
    before = slots_of.cumsum(0) - slots_of
    n_slots = case["n"] // C + 2 * case["chains"] + 1
    slot = torch.randperm(n_slots, generator=g, device=dev)
    return slot[before[run] + token // C] * C + token % C, n_slots


def prepare(case, seed):
    dev = "cuda" if torch.cuda.is_available() else "cpu"
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    n, hkv, rot = case["n"], case["kv_heads"], case["rot"]
    freq = case["base"] ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
    s = {"case": case, "freq": freq.to(dev)}
    if case["op"] == "move":
        run, at, start = _runs(case, g, dev, case["seg_len"])
        src, n_src = _places(case, g, dev, run, at, start)
        dst, n_dst = _places(case, g, dev, run, at, torch.randint(0, case["seg_len"], start.shape, generator=g, device=dev))
        shift = torch.randint(-case["shift"], case["shift"] + 1, start.shape, generator=g, device=dev)
        s["n_slots"] = n_src + n_dst
        s["src"], s["dst"] = src.to(torch.int32), (dst + n_src * case["seg_len"]).to(torch.int32)
        s["shift"] = shift[run].to(torch.int32)
    else:
        run, at, start = _runs(case, g, dev, case["first"])
        s["pos"] = (start[run] + at).to(torch.int32)
        kind = torch.bfloat16 if case["kind"] == "bf16" else torch.float32
        hq = case["q_heads"] if case.get("queries", True) else 0
        heads = hq + 2 * hkv
        # a projection's rows: channels of different size
        gain = torch.exp(0.5 * torch.randn(heads * D, generator=g, device=dev))
        rows = (torch.randn((n, heads * D), generator=g, device=dev) * gain).to(kind).view(n, heads, D)
        s["q"], s["k"], s["v"] = rows[:, :hq], rows[:, hq:hq + hkv], rows[:, hq + hkv:]
        if not case["fused"]:
            s["q"], s["k"], s["v"] = (t.contiguous() for t in (s["q"], s["k"], s["v"]))
        s["q_out"], s["k_out"], s["v_out"] = (torch.empty((n, h, D), dtype=torch.bfloat16, device=dev) for h in (hq, hkv, hkv))
        s["q_weight"], s["k_weight"] = ((1.0 + 0.2 * torch.randn(D, generator=g, device=dev)) if case["norm"] else None for _ in "qk")
        if case["op"] == "write":
            rows, s["n_slots"] = _places(case, g, dev, run, at, start)
            s["rows"] = rows.to(torch.int32)
    if "n_slots" in s:
        # rows that are not written hold what other sequences left there
        s["pool_k"], s["pool_v"] = (torch.randn((s["n_slots"], case["seg_len"], hkv, D), generator=g, device=dev, dtype=torch.bfloat16) for _ in "kv")
    if own:
        from paper_2508_17219_amd import binding as B
        steps = torch.from_numpy(B.tl_rope_steps(freq.numpy()).view("int64")).to(dev)
        s["rope"] = B.tl_rope_of(steps, case["inter"], case.get("factor", 1.0))
        if "n_slots" in s:
            s["pool"] = B.tl_pool_create(s["n_slots"], case["seg_len"], hkv, D, s["pool_k"], s["pool_v"])
    return s


EPS = 1e-6


# ---- the operators --------------------------------------------------------------------------------------
def _normed(x, weight):
    if weight is None:
        return x
    return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * weight


def _turned(x, angle, inter, factor):
    """x [n, heads, 128] in 32 bits, angle [n, rot / 2] in 64."""
    cos, sin = ((f(angle) * factor).float()[:, None] for f in (torch.cos, torch.sin))
    rot = 2 * angle.shape[1]
    if inter:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        turned = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        turned = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
    return torch.cat([turned, x[..., rot:]], -1)


def _plain(s):
    case = s["case"]
    if case["op"] == "move":
        k, v = s["pool_k"].view(-1, case["kv_heads"], D), s["pool_v"].view(-1, case["kv_heads"], D)
        src, dst = s["src"].long(), s["dst"].long()
        angle = s["shift"].double()[:, None] * s["freq"]
        k[dst] = _turned(k[src].float(), angle, case["inter"], 1.0).to(k.dtype)
        v[dst] = v[src]
        return s["pool_k"], s["pool_v"]
    angle = s["pos"].double()[:, None] * s["freq"]
    q = _turned(_normed(s["q"].float(), s["q_weight"]), angle, case["inter"], case["factor"]).to(torch.bfloat16) if s["q"].shape[1] else None
    k = _turned(_normed(s["k"].float(), s["k_weight"]), angle, case["inter"], case["factor"]).to(torch.bfloat16)
    v = torch.empty_like(s["v_out"]).copy_(s["v"])
    if case["op"] == "rotate":
        return q, k, v
    rows = s["rows"].long()
    s["pool_k"].view(-1, case["kv_heads"], D)[rows] = k
    s["pool_v"].view(-1, case["kv_heads"], D)[rows] = v
    out = [s["pool_k"], s["pool_v"]] + ([q] if q is not None else [])
    return out + [k, v] if case["dense"] else out


def run(s):
    if not own:
        return _plain(s)
    from paper_2508_17219_amd import binding as B
    case = s["case"]
    if case["op"] == "move":
        B.tl_pool_move_rows(s["pool"], s["rope"], s["src"], s["dst"], s["shift"])
        return s["pool_k"], s["pool_v"]
    if case["op"] == "rotate":
        B.tl_rotate_rows(s["rope"], s["pos"], s["q"], s["k"], s["v"], s["q_out"], s["k_out"], s["v_out"], s["q_weight"], s["k_weight"], EPS)
        return s["q_out"], s["k_out"], s["v_out"]
    has_q, dense = s["q"].shape[1] > 0, case["dense"]
    B.tl_pool_write_rows(s["pool"], s["rope"], s["pos"], s["rows"], s["k"], s["v"], s["q"] if has_q else None, s["q_out"] if has_q else None,
                         s["k_out"] if dense else None, s["v_out"] if dense else None, s["q_weight"] if has_q else None, s["k_weight"], EPS)
    out = [s["pool_k"], s["pool_v"]] + ([s["q_out"]] if has_q else [])
    return out + [s["k_out"], s["v_out"]] if dense else out


# ---- the definition in 64 bits: a pair of dimensions is a complex number, a position turns it --------------
def exact(case, seed):
    s = prepare(case, seed)
    half = case["rot"] // 2

    def at(x, steps, factor):
        phase = torch.polar(torch.full_like(steps, factor), steps).unsqueeze(1)
        y = x.clone()
        if case["inter"]:
            z = torch.view_as_complex(x[..., :2 * half].unflatten(-1, (half, 2)).contiguous()) * phase
            y[..., :2 * half] = torch.view_as_real(z).flatten(-2)
        else:
            z = torch.complex(x[..., :half].contiguous(), x[..., half:2 * half].contiguous()) * phase
            y[..., :half], y[..., half:2 * half] = z.real, z.imag
        return y

    if case["op"] == "move":
        angles = torch.outer(s["shift"].double(), s["freq"])
        k, v = s["pool_k"].double(), s["pool_v"].double()
        flat_k, flat_v = k.flatten(0, 1), v.flatten(0, 1)
        src, dst = s["src"].long(), s["dst"].long()
        flat_k[dst] = at(flat_k[src], angles, 1.0)
        flat_v[dst] = flat_v[src]
        return k, v
    angles = torch.outer(s["pos"].double(), s["freq"])

    def normed(x, weight):
        if weight is None:
            return x
        size = (torch.linalg.vector_norm(x, dim=-1, keepdim=True) ** 2 / D + EPS) ** 0.5
        return x / size * weight.double()

    q = at(normed(s["q"].double(), s["q_weight"]), angles, case["factor"])
    k = at(normed(s["k"].double(), s["k_weight"]), angles, case["factor"])
    v = s["v"].double()
    if case["op"] == "rotate":
        return q, k, v
    pool_k, pool_v = s["pool_k"].double(), s["pool_v"].double()
    pool_k.flatten(0, 1)[s["rows"].long()] = k
    pool_v.flatten(0, 1)[s["rows"].long()] = v
    out = [pool_k, pool_v] + ([q] if q.shape[1] else [])
    return out + [k, v] if case["dense"] else out
