"""Operators of a serving program around a ragged KV cache, as cases that can be timed: decode attention over cached rows
in 4 bits (alone, and as a decode step that rounds and appends the new row first), the append of new tokens with norms
and position rotation on the way, and the same norms and rotation without a cache.

A case is a dict of plain values:
  op       "attend": decode attention over the cached rows;  "step": append of one row a sequence, then attention;
           "append": norms, rotation and append of `tokens` (all sequences');  "rotate": norms and rotation alone
  heads, kv_heads, dim    query heads, cached heads, head dimension
  cache, act, out         types of the cached rows, of queries and new rows, of attention's outputs
  batch, shortest, longest, max_len, length_seed    sequences and their rows (attend, step: cached; append: new)
  first    append: rows that every sequence holds already (the new rows' positions begin there)
  rotary, interleaved, axes, norm    rotation: elements of a head that turn, how they pair, position axes; norms or not
  tokens   rotate: rows of the joined query / key / value projection

`own` False computes them in plain torch, True by the library.  Cached rows in 4 bits are e2m1 codes (two a byte, the
first in the low half) in blocks of 32 under a power of two, 2^(byte - 127).
"""
import math
import random

import numpy as np
import torch

own = False

DEV = "cuda:0"
GRANULE = 64
_TORCH = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
_BYTES = {"f16": 2.0, "bf16": 2.0, "f32": 4.0, "e4m3": 1.0, "mxfp4": 17 / 32}
_LARGEST = {"f16": 140, "bf16": 252}  # largest scale byte: every code of the block is finite in the type of new rows


def _attn(name, op, shape, types, batch, lens, max_len=2048, length_seed=1):
    case = dict(op=op, heads=shape[0], kv_heads=shape[1], dim=shape[2], cache="mxfp4", act=types[0], out=types[1], batch=batch,
                shortest=lens[0], longest=lens[1], max_len=max_len, length_seed=length_seed)
    return dict(case, name=name) if name else case


def _append(name, shape, types, batch, lens, rotation, first=0, max_len=2048, length_seed=1):
    case = dict(op="append", heads=shape[0], kv_heads=shape[1], dim=shape[2], cache=types[0], act=types[1], batch=batch,
                shortest=lens[0], longest=lens[1], first=first, rotary=rotation[0], interleaved=rotation[1], axes=rotation[2],
                norm=rotation[3], max_len=max_len, length_seed=length_seed)
    return dict(case, name=name) if name else case


def _rotate(name, shape, act, tokens, rotation):
    case = dict(op="rotate", heads=shape[0], kv_heads=shape[1], dim=shape[2], act=act, tokens=tokens, rotary=rotation[0],
                interleaved=rotation[1], axes=rotation[2], norm=rotation[3])
    return dict(case, name=name) if name else case


def listed():
    return [
        # the smallest batch: four short contexts of sixteen heads of 256, where the latency of a call counts
        _attn("step_few_short_f16", "step", (16, 16, 256), ("f16", "f16"), 4, (17, 128)),
        # one user with a long conversation, grouped heads
        _attn("step_one_long_bf16", "step", (32, 8, 128), ("bf16", "bf16"), 1, (8000, 8200), max_len=16384),
        # an ordinary serving batch of a multi-head model, 32-bit outputs
        _attn("step_b64_f16", "step", (16, 16, 256), ("f16", "f32"), 64, (32, 1000)),
        # an ordinary serving batch with grouped heads
        _attn("attend_grouped_b256_bf16", "attend", (32, 8, 128), ("bf16", "bf16"), 256, (32, 1000)),
        # sixteen query heads on one cached head
        _attn("attend_multi_query_b256_f16", "attend", (16, 1, 256), ("f16", "f16"), 256, (32, 1000)),
        # the batch and the contexts that a cache of 4 bits makes room for
        _attn("attend_grouped_b512_long_bf16", "attend", (32, 8, 128), ("bf16", "bf16"), 512, (512, 4096), max_len=4096),
        # one new token of each of 64 sequences, norms and rotation, 16-bit rows
        _append("append_decode_b64_bf16", (32, 8, 128), ("bf16", "bf16"), 64, (1, 1), (128, False, 1, True), first=700),
        # newcomers' prompts into rows of 4 bits
        _append("append_prompts_4bit_bf16", (32, 8, 128), ("mxfp4", "bf16"), 4, (900, 2047), (128, False, 1, True)),
        # prompts of a model that rotates 64 of 256 elements in neighbouring pairs, without norms
        _append("append_prompts_partial_f16", (16, 16, 256), ("f16", "f16"), 8, (32, 512), (64, True, 1, False)),
        # pictures and text (three position axes) into 8-bit rows, long runs
        _append("append_three_axes_8bit_bf16", (32, 8, 128), ("e4m3", "bf16"), 16, (1000, 2048), (128, False, 3, True)),
        # single tokens of a large batch, norms and rotation without a cache
        _rotate("rotate_decode_b256_bf16", (32, 8, 128), "bf16", 256, (128, False, 1, True)),
        # a long prompt's queries and keys, three axes
        _rotate("rotate_prompt_32k_bf16", (32, 8, 128), "bf16", 32768, (128, False, 3, True)),
    ]


_SHAPES = [(16, 16, 256), (12, 12, 128), (32, 32, 128), (16, 16, 64), (3, 3, 128), (32, 8, 128), (32, 8, 128), (16, 1, 256),
           (8, 1, 64), (12, 4, 128), (24, 8, 64), (64, 8, 128), (40, 5, 128), (16, 8, 128), (6, 3, 256), (12, 2, 128), (20, 1, 128)]
_MOST_BYTES = 1.0e9  # below the largest listed case


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attend", "attend", "step", "step", "append", "append", "rotate"])
    shape, act = rng.choice(_SHAPES), rng.choice(["f16", "bf16"])
    dim = shape[2]
    rotation = (rng.choice([dim, dim, dim // 2, dim // 4, 2 * rng.randint(1, dim // 2)]), rng.random() < 0.3, rng.choice([1, 1, 2, 3]),
                rng.random() < 0.6)
    if op == "rotate":
        c = _rotate(None, shape, act, _log_uniform(rng, 1, 20000), rotation)
        while work(c)["bytes"] > 0.6e9:
            c["tokens"] = c["tokens"] * 3 // 4
        return c
    max_len = 16384 if rng.random() < 0.2 else 2048
    longest = _log_uniform(rng, 1, max_len - 1)
    lens = (max(1, int(longest * rng.uniform(0.02, 1.0))), longest)
    seed = rng.randrange(1 << 30)
    if op == "append":
        cache = rng.choice([act, "e4m3", "mxfp4"])
        batch = _log_uniform(rng, 1, 256)
        first = rng.choice([0, rng.randrange(max_len - longest)])
        c = _append(None, shape, (cache, act), batch, lens, rotation, first, max_len, seed)
        while work(c)["bytes"] > 0.4e9 or c["batch"] * (c["first"] + c["longest"]) > 200000:
            if c["batch"] > 1:
                c["batch"] = c["batch"] * 3 // 4
            else:
                c["longest"] = c["longest"] * 3 // 4
                c["shortest"] = min(c["shortest"], c["longest"])
        return c
    c = _attn(None, op, shape, (act, rng.choice(["f32", act, act])), _log_uniform(rng, 1, 512), lens, max_len, seed)
    while work(c)["bytes"] > _MOST_BYTES:
        if c["batch"] > 1:
            c["batch"] = c["batch"] * 3 // 4
        else:
            c["longest"] = c["longest"] * 3 // 4
            c["shortest"] = min(c["shortest"], c["longest"])
    return c


def _lens(case):
    r = random.Random(case["length_seed"])
    return [r.randint(case["shortest"], case["longest"]) for _ in range(case["batch"])]


def work(case):
    q, kv, dim = case["heads"] * case["dim"], case["kv_heads"] * case["dim"], case["dim"]
    act = _BYTES[case["act"]]
    if case["op"] == "rotate":  # queries and keys read and written, positions and frequencies read
        n = case["tokens"]
        return {"bytes": n * (2.0 * (q + kv) * act + 4 * case["axes"]) + 2 * case["rotary"],
                "flops": float(n * (q + kv) * (4 if case["norm"] else 0) + 3 * n * (q + kv) / dim * case["rotary"])}
    n, rows = case["batch"], sum(_lens(case))
    cached = _BYTES[case["cache"]]
    if case["op"] == "append":  # queries read and written, keys and values read, stored (and, rounded, read back as numbers)
        back = 0.0 if case["cache"] == case["act"] else 2.0 * kv * (cached + act)
        return {"bytes": rows * (2.0 * q * act + 2 * kv * (act + cached) + back + 12 + 4 * case["axes"]) + 2 * case["rotary"],
                "flops": float(rows * (q + kv) * (4 if case["norm"] else 0) + 3 * rows * (q + kv) / dim * case["rotary"])}
    step = case["op"] == "step"
    moved = 2 * kv * cached * rows + n * (q * (act + _BYTES[case["out"]]) + 12)
    if step:  # new rows read, stored, and read back as numbers
        moved += 2.0 * n * kv * (act + cached + cached + act)
    return {"bytes": float(moved), "flops": 4.0 * q * (rows + (n if step else 0))}


# ---- inputs ------------------------------------------------------------------------------------------------------


def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _normal(g, shape, act):
    return torch.empty(shape, dtype=_TORCH[act], device=DEV).normal_(generator=g)


_E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _power(exponent, dtype=torch.float32):
    """2^exponent, from its bits (torch's own powers may be off by the last one on a GPU)."""
    if dtype == torch.float64:
        return ((exponent.long() + 1023) << 52).view(torch.float64)
    exponent = exponent.int()
    return torch.where(exponent < -126, 2.0 ** -127, ((exponent.clamp(min=-126) + 127) << 23).view(torch.float32))


def _to_blocks(x, act):
    """Numbers [..., D] in 32 bits -> codes [..., D / 2] and scale bytes [..., D / 32], both uint8."""
    b = x.reshape(*x.shape[:-1], -1, 32)
    most = b.abs().amax(-1)
    whole = torch.isfinite(b).all(-1)
    # the power of two under which the largest element is below 7, where the nearest code is 6 at the most
    byte = (((torch.where(whole, most, 1.0).view(torch.int32) + (1 << 21)) >> 23) - 2).clamp(1, _LARGEST[act])
    y = b / torch.where(whole, _power(byte - 127), 1.0).unsqueeze(-1)
    a = y.abs()
    code = torch.zeros_like(a, dtype=torch.int32)
    for k, (mid, up) in enumerate(((0.25, False), (0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True), (5.0, False))):
        code += (a >= mid) if up else (a > mid)  # a tie goes to the even code
    code = torch.where(torch.signbit(y), code + 8, code).reshape(*x.shape[:-1], -1, 2)
    return (code[..., 0] | code[..., 1] << 4).to(torch.uint8), torch.where(whole, byte, 255).to(torch.uint8)


def _from_blocks(codes, scales):
    table = torch.tensor(_E2M1 + tuple(-v for v in _E2M1), device=codes.device)
    low, high = (codes & 15).long(), (codes >> 4).long()
    x = table[torch.stack((low, high), -1)].flatten(-2)
    s = torch.where(scales == 255, math.nan, _power(scales.int() - 127))
    return x * s.repeat_interleave(32, -1)


def _to_e4m3(x):
    """Numbers in 32 bits -> the nearest that an e4m3 code stands for, ties to even, none beyond 448."""
    exponent = ((x.abs().view(torch.int32) >> 23) - 127).clamp(min=-6)
    step = _power(exponent - 3)
    return (torch.round(x / step) * step).clamp(-448, 448)


class _State:
    """What a serving program holds between two calls."""

    def __del__(self):
        if getattr(self, "arena", None) is not None:
            from paper_2306_06000_amd import binding as s3

            torch.cuda.synchronize()
            s3.s3_kv_arena_destroy(self.arena)
            self.arena = None


def _stored_rows(g, case, rows):
    """Cached rows of one plane: N(0, 1) in the type of new rows, rounded to blocks, some thousand rows at a time."""
    kv, dim = case["kv_heads"], case["dim"]
    codes = torch.empty((rows, kv, dim // 2), dtype=torch.uint8, device=DEV)
    scales = torch.empty((rows, kv, dim // 32), dtype=torch.uint8, device=DEV)
    for at in range(0, rows, 1 << 16):
        end = min(rows, at + (1 << 16))
        codes[at:end], scales[at:end] = _to_blocks(_normal(g, (end - at, kv, dim), case["act"]).float(), case["act"])
    return codes, scales


def _attention_inputs(case, seed):
    g, n, lens = _generator(seed), case["batch"], _lens(case)
    k, v = _stored_rows(g, case, sum(lens)), _stored_rows(g, case, sum(lens))
    q = _normal(g, (n, case["heads"], case["dim"]), case["act"])
    new = [_normal(g, (n, case["kv_heads"], case["dim"]), case["act"]) for _ in range(2)]
    return lens, k, v, q, new[0], new[1]


def _rotation_inputs(case, g, n, positions):
    """Positions on every axis, frequencies, norm weights."""
    pairs, axes = case["rotary"] // 2, case["axes"]
    pos = torch.stack([positions if a == 0 else torch.randint(0, 4096, (n,), generator=g, device=DEV, dtype=torch.int32)
                       for a in range(axes)])
    # time, height and width take turns over the pairs
    axis = np.arange(pairs, dtype=np.uint8) % axes
    inv_freq = (1e6 ** (-np.arange(pairs) / max(pairs, 1))).astype(np.float32)
    weights = [1 + 0.1 * torch.randn(case["dim"], generator=g, device=DEV) for _ in range(2)] if case["norm"] else [None, None]
    return pos, axis, torch.from_numpy(inv_freq).to(DEV), weights


def prepare(case, seed):
    s = _State()
    s.case = case
    return {"attend": _prepare_attention, "step": _prepare_attention, "append": _prepare_append, "rotate": _prepare_rotate}[case["op"]](s, case, seed)


def _arena(s, case, preds):
    from paper_2306_06000_amd import binding as s3

    code = {"f16": s3.S3_F16, "bf16": s3.S3_BF16, "e4m3": s3.S3_E4M3, "mxfp4": s3.S3_MXFP4}
    s.code = {"f16": s3.S3_F16, "bf16": s3.S3_BF16, "f32": s3.S3_F32}
    cfg = s3.make_config(1, case["heads"], case["dim"], code[case["cache"]], GRANULE, case["max_len"],
                         0 if case["kv_heads"] == case["heads"] else case["kv_heads"], code[case["act"]])
    s.caps = [s3.s3_kv_capacity_for(cfg, p) for p in preds]
    s.memory = torch.zeros(sum(s.caps) * s3.s3_kv_bytes_per_token(cfg), dtype=torch.uint8, device=DEV)
    st, s.arena = s3.s3_kv_arena_init(cfg, s.memory, s.memory.numel())
    s3.check(st, "s3_kv_arena_init")
    admitted, ids, offs, _caps = s3.s3_kv_alloc(s.arena, preds)
    if admitted != len(preds):
        raise RuntimeError("the arena does not hold the batch")
    return s3, ids, offs


def _offsets(case, preds):
    """Slots one behind the other, as the arena places them when it is empty."""
    caps = [min(case["max_len"], max(GRANULE, -(-p // GRANULE) * GRANULE)) for p in preds]
    return np.concatenate([[0], np.cumsum(caps)])


def _prepare_attention(s, case, seed):
    lens, k, v, s.q, s.k_new, s.v_new = _attention_inputs(case, seed)
    n, step = case["batch"], case["op"] == "step"
    preds = [min(case["max_len"], length + 1) for length in lens]
    starts = np.concatenate([[0], np.cumsum(lens)])
    s.pos = torch.tensor(lens, dtype=torch.int32, device=DEV)
    s.len = torch.zeros_like(s.pos)
    s.out = torch.zeros((n, case["heads"], case["dim"]), dtype=_TORCH[case["out"]], device=DEV)
    s.k_row, s.v_row = torch.zeros_like(s.k_new), torch.zeros_like(s.v_new)
    if own:
        s3, ids, offs = _arena(s, case, preds)
        stream = torch.cuda.current_stream().cuda_stream
        row = s3.s3_kv_bytes_per_token(s3.make_config(1, case["heads"], case["dim"], s3.S3_MXFP4, GRANULE, case["max_len"],
                                                      case["kv_heads"], s.code[case["act"]])) // 2
        s.slot_off = torch.tensor(offs.tolist(), dtype=torch.int64, device=DEV)
        packed = []
        for codes, scales in (k, v):  # stored rows: the codes of all heads, their scales, zeros up to 16 bytes
            p = torch.zeros((codes.shape[0], row), dtype=torch.uint8, device=DEV)
            c = codes[0].numel() if codes.shape[0] else 0
            p[:, :c] = codes.flatten(1)
            p[:, c:c + (scales[0].numel() if codes.shape[0] else 0)] = scales.flatten(1)
            packed.append([p[starts[i]:starts[i + 1]] for i in range(n)])
        s3.check(s3.s3_kv_fill_batch(s.arena, 0, ids, np.array(lens, np.int32), packed[0], packed[1], stream), "s3_kv_fill_batch")
        s3.check(s3.s3_kv_reserve_scratch(s.arena, n), "s3_kv_reserve_scratch")
        torch.cuda.synchronize()
        return s
    at = _offsets(case, preds)
    s.lens, s.starts, s.planes = lens, at[:-1].tolist(), []
    for codes, scales in (k, v):
        full = [torch.zeros((int(at[-1]), *x.shape[1:]), dtype=torch.uint8, device=DEV) for x in (codes, scales)]
        for i in range(n):
            for f, x in zip(full, (codes, scales)):
                f[at[i]:at[i] + lens[i]] = x[starts[i]:starts[i + 1]]
        s.planes.append(full)
    s.new_rows = torch.tensor([s.starts[i] + lens[i] for i in range(n)], device=DEV) if step else None
    return s


def _append_inputs(case, seed):
    g, lens = _generator(seed), _lens(case)
    n = sum(lens)
    heads, kv, dim = case["heads"], case["kv_heads"], case["dim"]
    # the rows of one joined projection, as it leaves the product: queries, keys, values of a token side by side
    joined = _normal(g, (n, (heads + 2 * kv) * dim), case["act"])
    pos = torch.from_numpy(np.concatenate([np.arange(case["first"], case["first"] + length) for length in lens]).astype(np.int32)).to(DEV)
    preds = [case["first"] + length for length in lens]
    return lens, preds, joined, pos, _rotation_inputs(case, g, n, pos)


def _split(case, joined):
    heads, kv, dim = case["heads"], case["kv_heads"], case["dim"]
    n = joined.shape[0]
    return (joined[:, :heads * dim].view(n, heads, dim), joined[:, heads * dim:(heads + kv) * dim].view(n, kv, dim),
            joined[:, (heads + kv) * dim:].view(n, kv, dim))


def _prepare_append(s, case, seed):
    lens, preds, s.joined, s.pos, (s.rot_pos, axis, s.inv_freq, s.weights) = _append_inputs(case, seed)
    s.q, s.k, s.v = _split(case, s.joined)
    n = s.joined.shape[0]
    s.q_out = torch.zeros(s.q.shape, dtype=s.q.dtype, device=DEV)
    s.k_row, s.v_row = [torch.zeros(s.k.shape, dtype=s.k.dtype, device=DEV) for _ in range(2)]
    at = _offsets(case, preds)
    if own:
        s3, _ids, offs = _arena(s, case, preds)
        s.rule = s3.make_rotary(case["rotary"], s.inv_freq, interleaved=case["interleaved"], n_axes=case["axes"],
                                axis_of_pair=axis if case["axes"] > 1 else None, q_weight=s.weights[0], k_weight=s.weights[1], eps=1e-6)
        s.slot_off = torch.from_numpy(np.repeat(offs, lens)).to(DEV)
        if case["cache"] == case["act"]:
            s.cache = s.memory.view(_TORCH[case["act"]]).view(2, sum(s.caps), case["kv_heads"], case["dim"])
        return s
    s.axis = torch.from_numpy(axis.astype(np.int64)).to(DEV)
    s.rows = torch.from_numpy(np.repeat(at[:-1], lens)).to(DEV) + s.pos.long()
    if case["cache"] == "mxfp4":
        s.planes = [[torch.zeros((int(at[-1]), case["kv_heads"], case["dim"] // d), dtype=torch.uint8, device=DEV) for d in (2, 32)]
                    for _ in range(2)]
    else:
        dtype = torch.float8_e4m3fn if case["cache"] == "e4m3" else _TORCH[case["act"]]
        s.cache = torch.zeros((2, int(at[-1]), case["kv_heads"], case["dim"]), dtype=dtype, device=DEV)
    return s


def _rotate_inputs(case, seed):
    g, n = _generator(seed), case["tokens"]
    joined = _normal(g, (n, (case["heads"] + 2 * case["kv_heads"]) * case["dim"]), case["act"])
    pos = torch.randint(0, 131072, (n,), generator=g, device=DEV, dtype=torch.int32)
    return joined, _rotation_inputs(case, g, n, pos)


def _prepare_rotate(s, case, seed):
    s.joined, (s.rot_pos, axis, s.inv_freq, s.weights) = _rotate_inputs(case, seed)
    s.q, s.k, _v = _split(case, s.joined)
    if own:
        from paper_2306_06000_amd import binding as s3

        s.dtype = {"f16": s3.S3_F16, "bf16": s3.S3_BF16}[case["act"]]
        s.rule = s3.make_rotary(case["rotary"], s.inv_freq, interleaved=case["interleaved"], n_axes=case["axes"],
                                axis_of_pair=axis if case["axes"] > 1 else None, q_weight=s.weights[0], k_weight=s.weights[1], eps=1e-6)
        s.joined_out = torch.zeros_like(s.joined)
        s.q_out, s.k_out, _v = _split(case, s.joined_out)
    else:
        s.axis = torch.from_numpy(axis.astype(np.int64)).to(DEV)
    return s


# ---- one pass ------------------------------------------------------------------------------------------------------


def run(s):
    return (_run_own if own else _run_plain)(s, s.case)


def _run_own(s, case):
    from paper_2306_06000_amd import binding as s3

    stream = torch.cuda.current_stream().cuda_stream
    op, heads, kv, dim = case["op"], case["heads"], case["kv_heads"], case["dim"]
    width = (heads + 2 * kv) * dim
    if op == "attend":
        s3.check(s3.s3_decode_attention(s.arena, 0, case["batch"], s.q, s.slot_off, s.pos, s.out, s.code[case["out"]], 0.0, stream), op)
        return {"out": s.out}
    if op == "step":
        s3.check(s3.s3_decode_step(s.arena, 0, case["batch"], s.slot_off, s.pos, s.q, s.k_new, s.v_new, s.out, s.code[case["out"]], 0.0,
                                   s.len, stream), op)
        s3.check(s3.s3_kv_fetch(s.arena, 0, case["batch"], s.slot_off, s.pos, s.k_row, s.v_row, stream), "s3_kv_fetch")
        return {"out": s.out, "len": s.len, "k_row": s.k_row, "v_row": s.v_row}
    if op == "append":
        n = s.joined.shape[0]
        s3.check(s3.s3_kv_append_rotary(s.arena, 0, n, s.slot_off, s.pos, s.rule, s.q, s.k, s.v, s.q_out, rot_pos=s.rot_pos,
                                        q_stride=width, k_stride=width, v_stride=width, stream=stream), op)
        if case["cache"] == case["act"]:
            return {"q": s.q_out, "cache": s.cache}
        s3.check(s3.s3_kv_fetch(s.arena, 0, n, s.slot_off, s.pos, s.k_row, s.v_row, stream), "s3_kv_fetch")
        return {"q": s.q_out, "k_row": s.k_row, "v_row": s.v_row}
    s3.check(s3.s3_qk_rotary(s.rule, s.dtype, dim, case["tokens"], s.rot_pos, s.q, heads, s.k, kv, s.q_out, s.k_out, q_stride=width,
                             k_stride=width, stream=stream), op)
    return {"q": s.q_out, "k": s.k_out}


def _norm_rotate(x, weight, case, cos, sin):
    """x [n][heads][dim] -> its norms and rotation in 32 bits."""
    x = x.float()
    if weight is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6) * weight
    r = case["rotary"]
    turned, rest = x[..., :r], x[..., r:]
    a, b = (turned[..., 0::2], turned[..., 1::2]) if case["interleaved"] else (turned[..., :r // 2], turned[..., r // 2:])
    pair = (a * cos - b * sin, a * sin + b * cos)
    turned = torch.stack(pair, -1).flatten(-2) if case["interleaved"] else torch.cat(pair, -1)
    return torch.cat((turned, rest), -1)


def _angles(s):
    # far positions: angles in 64 bits
    angle = s.rot_pos.double()[s.axis].t() * s.inv_freq.double()
    return angle.cos().float().unsqueeze(1), angle.sin().float().unsqueeze(1)


def _run_plain(s, case):
    op, act = case["op"], _TORCH[case["act"]]
    if op in ("append", "rotate"):
        cos, sin = _angles(s)
        q = _norm_rotate(s.q, s.weights[0], case, cos, sin).to(act)
        k = _norm_rotate(s.k, s.weights[1], case, cos, sin)
        if op == "rotate":
            return {"q": q, "k": k.to(act)}
        if case["cache"] == "mxfp4":
            back = []
            for (codes, scales), x in zip(s.planes, (k, s.v.float())):
                codes[s.rows], scales[s.rows] = _to_blocks(x, case["act"])
                back.append(_from_blocks(codes[s.rows], scales[s.rows]).to(act))
            return {"q": q, "k_row": back[0], "v_row": back[1]}
        if case["cache"] == "e4m3":
            bits = s.cache.view(torch.uint8)
            for plane, x in zip(bits, (k, s.v.float())):
                plane[s.rows] = _to_e4m3(x).to(torch.float8_e4m3fn).view(torch.uint8)
            back = [plane[s.rows].view(torch.float8_e4m3fn).to(act) for plane in bits]
            return {"q": q, "k_row": back[0], "v_row": back[1]}
        s.cache[0][s.rows], s.cache[1][s.rows] = k.to(act), s.v
        return {"q": q, "cache": s.cache}

    heads, kv, dim = case["heads"], case["kv_heads"], case["dim"]
    step = op == "step"
    back = []
    if step:
        for (codes, scales), x in zip(s.planes, (s.k_new, s.v_new)):
            codes[s.new_rows], scales[s.new_rows] = _to_blocks(x.float(), case["act"])
            back.append(_from_blocks(codes[s.new_rows], scales[s.new_rows]).to(act))
    out = torch.empty_like(s.out)
    for b, (start, length) in enumerate(zip(s.starts, s.lens)):
        end = start + length + (1 if step else 0)
        k, v = [_from_blocks(codes[start:end], scales[start:end]).transpose(0, 1).contiguous() for codes, scales in s.planes]
        scores = torch.matmul(s.q[b].float().view(kv, heads // kv, dim), k.transpose(1, 2).contiguous()) / math.sqrt(dim)
        weights = torch.exp(scores - scores.amax(-1, keepdim=True))
        out[b] = (torch.matmul(weights, v) / weights.sum(-1, keepdim=True)).view(heads, dim)
    return {"out": out, "len": s.pos + 1, "k_row": back[0], "v_row": back[1]} if step else {"out": out}


# ---- the definition in 64 bits ---------------------------------------------------------------------------------------


def _exact_blocks(x, act):
    """What a block of 32 numbers is held as, by a search over the values that a code can stand for."""
    values = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device=x.device)
    b = x.double().unflatten(-1, (-1, 32))
    most = b.abs().amax(-1, keepdim=True)
    fraction, exponent = torch.frexp(most)  # most = fraction * 2^exponent, fraction in [0.5, 1)
    power = exponent - 3 + (fraction >= 0.875).int()
    power = torch.where(most == 0, -126, power).clamp(-126, _LARGEST[act] - 127)
    unit = _power(power, torch.float64)
    y = (b / unit).abs()
    best = torch.full_like(y, 100.0)
    held = torch.zeros_like(y)
    for k in (0, 2, 4, 6, 1, 3, 5, 7):  # even codes first: a tie stays with them
        off = (y - values[k]).abs()
        held = torch.where(off < best, values[k], held)
        best = torch.minimum(best, off)
    return (held * unit * torch.where(b < 0, -1.0, 1.0)).flatten(-2)


def _exact_rotation(x, weight, case, angle):
    x = x.double()
    if weight is not None:
        x = x / torch.sqrt(x.pow(2).sum(-1, keepdim=True) / case["dim"] + 1e-6) * weight.double()
    half = case["rotary"] // 2
    first = torch.arange(half, device=x.device) * (2 if case["interleaved"] else 1)
    second = first + (1 if case["interleaved"] else half)
    y = x.clone()
    c, s = torch.cos(angle)[:, None], torch.sin(angle)[:, None]
    y[..., first] = x[..., first] * c - x[..., second] * s
    y[..., second] = x[..., second] * c + x[..., first] * s
    return y


def exact(case, seed):
    if case["op"] in ("append", "rotate"):
        if case["op"] == "append":
            lens, preds, joined, pos, (rot_pos, axis, inv_freq, weights) = _append_inputs(case, seed)
        else:
            joined, (rot_pos, axis, inv_freq, weights) = _rotate_inputs(case, seed)
        q, k, v = _split(case, joined)
        angle = torch.stack([rot_pos[int(a)].double() * f for a, f in zip(axis, inv_freq.double())], -1)
        q, k = _exact_rotation(q, weights[0], case, angle), _exact_rotation(k, weights[1], case, angle)
        if case["op"] == "rotate":
            return {"q": q, "k": k}
        if case["cache"] == "mxfp4":
            return {"q": q, "k_row": _exact_blocks(k, case["act"]), "v_row": _exact_blocks(v, case["act"])}
        if case["cache"] == "e4m3":
            held = []
            for x in (k, v.double()):  # three fraction bits, a least exponent of -6, none beyond 448
                step = _power((torch.frexp(x)[1] - 1).clamp(min=-6) - 3, torch.float64)
                held.append((torch.round(x / step) * step).clamp(-448, 448))
            return {"q": q, "k_row": held[0], "v_row": held[1]}
        at = _offsets(case, preds)
        cache = torch.zeros((2, int(at[-1]), case["kv_heads"], case["dim"]), dtype=torch.float64, device=DEV)
        begin = 0
        for i, length in enumerate(lens):
            row = int(at[i]) + case["first"]
            cache[0, row:row + length], cache[1, row:row + length] = k[begin:begin + length], v[begin:begin + length].double()
            begin += length
        return {"q": q, "cache": cache}

    lens, k, v, q, k_new, v_new = _attention_inputs(case, seed)
    heads, kv, dim = case["heads"], case["kv_heads"], case["dim"]
    step = case["op"] == "step"
    rows = [_exact_blocks(k_new, case["act"]), _exact_blocks(v_new, case["act"])] if step else [None, None]
    out = torch.empty((case["batch"], heads, dim), dtype=torch.float64, device=DEV)
    at = 0
    for b, length in enumerate(lens):
        both = []
        for (codes, scales), new in zip((k, v), rows):
            c = torch.stack((codes[at:at + length] % 16, codes[at:at + length] // 16), -1).flatten(-2)
            kind = (c % 8).double()  # 0 and 0.5 below 2, then two values to a power of two
            x = torch.where(kind < 2, kind / 2, (1 + (kind % 2) / 2) * 2 ** (torch.floor(kind / 2) - 1))
            x = torch.where(c >= 8, -x, x) * _power(scales[at:at + length].int() - 127, torch.float64).repeat_interleave(32, -1)
            both.append((torch.cat([x, new[b:b + 1]]) if step else x).permute(1, 0, 2).contiguous())
        scores = torch.matmul(q[b].double().view(kv, heads // kv, dim), both[0].transpose(1, 2).contiguous()) * dim ** -0.5
        out[b] = torch.matmul(torch.softmax(scores, -1), both[1]).view(heads, dim)
        at += length
    if not step:
        return {"out": out}
    return {"out": out, "len": None, "k_row": rows[0], "v_row": rows[1]}
