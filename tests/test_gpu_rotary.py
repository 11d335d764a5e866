"""Norms, rotation and append in one pass on the GPU, through the C ABI, against plain 64-bit forms.

Tolerance.  An output is x * inv * w turned by an angle: the norm's sum of squares is a tree of at most 13 roundings, with the root,
the quotient and two products below 13 * 2^-24; the sine and cosine are off by 2^-25 * 2 pi (the turn in 32 bits) and 2^-23 of
arithmetic; two products and a sum: together below 2^-19 of |a| + |b|.  Then one rounding to the output's type, or to a code."""
import os

import numpy as np
import pytest

from paper_2306_06000_amd import binding as s3
from tests import fp4_plain as plain

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
DEV = "cuda:0"
TDT = {0: torch.float16, 1: torch.bfloat16}


@pytest.fixture(scope="module", autouse=True)
def need_gpu_and_lib():
    assert torch.cuda.is_available(), "these tests need a GPU"
    assert os.path.exists(s3.LIB_PATH), "libs3kv.so must be built before the GPU tests run"
    s3.lib()


def close(got, want, mag, act, what=""):
    got = got.double().cpu().numpy()
    tol = 2.0 ** -19 * mag + plain.HALF_STEP[act] * (np.abs(want) + 2.0 ** -19 * mag) + (2.0 ** -25 if act == 0 else 0.0)
    off = np.abs(got - want)
    assert (off <= tol).all(), (what, float((off / np.maximum(tol, 1e-300)).max()))


class Inputs:
    def __init__(self, heads, kv, d, act, n, rotary, interleaved, axes, norm, seed=0, far=1 << 20):
        self.heads, self.kv, self.d, self.act, self.n = heads, kv, d, act, n
        self.rotary, self.interleaved = rotary, interleaved
        rng = np.random.default_rng([seed, heads, kv, d, n, rotary])
        joined = torch.from_numpy(rng.standard_normal((n, (heads + 2 * kv) * d)) * np.exp(rng.uniform(-3, 3, (n, 1)))).to(TDT[act])
        self.width = joined.shape[1]
        self.joined = joined.to(DEV)
        self.q, self.k, self.v = self.split(self.joined)
        self.q64, self.k64, self.v64 = (x.double().numpy() for x in self.split(joined))
        self.rot = rng.integers(-far, far, (axes, n)).astype(np.int32)
        inv = (1e4 ** (-rng.uniform(0, 1, rotary // 2))).astype(np.float32)
        self.axis = rng.integers(0, axes, rotary // 2)
        self.wq, self.wk = ((1 + 0.3 * rng.standard_normal(d)).astype(np.float32) if norm else None for _ in range(2))
        self.inv64 = inv.astype(np.float64)
        up = lambda x: None if x is None else torch.from_numpy(x).to(DEV)
        self.rule = s3.make_rotary(rotary, up(inv), interleaved, axes, self.axis if axes > 1 else None, up(self.wq), up(self.wk), 1e-5)
        self.rot_d = up(self.rot)

    def split(self, x):
        n, h, kv, d = x.shape[0], self.heads, self.kv, self.d
        return x[:, :h * d].view(n, h, d), x[:, h * d:(h + kv) * d].view(n, kv, d), x[:, (h + kv) * d:].view(n, kv, d)

    def want(self, rot=None):
        rot = self.rot if rot is None else rot
        angle = rot[self.axis].T.astype(np.float64) * self.inv64 if self.rotary else np.zeros((self.n, 0))
        eps = float(np.float32(1e-5))
        return (plain.rotate(self.q64, self.wq, self.rotary, self.interleaved, angle, eps),
                plain.rotate(self.k64, self.wk, self.rotary, self.interleaved, angle, eps))


CASES = [(32, 8, 128, 128, False, 1, True), (16, 16, 256, 64, True, 1, False), (12, 12, 128, 128, False, 3, True), (8, 1, 64, 64, False, 2, False),
         (7, 7, 64, 32, False, 1, True), (6, 3, 256, 256, False, 4, True), (64, 64, 96, 96, False, 1, True), (4, 2, 96, 40, True, 2, False),
         (5, 5, 128, 36, False, 1, True), (3, 1, 64, 2, False, 1, False), (2, 2, 256, 254, False, 2, True), (4, 4, 128, 126, True, 3, True),
         (4, 1, 128, 0, False, 1, True), (9, 3, 64, 0, False, 1, False), (1, 1, 128, 128, True, 1, True), (20, 1, 128, 96, False, 1, True)]


@pytest.mark.parametrize("act", [0, 1], ids=["f16", "bf16"])
@pytest.mark.parametrize("case", CASES, ids=str)
def test_queries_and_keys(case, act):
    heads, kv, d, rotary, interleaved, axes, norm = case
    for n in (1, 3, 37, 5000 // (heads + kv)):
        x = Inputs(heads, kv, d, act, n, rotary, interleaved, axes, norm, seed=n)
        (q64, qm), (k64, km) = x.want()
        out = torch.full_like(x.joined, 9.0)
        qo, ko, vo = x.split(out)
        keep = x.joined.clone()
        assert s3.s3_qk_rotary(x.rule, act, d, n, x.rot_d, x.q, heads, x.k, kv, qo, ko, x.width, x.width) == 0
        close(qo, q64, qm, act, (case, n, "q"))
        close(ko, k64, km, act, (case, n, "k"))
        assert (vo == 9).all() and torch.equal(x.joined, keep)
        # dense, and only one of the two
        q, k = x.q.contiguous(), x.k.contiguous()
        q1, k1 = torch.empty_like(q), torch.empty_like(k)
        assert s3.s3_qk_rotary(x.rule, act, d, n, x.rot_d, q, heads, None, kv, q1, None) == 0
        assert s3.s3_qk_rotary(x.rule, act, d, n, x.rot_d, None, 0, k, kv, None, k1) == 0
        assert torch.equal(q1, qo) and torch.equal(k1, ko)
        # in place
        assert s3.s3_qk_rotary(x.rule, act, d, n, x.rot_d, x.q, heads, x.k, kv, x.q, x.k, x.width, x.width) == 0
        assert torch.equal(x.q, qo) and torch.equal(x.k, ko) and torch.equal(x.v.double().cpu(), torch.from_numpy(x.v64))


def test_norm_of_extremes():
    """A head of zeros stays zero, one of the largest numbers overflows no further than its sum of squares does in 32 bits."""
    x = Inputs(4, 1, 128, 1, 2, 128, False, 1, True)
    q = torch.zeros((2, 4, 128), dtype=torch.bfloat16, device=DEV)
    q[1, 1] = 2.0 ** 50
    q[1, 2] = 2.0 ** -60
    out = torch.empty_like(q)
    assert s3.s3_qk_rotary(x.rule, 1, 128, 2, x.rot_d, q, 4, None, 0, out, None) == 0
    assert (out[0] == 0).all() and torch.isfinite(out).all()
    bad = q.clone()
    bad[0, 0, 3] = float("nan")
    assert s3.s3_qk_rotary(x.rule, 1, 128, 2, x.rot_d, bad, 4, None, 0, out, None) == 0
    assert torch.isnan(out[0, 0]).all() and torch.isfinite(out[0, 1:]).all() and torch.isfinite(out[1]).all()


class Cache:
    def __init__(self, x, kv_dtype, preds, max_len=2048, granule=64):
        self.x, self.kv_dtype = x, kv_dtype
        cfg = s3.make_config(2, x.heads, x.d, kv_dtype, granule, max_len, 0 if x.heads == x.kv else x.kv, x.act)
        bpt = s3.s3_kv_bytes_per_token(cfg)
        self.N = sum(s3.s3_kv_capacity_for(cfg, p) for p in preds)
        self.row = bpt // 4
        self.mem = torch.full((self.N * bpt,), 0x33, dtype=torch.uint8, device=DEV)
        st, self.a = s3.s3_kv_arena_init(cfg, self.mem, self.mem.numel())
        assert st == 0
        rc, self.ids, self.offs, _ = s3.s3_kv_alloc(self.a, preds)
        assert rc == len(preds)

    def rows(self):
        """The arena as stored rows [layers][2][N][row] (4-bit rows: codes and scales lie in planes of their own)."""
        codes = self.x.kv * self.x.d // 2 if self.kv_dtype == s3.S3_MXFP4 else self.row
        cut = 4 * self.N * codes
        parts = [self.mem[:cut].view(2, 2, self.N, codes), self.mem[cut:].view(2, 2, self.N, self.row - codes)]
        return torch.cat(parts, -1).cpu().numpy()

    def fetch(self, layer, off, pos):
        k, v = (torch.full((len(pos), self.x.kv, self.x.d), 7.0, dtype=TDT[self.x.act], device=DEV) for _ in range(2))
        assert s3.s3_kv_fetch(self.a, layer, len(pos), off, pos, k, v) == 0
        return k, v

    def close(self):
        torch.cuda.synchronize()
        s3.s3_kv_arena_destroy(self.a)


def check_keys(got, raw, want, mag, kv_dtype, act, kv, d):
    """Stored keys against the exact ones: off by 32-bit arithmetic and by half the distance between two codes."""
    tol = 2.0 ** -19 * mag
    if kv_dtype in (s3.S3_F16, s3.S3_BF16):
        return close(got, want, mag, act)
    got = got.double().cpu().numpy()
    if kv_dtype == s3.S3_E4M3:
        small = np.clip(want, -448, 448)
        step = 2.0 ** (np.maximum(np.floor(np.log2(np.maximum(np.abs(small), 2.0 ** -30))), -6) - 3)
        assert (np.abs(got - small) <= step * (0.5 + 2.0 ** -20) + 2 * tol).all()
        return None
    n = want.shape[0]
    scale = 2.0 ** (raw[:, kv * d // 2:kv * (d // 2 + d // 32)].reshape(n, kv, d // 32).astype(np.float64) - 127)
    most = np.abs(want).reshape(n, kv, d // 32, 32).max(-1)
    t = tol.reshape(n, kv, d // 32, 32).max(-1)
    assert ((most - t < 7 * scale) & ((most + t >= 3.5 * scale) | (scale == 2.0 ** -126))).all()
    s = scale.repeat(32, -1)
    y = np.abs(want) / s
    half = np.where(y < 2, 0.25, np.where(y < 4, 0.5, 1.0))
    assert (np.abs(got - want) <= s * half + 2 * tol).all()


@pytest.mark.parametrize("act", [0, 1], ids=["f16", "bf16"])
@pytest.mark.parametrize("kv_dtype", ["own", s3.S3_E4M3, s3.S3_MXFP4], ids=["16bit", "e4m3", "mxfp4"])
@pytest.mark.parametrize("case", CASES, ids=str)
def test_append(case, kv_dtype, act):
    """A mix of prompts, single tokens and padding: rows, queries, and nothing else."""
    heads, kv, d, rotary, interleaved, axes, norm = case
    kv_dtype = act if kv_dtype == "own" else kv_dtype
    if d == 96 and (kv_dtype != act or kv != heads):
        pytest.skip("heads of 96: multi-head 16-bit caches only")
    runs = [(0, 40), (700, 1), (3, 1), (0, 130), (63, 2), (0, 1)]  # (first row, rows) of each sequence
    n = sum(r for _, r in runs) + 3
    x = Inputs(heads, kv, d, act, n, rotary, interleaved, axes, norm, seed=5)
    c = Cache(x, kv_dtype, [f + r for f, r in runs])
    off = np.concatenate([np.repeat(c.offs, [r for _, r in runs]), [-1, -1, 0]])
    pos = np.concatenate([np.arange(f, f + r) for f, r in runs] + [[0, 5, 2048]]).astype(np.int32)
    mix = np.random.default_rng(1).permutation(n)  # (rows in any order)
    off, pos = off[mix], pos[mix]
    off_d, pos_d = torch.from_numpy(off.astype(np.int64)).to(DEV), torch.from_numpy(pos).to(DEV)
    live = (off >= 0) & (pos < 2048)
    before = c.rows()
    for rot in (x.rot_d, None):
        (q64, qm), (k64, km) = x.want(None if rot is not None else np.repeat(pos[None], axes, 0))
        q_out = torch.full((n, heads, d), 9.0, dtype=TDT[act], device=DEV)
        assert s3.s3_kv_append_rotary(c.a, 1, n, off_d, pos_d, x.rule, x.q, x.k, x.v, q_out, rot, x.width, x.width, x.width) == 0
        torch.cuda.synchronize()
        close(q_out[torch.from_numpy(live)], q64[live], qm[live], act, case)
        assert (q_out[torch.from_numpy(~live)] == 9).all()
        after = c.rows()
        at = (off + pos)[live]
        k, v = c.fetch(1, off_d, pos_d)
        assert (k[torch.from_numpy(~live)] == 7).all()
        check_keys(k[torch.from_numpy(live)], after[1, 0][at], k64[live], km[live], kv_dtype, act, kv, d)
        # values: what s3_kv_append writes, bit for bit
        other = Cache(x, kv_dtype, [f + r for f, r in runs])
        assert s3.s3_kv_append(other.a, 1, n, off_d, pos_d, x.k.contiguous(), x.v.contiguous()) == 0
        torch.cuda.synchronize()
        plane = other.rows()
        assert np.array_equal(after[1, 1], plane[1, 1])
        untouched = np.ones(c.N, bool)
        untouched[at] = False
        assert np.array_equal(after[1, 0][untouched], before[1, 0][untouched]) and np.array_equal(after[0], before[0])
        if rotary == 0 and not norm:
            assert np.array_equal(after, plane)
        if kv_dtype == s3.S3_MXFP4:
            assert np.array_equal(after[1, 0][at][:, kv * (d // 2 + d // 32):], np.zeros((len(at), c.row - kv * (d // 2 + d // 32)), np.uint8))
        other.close()
    c.close()


def test_keys_alone_in_place_and_refusals():
    x = Inputs(8, 2, 128, 1, 4, 128, False, 1, True)
    c = Cache(x, s3.S3_BF16, [64] * 4)
    off = torch.from_numpy(c.offs).to(DEV)
    pos = torch.tensor([1, 2, 3, 4], dtype=torch.int32, device=DEV)
    q, k, v = x.q.contiguous(), x.k.contiguous(), x.v.contiguous()
    q_out = torch.empty_like(q)
    call = lambda **kw: s3.s3_kv_append_rotary(**{**dict(arena=c.a, layer=0, n=4, slot_off=off, pos=pos, rule=x.rule, q=q, k_new=k, v_new=v, q_out=q_out), **kw})
    assert call() == 0 and call(n=0) == 0
    rows = c.fetch(0, off, pos)
    c.mem.fill_(0)
    assert call(q=None, q_out=None) == 0
    again = c.fetch(0, off, pos)
    assert torch.equal(rows[0], again[0]) and torch.equal(rows[1], again[1])
    same = q.clone()
    assert call(q=same, q_out=same) == 0
    assert torch.equal(same, q_out)
    before = c.mem.clone()
    bad = s3.S3_ERR_INVALID
    for kw in (dict(layer=2), dict(layer=-1), dict(n=-1), dict(rule=None), dict(slot_off=None), dict(pos=None), dict(k_new=None), dict(v_new=None),
               dict(q_out=None), dict(k_stride=248), dict(v_stride=257), dict(q_stride=1000), dict(q=x.q, q_out=x.q, q_stride=x.width),
               dict(k_new=k.data_ptr() + 8), dict(q_out=q_out.data_ptr() + 2), dict(rule=s3.make_rotary(130, 1 << 12)),
               dict(slot_id=c.ids, pos_host=[65, 0, 0, 0]), dict(slot_id=[99, 0, 1, 2], pos_host=[0, 0, 0, 0])):
        assert call(**kw) == bad, kw
    assert call(slot_id=c.ids, pos_host=[64, 1, 2, 3]) == s3.S3_ERR_SLOT_FULL
    assert s3.s3_kv_fetch(c.a, 0, 4, off, pos, None, None) == bad and s3.s3_kv_fetch(c.a, 2, 4, off, pos, k, v) == bad
    assert s3.s3_kv_fetch(c.a, 0, 4, off, pos, k.data_ptr() + 8, v) == bad and s3.s3_kv_fetch(c.a, 0, 0, None, None, None, None) == 0
    torch.cuda.synchronize()
    assert torch.equal(before, c.mem)
    c.close()


@pytest.mark.parametrize("kv_dtype", [s3.S3_BF16, s3.S3_E4M3, s3.S3_MXFP4], ids=["16bit", "e4m3", "mxfp4"])
def test_a_prompt_and_its_tokens_together(kv_dtype):
    """As a serving loop runs them, on a stream of its own and from a recorded graph: prompts in, then tokens one by one with the
    rotation in the append and attention over the rows; against 64-bit attention over the rows that the cache holds."""
    heads, kv, d, n = 16, 4, 128, 3
    prompts, steps = [50, 1, 131], 6
    x = Inputs(heads, kv, d, 1, sum(prompts), 128, False, 1, True, seed=2)
    c = Cache(x, kv_dtype, [p + steps for p in prompts])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    st = side.cuda_stream
    with torch.cuda.stream(side):
        off = torch.from_numpy(np.repeat(c.offs, prompts)).to(DEV)
        pos = torch.from_numpy(np.concatenate([np.arange(p) for p in prompts]).astype(np.int32)).to(DEV)
        q_all = torch.empty((sum(prompts), heads, d), dtype=torch.bfloat16, device=DEV)
        assert s3.s3_kv_append_rotary(c.a, 0, len(pos), off, pos, x.rule, x.q, x.k, x.v, q_all, None, x.width, x.width, x.width, st) == 0
        offs = torch.from_numpy(c.offs).to(DEV)
        at = torch.tensor(prompts, dtype=torch.int32, device=DEV)
        t = Inputs(heads, kv, d, 1, n, 128, False, 1, True, seed=3)
        q_out = torch.empty((n, heads, d), dtype=torch.bfloat16, device=DEV)
        out = torch.empty((n, heads, d), dtype=torch.float32, device=DEV)
        lens = at + 1

        def token():
            assert s3.s3_kv_append_rotary(c.a, 0, n, offs, at, t.rule, t.q, t.k, t.v, q_out, None, t.width, t.width, t.width, st) == 0
            assert s3.s3_decode_attention(c.a, 0, n, q_out, offs, lens, out, s3.S3_F32, 0.0, st) == 0

        assert s3.s3_kv_reserve_scratch(c.a, n) == 0
        token()
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            token()
        for step in range(steps):
            at.copy_(torch.tensor(prompts, dtype=torch.int32) + step)
            lens.copy_(at + 1)
            t.joined.copy_(torch.randn_like(t.joined))
            graph.replay()
            side.synchronize()
            for b in range(n):
                rows = torch.arange(prompts[b] + step + 1, dtype=torch.int32, device=DEV)
                k, v = c.fetch(0, torch.full((len(rows),), int(c.offs[b]), dtype=torch.int64, device=DEV), rows)
                torch.cuda.synchronize()
                want, bound = plain.attention(*(y.double().cpu().numpy() for y in (q_out[b], k, v)))
                # (8-bit rows of shared heads are attended over with weights in two 16-bit parts of bf16)
                parts = 0.0 if kv_dtype == s3.S3_MXFP4 else 2.0 ** -16 * v.double().abs().amax(0).cpu().numpy().repeat(heads // kv, 0)
                assert (np.abs(out[b].double().cpu().numpy() - want) <= plain.allowed(want, bound, 0.0, 2) + parts).all()
    c.close()


def test_a_long_prompt_and_far_positions():
    x = Inputs(8, 2, 128, 1, 20000, 128, False, 2, True, far=(1 << 31) - 1)
    (q64, qm), (k64, km) = x.want()
    qo, ko = torch.empty_like(x.q.contiguous()), torch.empty_like(x.k.contiguous())
    assert s3.s3_qk_rotary(x.rule, 1, 128, x.n, x.rot_d, x.q.contiguous(), 8, x.k.contiguous(), 2, qo, ko) == 0
    # (a turn of 2^31 positions is off by 2^-53 * 2^31 of itself, far below 2^-25)
    close(qo, q64, qm, 1)
    close(ko, k64, km, 1)
