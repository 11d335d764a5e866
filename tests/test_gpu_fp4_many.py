"""4-bit rows in batches of many contexts, which equal shares of all rows serve: every layout of heads, lengths that share borders cut in
every way, steps, blocks that are NaN, scales that fp16 does not hold, recorded graphs; against plain 64-bit forms."""
import numpy as np
import pytest

from paper_2306_06000_amd import binding as s3
from tests import fp4_plain as plain
from tests.test_gpu_fp4 import DEV, Rig, need_gpu_and_lib, numbers  # noqa: F401  (the fixture holds here too)

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


class Many(Rig):
    """Contexts whose rows are windows of one pool of stored rows."""

    def fill(self, lens, layer=0, spread=0.5, pool=None):
        longest = max(max(lens), 1)
        if pool is None:
            pool = [plain.to_rows(numbers(self.rng, (longest + 97, self.kv, self.d), self.act, spread)[1], self.act) for _ in range(2)]
        wide = [plain.from_rows(p, self.kv, self.d) for p in pool]
        dev = [torch.from_numpy(p).to(DEV) for p in pool]
        self.k, self.v = [], []
        for i, (sid, L) in enumerate(zip(self.ids.tolist(), lens)):
            at = i * 13 % 97
            if L:
                assert s3.s3_kv_fill(self.a, sid, layer, 0, L, dev[0][at:at + L], dev[1][96 - at:96 - at + L], self.stream) == 0
            self.k.append(wide[0][at:at + L])
            self.v.append(wide[1][96 - at:96 - at + L])
        torch.cuda.synchronize()

    def check_some(self, out, q64, lens, out_dtype, which, scale=None, what=""):
        kept = self.k, self.v
        self.k, self.v = ([x[i] for i in which] for x in kept)
        self.check(out[torch.tensor(which, device=DEV)], q64[which], [lens[i] for i in which], out_dtype, scale, what)
        self.k, self.v = kept


def some(lens, n=40):
    """The longest, the empty ones, and n spread over the batch."""
    order = np.argsort(lens, kind="stable")
    return sorted({int(order[-1]), int(order[-2]), int(order[0]), *np.linspace(0, len(lens) - 1, n).astype(int).tolist()})


# contexts times columns of 256 elements: at least three a compute unit, five with heads of 256
MANY = [((16, 16, 256), 81), ((16, 1, 256), 1300), ((34, 2, 256), 330), ((32, 8, 128), 200), ((3, 3, 128), 400), ((12, 12, 128), 130), ((20, 1, 128), 400),
        ((16, 16, 64), 200), ((7, 7, 64), 400), ((24, 3, 64), 400), ((20, 1, 64), 400), ((5, 5, 64), 400), ((8, 1, 64), 1200)]


@pytest.mark.parametrize("act", [0, 1], ids=["f16", "bf16"])
@pytest.mark.parametrize("shape,n", MANY, ids=str)
def test_many_contexts(shape, n, act):
    """Contexts of up to 8 tiles (none is cut), of up to 40, and one long one among short ones."""
    rng = np.random.default_rng([n, act])
    short = rng.integers(0, 257, n)
    mixed = np.where(rng.random(n) < 0.7, rng.integers(0, 200, n), rng.integers(200, 1281, n))
    alone = rng.integers(0, 40, n)
    mixed[n // 2], alone[n // 3], short[n - 1] = 1280, 5003, 0
    # (every kind needs the capacities of its own lengths)
    for lens in (short.tolist(), mixed.tolist(), alone.tolist()):
        rig = Many(*shape, act, [max(L, 1) for L in lens], max_len=8192)
        rig.fill(lens)
        q, q64 = numbers(rig.rng, (n, rig.heads, rig.d), act, 0.5)
        first = rig.attend(q, lens)
        rig.check_some(first, q64, lens, 2, some(lens), what=shape)
        rig.check_some(rig.attend(q, lens, act), q64, lens, act, some(lens, 10), what=shape)
        assert torch.isfinite(first).all()
        assert (first[rig.lens_d(lens) == 0] == 0).all()
        for sync in (1, 0):  # the order in which pieces meet does not show
            assert s3.s3_kv_set_param(rig.a, "merge_sync", sync) == 0
            assert torch.equal(first, rig.attend(q, lens))
        rig.close()


@pytest.mark.parametrize("shape,n,act", [((16, 16, 256), 90, 0), ((32, 8, 128), 200, 1), ((3, 3, 128), 400, 0), ((7, 7, 64), 400, 1), ((20, 1, 64), 400, 1),
                                         ((8, 1, 64), 1200, 0)], ids=str)
def test_step_is_append_and_attention_of_many(shape, n, act):
    """Bit for bit, with entries that are refused among the others; the new lengths; nothing else of the arena."""
    rng = np.random.default_rng(n)
    pos = rng.integers(0, 700, n)
    pos[:40] = np.arange(24, 64)
    pos = pos.tolist()
    one, two = (Many(*shape, act, [p + 1 for p in pos], seed=3) for _ in range(2))
    (q, q64), (k, k64), (v, v64) = (numbers(rng, (n, h, one.d), act, 1.0) for h in (one.heads, one.kv, one.kv))
    refused = [41, n - 2]
    outs = []
    for rig in (one, two):
        rig.fill(pos)
        off = rig.off_d.clone()
        off[refused[0]] = -1
        p = rig.lens_d(pos)
        p[refused[1]] = -1
        if rig is one:
            out = torch.full((n, rig.heads, rig.d), float("nan"), dtype=torch.float32, device=DEV)
            new = torch.full((n,), -7, dtype=torch.int32, device=DEV)
            assert s3.s3_decode_step(rig.a, 0, n, off, p, q, k, v, out, 2, 0.0, new, rig.stream) == 0
            torch.cuda.synchronize()
            assert torch.equal(new, p + 1)
        else:
            assert s3.s3_kv_append(rig.a, 0, n, off, p, k, v, rig.stream) == 0
            lens = [x + 1 for x in pos]
            lens[refused[1]] = 0
            out = rig.attend(q, lens, off=off)
        outs.append(out)
    assert torch.equal(one.mem, two.mem)
    assert torch.equal(outs[0], outs[1])
    assert (outs[0][refused] == 0).all()
    for i in range(n):
        one.k[i] = np.concatenate([one.k[i], plain.from_rows(plain.to_rows(k64[i:i + 1], act), one.kv, one.d)])
        one.v[i] = np.concatenate([one.v[i], plain.from_rows(plain.to_rows(v64[i:i + 1], act), one.kv, one.d)])
    one.check_some(outs[0], q64, [x + 1 for x in pos], 2, [i for i in range(44) if i not in refused])
    one.close()
    two.close()


@pytest.mark.parametrize("act", [0, 1], ids=["f16", "bf16"])
@pytest.mark.parametrize("shape,n", [((7, 7, 64), 400), ((24, 3, 64), 400), ((3, 3, 128), 400), ((16, 16, 64), 200), ((4, 4, 256), 330)], ids=str)
def test_a_block_that_is_nan_stays_with_its_head_in_many(shape, n, act):
    """A key block: its head's queries; a value block: its 32 elements; other heads and other contexts keep their numbers."""
    heads, kv, d = shape
    rng = np.random.default_rng(7)
    lens = rng.integers(1, 500, n).tolist()
    sick = 11
    lens[sick] = 300
    rig = Many(*shape, act, lens)
    rig.fill(lens)
    q, q64 = numbers(rig.rng, (n, heads, d), act)
    clean = rig.attend(q, lens)
    rows = [plain.to_rows(x[sick], act) for x in (rig.k, rig.v)]
    group = heads // kv
    others = torch.arange(n, device=DEV) != sick
    for which, head, row in ((0, kv - 1, 299), (1, 1, 3), (0, 1, 40), (1, kv - 1, 150)):
        now = [r.copy() for r in rows]
        now[which][row, kv * d // 2 + head * (d // 32)] = 255
        kd, vd = (torch.from_numpy(r).to(DEV) for r in now)
        assert s3.s3_kv_fill(rig.a, int(rig.ids[sick]), 0, 0, 300, kd, vd, rig.stream) == 0
        got = rig.attend(q, lens)
        assert torch.equal(got[others], clean[others])
        bad = np.zeros((heads, d), bool)
        bad[head * group:(head + 1) * group, :d if which == 0 else 32] = True
        mine = got[sick].double().cpu().numpy()
        assert np.isnan(mine[bad]).all()
        want, bound = plain.attention(q64[sick], rig.k[sick], rig.v[sick])
        tol = plain.allowed(want, bound, np.abs(rig.v[sick]).max(0).repeat(group, 0), 2)
        assert (np.abs(mine - want)[~bad] <= tol[~bad]).all()
    rig.close()


@pytest.mark.parametrize("shape,n", [((8, 2, 128), 6), ((32, 8, 128), 200), ((8, 1, 64), 5), ((7, 7, 64), 400), ((16, 16, 256), 81)], ids=str)
@pytest.mark.parametrize("low,high,scale", [(118, 141, 2.0 ** -17), (60, 109, 2.0 ** 18), (100, 108, 2.0 ** 19), (138, 190, 2.0 ** -66)], ids=str)
def test_key_scales_at_and_beyond_the_ends_of_fp16(shape, n, low, high, scale):
    """fp16 queries, small ones among them, against blocks whose scales fp16 holds as normal numbers, below them, or not at all."""
    rng = np.random.default_rng([n, low])
    lens = rng.integers(1, 400, n).tolist()
    rig = Many(*shape, 0, lens)
    pool = [plain.to_rows(rng.standard_normal((500, rig.kv, rig.d)), 0) for _ in range(2)]
    cut = rig.kv * rig.d // 2
    pool[0][:, cut:cut + rig.kv * rig.d // 32] = rng.integers(low, high + 1, (500, rig.kv * rig.d // 32))
    rig.fill(lens, pool=pool)
    x = rng.standard_normal((n, rig.heads, rig.d))
    x[::3, :, ::2] *= 2.0 ** -16  # below the normal numbers of fp16
    t = torch.from_numpy(x).to(torch.float16)
    out = rig.attend(t.to(DEV), lens, 2, scale)
    rig.check_some(out, t.double().numpy(), lens, 2, some(lens, 20) if n > 20 else list(range(n)), scale)
    rig.close()


def test_replayed_graphs_of_many():
    """Steps and attention, recorded, replayed between eager work of other batches."""
    shape, n = (32, 8, 128), 200
    rng = np.random.default_rng(5)
    pos = rng.integers(0, 900, n).tolist()
    rig = Many(*shape, 1, [p + 1 for p in pos])
    rig.fill(pos)
    (q, _), (k, _), (v, _) = (numbers(rig.rng, (n, h, 128), 1) for h in (32, 8, 8))
    p, lens = rig.lens_d(pos), rig.lens_d([x + 1 for x in pos])
    assert s3.s3_kv_reserve_scratch(rig.a, n) == 0
    want = torch.empty((n, 32, 128), dtype=torch.bfloat16, device=DEV)
    assert s3.s3_decode_step(rig.a, 0, n, rig.off_d, p, q, k, v, want, 1, 0.0, None, rig.stream) == 0
    torch.cuda.synchronize()
    outs = [torch.empty_like(want) for _ in range(3)]
    side = torch.cuda.Stream()
    graphs = []
    with torch.cuda.stream(side):
        for i in range(3):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=side):
                if i < 2:
                    step = (s3.s3_decode_step, s3.s3_decode_step_static)[i]
                    assert step(rig.a, 0, n, rig.off_d, p, q, k, v, outs[i], 1, 0.0, None, side.cuda_stream) == 0
                else:
                    assert s3.s3_decode_attention(rig.a, 0, n, q, rig.off_d, lens, outs[i], 1, 0.0, side.cuda_stream) == 0
            graphs.append(g)
    torch.cuda.synchronize()
    few = [x + 1 for x in pos[:3]]
    first = rig.attend(q[:3].contiguous(), few, 1, off=rig.off_d[:3])
    for _ in range(4):
        for g, out in zip(graphs, outs):
            out.fill_(float("nan"))
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want)
        assert torch.equal(rig.attend(q[:3].contiguous(), few, 1, off=rig.off_d[:3]), first)
    rig.close()


@pytest.mark.parametrize("grid", [0, 512], ids=["shares", "chunks"])
@pytest.mark.parametrize("n", [1024, 1025, 4095])
def test_largest_batches_of_wide_heads(n, grid):
    """Units of 256 elements need the most LDS beside the view of the batch."""
    lens = np.random.default_rng(n).integers(0, 70, n).tolist()
    lens[17] = 900
    rig = Many(4, 2, 256, 1, [max(L, 1) for L in lens])
    assert s3.s3_kv_set_param(rig.a, "grid_blocks", grid) == 0
    rig.fill(lens)
    q, q64 = numbers(rig.rng, (n, 4, 256), 1)
    out = rig.attend(q, lens)
    rig.check_some(out, q64, lens, 2, some(lens))
    assert (out[rig.lens_d(lens) == 0] == 0).all()
    rig.close()
