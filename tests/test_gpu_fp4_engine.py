"""A decode loop over 4-bit rows: newcomers' rows filled, steps, doublings, retirements, sequences that go to the host and come back,
against a plain 64-bit replay of every sequence by itself."""
import numpy as np
import pytest

from paper_2306_06000_amd import binding as s3
from paper_2306_06000_amd import workloads as wl
from tests import fp4_plain as plain
from tests.test_gpu_fp4 import DEV, need_gpu_and_lib  # noqa: F401

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.mark.parametrize("fused", [True, False], ids=["step", "append+attend"])
@pytest.mark.parametrize("layers,arena_tokens", [(2, None), (1, 1088)])
def test_a_decode_loop(layers, arena_tokens, fused):
    from paper_2306_06000_amd.engine import DecodeEngine

    heads, kv, d, act, steps = 8, 2, 64, s3.S3_BF16, 70
    rng = np.random.default_rng(11)

    def draw():
        p, g = int(rng.integers(1, 90)), int(rng.integers(2, 110))
        return wl.Seq(p, g, p + max(1, g // int(rng.integers(1, 4))))

    w = wl.Workload("4-bit rows", 9, layers, heads, d, wl.MXFP4, 32, 256, 8, steps, [draw() for _ in range(8)], [draw() for _ in range(20)], refill=True,
                    n_kv_heads=kv, act_dtype=act)
    assert w.row_bytes == plain.row_bytes(kv, d)
    eng = DecodeEngine(w, arena_tokens=arena_tokens, fused=fused)
    assert w.bytes_per_token == eng.bpt
    held = {}  # (serial, layer) -> stored K rows, stored V rows

    def prefill(serial, layer, rows):
        r = np.random.default_rng([serial, layer])
        held[serial, layer] = [plain.to_rows(r.standard_normal((rows, kv, d)).astype(np.float16).astype(np.float64), 1) for _ in range(2)]
        return tuple(torch.from_numpy(x).to(DEV) for x in held[serial, layer])

    eng.start(prefill)
    last = {}

    def tensors_at(step):
        def tensors(layer, n):
            r = np.random.default_rng([step, layer, 5])
            q, k, v = (torch.from_numpy(r.standard_normal((n, h, d))).to(torch.bfloat16) for h in (heads, kv, kv))
            for b, serial in enumerate(eng.serial.tolist()):
                mine = held[serial, layer]
                for which, x in enumerate((k, v)):
                    mine[which] = np.concatenate([mine[which], plain.to_rows(x[b:b + 1].double().numpy(), 1)])
            if layer == layers - 1:
                last["q"], last["serial"] = q.double().numpy(), eng.serial.tolist()
            return q.to(DEV), k.to(DEV), v.to(DEV)

        return tensors

    for t in range(steps):
        out = eng.step(tensors_at(t), prefill, check_host=True)
        if t % 9 and t != steps - 1 or out is None:
            continue
        got = out.double().cpu().numpy()
        for b, serial in enumerate(last["serial"]):
            kk, vv = (plain.from_rows(x, kv, d) for x in held[serial, layers - 1])
            want, bound = plain.attention(last["q"][b], kk, vv)
            tol = plain.allowed(want, bound, np.abs(vv).max(0).repeat(heads // kv, 0), 2)
            assert (np.abs(got[b] - want) <= tol).all(), (t, b)
    assert s3.s3_kv_get_param(eng.arena, "n_grows")[1] > 0 and eng.n_retired > 0
    if arena_tokens:
        assert eng.n_swapped_out > 0 and eng.n_swapped_in > 0
    for a in eng.active:
        for layer in range(layers):
            for which in range(2):
                assert np.array_equal(eng.read_slot(a, layer, which), held[a.serial, layer][which][:a.len])
    per_row = 2 * w.row_bytes
    assert eng.algorithmic_bytes() == per_row * int(eng.len.sum()) + eng.n_active * (heads * d * (2 + 4) + 2 * kv * d * 2 + per_row)
    eng.close()
