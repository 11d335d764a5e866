"""Host side of the 4-bit rows and of the rotation: configurations, sizes, bookkeeping of a metadata-only arena, refusals that need
no device, and the plain forms that the GPU tests compare with."""
import ctypes

import numpy as np
import pytest

from paper_2306_06000_amd import binding as s3
from tests import fp4_plain as plain

BAD = s3.S3_ERR_INVALID


@pytest.mark.parametrize("heads,kv,dim", [(16, 0, 256), (32, 8, 128), (8, 1, 64), (3, 0, 128), (6, 3, 64), (7, 0, 64)])
@pytest.mark.parametrize("act", [s3.S3_F16, s3.S3_BF16])
def test_bytes_of_a_token(heads, kv, dim, act):
    cfg = s3.make_config(5, heads, dim, s3.S3_MXFP4, 64, 2048, kv, act)
    assert s3.s3_kv_bytes_per_token(cfg) == 2 * 5 * plain.row_bytes(kv or heads, dim)


@pytest.mark.parametrize("cfg", [(1, 16, 256, s3.S3_MXFP4, 64, 2048, 0, s3.S3_F32), (1, 16, 256, s3.S3_MXFP4, 64, 2048, 0, s3.S3_MXFP4),
                                 (1, 16, 96, s3.S3_MXFP4, 64, 2048, 0, s3.S3_F16), (1, 16, 256, s3.S3_MXFP4, 64, 2048, 5, s3.S3_F16),
                                 (1, 16, 256, s3.S3_MXFP4, 64, 100, 0, s3.S3_F16), (1, 16, 256, 6, 64, 2048, 0, s3.S3_F16)])
def test_configurations_refused(cfg):
    assert s3.s3_kv_bytes_per_token(s3.make_config(*cfg)) == BAD


def test_metadata_only_arena():
    cfg = s3.make_config(2, 32, 128, s3.S3_MXFP4, 64, 1024, 8, s3.S3_BF16)
    bpt = s3.s3_kv_bytes_per_token(cfg)
    st, a = s3.s3_kv_arena_init(cfg, None, 512 * bpt + 5)
    assert st == 0
    assert s3.s3_kv_stats(a)[1:] == (0, 512, 512, 512)
    rc, ids, offs, caps = s3.s3_kv_alloc(a, [100, 65, 700, 10])
    assert rc == 3 and offs.tolist() == [0, 128, -1, 256] and caps.tolist() == [128, 128, 0, 64]
    assert s3.s3_kv_evict_bytes(a, 33) == 4 * 33 * plain.row_bytes(8, 128)
    assert s3.s3_kv_get_param(a, "kernel_kind") == (0, 5) and s3.s3_kv_get_param(a, "n_variants") == (0, 1)
    assert s3.s3_kv_set_param(a, "variant", 0) == 0 and s3.s3_kv_set_param(a, "variant", 1) == BAD
    # no rows: everything that touches them is refused
    x = 1 << 20
    rule = s3.make_rotary(128, x)
    assert s3.s3_kv_append(a, 0, 1, x, x, x, x) == BAD
    assert s3.s3_kv_append_rotary(a, 0, 1, x, x, rule, x, x, x, x) == BAD
    assert s3.s3_kv_fetch(a, 0, 1, x, x, x, x) == BAD
    assert s3.s3_decode_attention(a, 0, 1, x, x, x, x) == BAD
    s3.s3_kv_arena_destroy(a)


def qk(rule, dtype=s3.S3_BF16, dim=128, n=4, pos=64, q=1 << 12, heads=4, k=1 << 13, kv=2, q_out=1 << 14, k_out=1 << 15, **kw):
    return s3.s3_qk_rotary(rule, dtype, dim, n, pos, q, heads, k, kv, q_out, k_out, **kw)


def test_rotation_refusals_without_a_device():
    ok = s3.make_rotary(128, 1 << 12)
    assert qk(ok, n=0) == 0 and qk(ok, q=None, k=None) == 0  # nothing to do: no device is asked for
    for rule in (None, s3.make_rotary(127, 64), s3.make_rotary(-2, 64), s3.make_rotary(130, 64), s3.make_rotary(128, None),
                 s3.make_rotary(128, 64, n_axes=0), s3.make_rotary(128, 64, n_axes=5, axis_of_pair=[0] * 64),
                 s3.make_rotary(128, 64, n_axes=2), s3.make_rotary(128, 64, n_axes=2, axis_of_pair=[0] * 63 + [2]),
                 s3.make_rotary(128, 64, interleaved=2), s3.make_rotary(128, 64, q_weight=64, eps=-1.0),
                 s3.make_rotary(128, 64, k_weight=64, eps=float("nan"))):
        assert qk(rule) == BAD
    for kw in (dict(dtype=s3.S3_F32), dict(dtype=s3.S3_E4M3), dict(dim=80), dict(n=-1), dict(pos=None), dict(heads=-1), dict(kv=-1),
               dict(q=(1 << 12) + 8), dict(k=(1 << 13) + 2), dict(q_out=None), dict(k_out=None), dict(q_out=(1 << 14) + 8),
               dict(q_stride=504), dict(k_stride=255), dict(q_stride=516), dict(k_stride=-256), dict(heads=70000)):
        assert qk(ok, **kw) == BAD, kw
    with pytest.raises(ValueError):
        s3.make_rotary(128, 64, n_axes=2, axis_of_pair=[0] * 10)
    torch = pytest.importorskip("torch")
    with pytest.raises(ValueError):
        s3.make_rotary(128, torch.zeros(64, dtype=torch.float64))
    with pytest.raises(ValueError):
        s3.make_rotary(128, torch.zeros(63))


def test_entry_points_take_no_arena():
    none, x = ctypes.c_void_p(None), 1 << 20
    rule = s3.make_rotary(128, x)
    assert s3.s3_kv_append_rotary(none, 0, 1, x, x, rule, x, x, x, x) == BAD
    assert s3.s3_kv_fetch(none, 0, 1, x, x, x, x) == BAD


def test_plain_rounding_of_blocks():
    """The tests' own rounding, against cases worked by hand."""
    x = np.zeros((1, 1, 64))
    x[0, 0, :10] = [6.9, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.2, -5.5]      # scale 1: ties to even codes
    x[0, 0, 32:36] = [7.0, 1.0, -0.5, 1.5]                                       # scale 2
    rows = plain.to_rows(x, 1)
    back = plain.from_rows(rows, 1, 64)[0, 0]
    assert back[:10].tolist() == [6, 0, 1, 1, 2, 2, 4, 4, 0, -6] and rows[0, 32:34].tolist() == [127, 128]
    assert back[32:36].tolist() == [8, 1, 0, 2] or back[32:36].tolist() == [8, 1, -0.0, 2]
    # against the nearest of all values of the block's scale, for random numbers
    rng = np.random.default_rng(5)
    x = rng.standard_normal((40, 3, 64)) * np.exp(rng.uniform(-20, 20, (40, 3, 1)))
    back = plain.from_rows(plain.to_rows(x, 1), 3, 64).reshape(40, 3, 2, 32)
    b = x.reshape(40, 3, 2, 32)
    unit = 2.0 ** (np.ceil(np.log2(np.abs(b).max(-1) / 7)))  # (no largest value is 7 times a power of two)
    near = np.abs(np.abs(b / unit[..., None])[..., None] - plain.VALUES).min(-1)
    assert np.allclose(np.abs(b - back) / unit[..., None], near, rtol=0, atol=1e-12)
    x[3, 1, 7], x[4, 2, 40] = np.nan, -np.inf
    back = plain.from_rows(plain.to_rows(x, 0), 3, 64)
    assert np.isnan(back[3, 1, :32]).all() and np.isnan(back[4, 2, 32:]).all() and np.isnan(back).sum() == 64
