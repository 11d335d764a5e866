"""The C call path of the calls around an append hands over what the ctypes path does, and leaves other argument types to it."""
import ctypes

import numpy as np
import pytest

from paper_2306_06000_amd import binding as s3

torch = pytest.importorskip("torch")
SIG = ("s3_kv_append_rotary", "s3_qk_rotary", "s3_kv_fetch")
T = [torch.zeros(8, dtype=torch.int16) for _ in range(6)]
HIGH = 0xFFFF_8000_1234_5678
CASES = {"tensors": (T, 0), "addresses": ([16 * i for i in range(1, 6)] + [HIGH], HIGH), "arrays": ([np.zeros(4, np.int64) for _ in range(6)], 1),
         "none": (T[:2] + [None] * 4, None)}


@pytest.fixture
def recorder(monkeypatch):
    seen, keep = {}, []
    handle = type("Handle", (), {})()
    for k, name in enumerate(SIG):
        res, args = s3.SIGNATURES[name]
        plain = [ctypes.c_void_p if hasattr(a, "contents") or a in (s3._pi32,) else a for a in args]

        def body(*values, name=name, k=k):
            seen.setdefault(name, []).append(list(values))
            return -10 - k

        fn = ctypes.CFUNCTYPE(res, *plain)(body)
        keep.append(fn)
        setattr(handle, name, ctypes.CFUNCTYPE(res, *args)(ctypes.cast(fn, ctypes.c_void_p).value))
    s3.lib()
    real = s3._connect_rows()
    lib = s3._lib
    monkeypatch.setattr(s3, "_rows", None)
    monkeypatch.setattr(s3, "_lib", handle)
    monkeypatch.setattr(s3, "_call", real)
    yield seen
    real.connect_rows(*[ctypes.cast(getattr(lib, f), ctypes.c_void_p).value for f in SIG])  # the extension is one per process


def calls(arena, p, stream, rule, n=7):
    a, b, c, d, e, f = p
    return {"s3_kv_append_rotary": lambda: s3.s3_kv_append_rotary(arena, 3, n, a, b, rule, c, d, e, f, a, 512, 1 << 33, 0, stream),
            "s3_qk_rotary": lambda: s3.s3_qk_rotary(rule, s3.S3_BF16, 128, n, a, b, 4, c, 2, d, e, 1 << 34, 8, stream),
            "s3_kv_fetch": lambda: s3.s3_kv_fetch(arena, 2, n, a, b, c, d, stream)}


@pytest.mark.parametrize("case", CASES, ids=list(CASES))
def test_the_call_path_passes_what_ctypes_passes(recorder, monkeypatch, case):
    p, stream = CASES[case]
    arena, rule = ctypes.c_void_p(0x7F00_0000_1000), s3.make_rotary(128, 1 << 12)
    for k, name in enumerate(SIG):
        assert calls(arena, p, stream, rule)[name]() == -10 - k

    class Refusing:
        append_rotary = qk_rotary = fetch = staticmethod(lambda *a: None)

    monkeypatch.setattr(s3, "_rows", Refusing)
    for k, name in enumerate(SIG):
        assert calls(arena, p, stream, rule)[name]() == -10 - k
        one, two = recorder[name]
        assert one == two, (name, one, two)
    assert recorder["s3_qk_rotary"][0][0] == ctypes.addressof(rule) == recorder["s3_kv_append_rotary"][0][7]


def test_other_types_take_the_ctypes_path(recorder):
    arena, rule = ctypes.c_void_p(16), s3.make_rotary(128, 1 << 12)
    for k, name in enumerate(SIG):
        assert calls(arena, T, 0, rule, n=np.int64(7))[name]() == -10 - k
        assert calls(None, T, 0, rule)[name]() == -10 - k
    for name in SIG[:2]:  # no rule: the library refuses it
        assert calls(arena, T, 0, None)[name]() == -10 - SIG.index(name) and recorder[name][-1][0 if name == "s3_qk_rotary" else 7] is None
    for name in SIG:
        with pytest.raises(TypeError):
            calls(arena, ["x"] + T[1:], 0, rule)[name]()
    for name in ("s3_kv_append_rotary", "s3_kv_fetch"):
        with pytest.raises(ctypes.ArgumentError):
            calls(1.5, T, 0, rule)[name]()
