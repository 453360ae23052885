"""The calls of group norm and of the 4-bit operators: whatever arguments they are given, the library receives the same through
_alcs_call and through ctypes, or the same exception is raised.  (No GPU: the library's functions are replaced by ones that record.)"""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2109_00170_b200 import binding as B
from test_binding_host import INTEGERS, MEMORY, STREAMS, I, U, VP, outcome, variants

F, SZ, LL = C.c_float, C.c_size_t, C.c_longlong
TYPES = {"alcs_group_norm": [VP, VP] + [I] * 5 + [VP, VP, F, U, I, VP, VP, VP, SZ, VP], "alcs_group_norm_backward": [VP] * 3 + [I] * 5 + [VP] * 6 + [U, I, VP, SZ, VP],
         "alcs_mx4_quantize": [VP, I, I, LL, I, VP, VP, VP], "alcs_mx4_dequantize": [VP, VP, I, I, VP, LL, I, VP],
         "alcs_mx4_product": [VP, VP, I, VP, VP, I, I, VP, VP, VP, U, I, VP]}
FLOATS = [0.5, 1e-5, 0.1, -1.0, float("inf"), 1, True, np.float32(0.25), np.float64(0.25), C.c_float(2.0), "1", None, 1e300]
ORDINARY = {VP: 4096, I: 3, U: 1, F: 1e-5, SZ: 512, LL: 64}
VALUES = {VP: MEMORY, I: INTEGERS, U: INTEGERS, F: FLOATS, SZ: INTEGERS, LL: INTEGERS}


class Library:
    def __init__(self, calls):
        self.keep = []
        for name, types in TYPES.items():
            def record(*args, name=name):
                calls.append((name, args))
                return 0
            call = C.CFUNCTYPE(I, *types)(record)
            self.keep.append(call)
            f = C.CFUNCTYPE(I, *types)(C.cast(call, VP).value)
            f.argtypes, f.restype = types, I
            setattr(self, name, f)


@pytest.mark.parametrize("name", TYPES)
def test_same_through_both_ways(monkeypatch, name):
    native = pytest.importorskip("paper_2109_00170_b200._alcs_call")
    types = TYPES[name]
    call, ordinary = getattr(B, name), [ORDINARY[t] for t in types[:-1]] + [None]
    places = [(i, VALUES[t]) for i, t in enumerate(types[:-1])] + [(len(types) - 1, STREAMS)]
    B.lib()
    real, calls = B._lib, []
    fake = Library(calls)
    monkeypatch.setattr(B, "_lib", fake)
    native.bind_dense(*(C.cast(getattr(fake, n), VP).value for n in B.DENSE))
    try:
        for args in variants(ordinary, [(0, [ordinary[0]])] + places):
            monkeypatch.setattr(B, "_call", native)
            got = outcome(calls, call, args)
            monkeypatch.setattr(B, "_call", B._NoCall)
            want = outcome(calls, call, args)
            assert got == want or repr(got) == repr(want), args        # (NaN is not itself)
        plain = [torch.zeros(1) if t is VP else a for t, a in zip(types[:-1], ordinary)]
        assert getattr(native, name[5:])(*plain, None) == 0 and len(calls) > 0
        assert getattr(native, name[5:])(*plain, np.int64(1)) is None and getattr(native, name[5:])(*plain) is None
        assert getattr(native, name[5:])(*plain, None, None) is None
    finally:
        native.bind_dense(*(C.cast(getattr(real, n), VP).value for n in B.DENSE))
