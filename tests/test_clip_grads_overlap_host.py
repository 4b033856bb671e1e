"""Gradient clipping refuses outputs that share memory with other outputs or other gradients, before any CUDA call."""
import ctypes as C
import math

import pytest

from paper_1810_08313_b200 import binding as b

P = 1 << 20            # addresses that no refused call looks at


def _clip(grads, outs, m, most=1.0):
    """Tensors as (address, elements a replica, distance between replicas, type)."""
    def lists(tensors):
        cols = list(zip(*tensors))
        n = len(tensors)
        return (C.c_void_p * n)(*cols[0]), (C.c_int64 * n)(*cols[1]), (C.c_int64 * n)(*cols[2]), (C.c_int32 * n)(*cols[3])

    gp, n, gs, gt = lists(grads)
    op, _, os_, ot = lists(outs) if outs is not None else (None,) * 4
    return b._lib().ls_clip_grads(gp, n, gs, gt, len(grads), m, most, op, os_, ot, P, 1 << 40, 1 << 40, None)


FP32, BF16 = 0, 1
REFUSED = {
    "outputs are each other's gradients": ([(P, 100, 100, FP32), (2 * P, 100, 100, FP32)], [(2 * P, 100, 100, FP32), (P, 100, 100, FP32)], 1),
    "an output twice": ([(P, 100, 100, FP32), (2 * P, 100, 100, FP32)], [(3 * P, 100, 100, BF16), (3 * P, 100, 100, BF16)], 1),
    "a gradient twice in place": ([(P, 100, 100, FP32), (P, 100, 100, FP32)], None, 1),
    "in place and another's output": ([(P, 100, 100, FP32), (2 * P, 100, 100, FP32)], [(P, 100, 100, FP32), (P + 396, 100, 100, FP32)], 1),
    "the last element": ([(P, 100, 100, FP32), (P + 396, 7, 7, FP32)], None, 1),
    "an output inside its own gradient": ([(P, 100, 100, FP32)], [(P + 4, 100, 100, FP32)], 1),
    "an output of bf16 in its own gradient's second half": ([(P, 100, 100, FP32)], [(P + 200, 100, 100, BF16)], 1),
    "another replica": ([(P, 100, 1000, FP32), (2 * P, 50, 500, FP32)], [(3 * P, 100, 1000, FP32), (P + 8 + 2 * 4000, 50, 500, FP32)], 3),
    "views of one replica vector": ([(P, 100, 300, FP32), (P + 400, 100, 300, FP32), (P + 796, 101, 300, FP32)], None, 4),
    "replicas beside each other in another one's gaps": ([(P, 10, 30, FP32), (P + 40, 10, 25, FP32)], None, 9),
    "gradients as outputs in a packed vector": ([(P, 10, 30, FP32), (P + 40, 10, 30, FP32)], [(P + 80, 10, 30, FP32), (P, 10, 30, FP32)], 2),
}


@pytest.mark.parametrize("name", REFUSED)
def test_shared_memory_is_refused(name):
    grads, outs, m = REFUSED[name]
    assert _clip(grads, outs, m) == b.LS_ERR_INVALID_ARG
    if outs is not None:                          # whatever max_norm: results are written
        assert _clip(grads, outs, m, math.inf) == b.LS_ERR_INVALID_ARG
