"""What the operators on rows in 8 bits ask for in work memory, without a GPU: who promises nothing is told enough for what a call takes, however
its arrays happen to lie."""
import ctypes as C
import itertools

import paper_2111_00705_amd as P


def ask(name, *args):
    n = C.c_uint64(0)
    assert getattr(P.lib(), f"comp_ams_{name}_work_bytes")(*args, C.byref(n)) == P.OK
    return n.value


def test_weight_gradients_without_a_promise_have_enough_for_aligned_rows():
    for rows, n, cols, outs in itertools.product((1, 640, 16_000), (1, 2), (1, 9, 12, 17, 33, 64, 300, 1001, 4096), (1, 8, 16, 24, 77, 200, 2304)):
        for binary, dtype in itertools.product((0, 1), (0, 1, 2)):
            size = [ask("linear_weight_grad", rows // n * n, cols, outs, n, binary, dtype, promised) for promised in (0, 1)]
            assert size[0] >= size[1], (rows, n, cols, outs, binary, dtype)


def test_products_without_a_promise_have_enough_for_aligned_rows():
    for rows, cols, outs in itertools.product((1, 17, 40, 128, 1000, 16_000), (1, 16, 130, 1008, 16_400), (1, 64, 333, 4096)):
        size = {promised: ask("linear_q8", rows, cols, outs, *promised) for promised in itertools.product((0, 1), (0, 1))}
        assert max(size.values()) == size[0, 0] and min(size.values()) == size[1, 1], (rows, cols, outs, size)
