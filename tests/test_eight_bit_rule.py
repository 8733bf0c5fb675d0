"""Which kernels the tests of products with 8-bit weights run: all that the rule may take."""
import shutil

import pytest

from tests import eight_bit_rule, eight_bit_shapes


@pytest.mark.skipif(not shutil.which("g++"), reason="no compiler")
def test_every_kernel_of_products_is_tested(tmp_path):
    pick, shapes = eight_bit_rule.load(str(tmp_path))
    assert len(shapes) == 20 and len(shapes[0]) == 3 and len(shapes[-1]) == 2
    for gated, products in ((0, eight_bit_shapes.PLAIN), (1, eight_bit_shapes.GATED)):
        odd = {v for v, s in enumerate(shapes) if gated and len(s) == 3 and s[1] % 2}          # gate and up fragments come in pairs
        taken = {}
        for M, N, Kd in products:
            taken.setdefault(pick(M, N, Kd, gated), []).append((M, N, Kd))
        assert set(taken) == set(range(len(shapes))) - odd
        for v, products in taken.items():                                        # something left over, and more stages than a ring holds twice
            assert any(M % 16 and N % 16 and -(-Kd // 128) % 2 and Kd > 1024 for M, N, Kd in products), shapes[v]
            rows = 16 * max(1, shapes[v][0])
            assert any(M % rows for M, *_ in products), shapes[v]
