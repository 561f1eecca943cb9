"""The rule that cuts a product into tiles, asked without a device: what the kernel's forms and the interface rely on, over many shapes."""
import math
import random

import pytest

import __graft_entry__ as entry
from product_forms import DLOGITS, GATED, LSE, STORE, gated_forms, loss_forms, pieces, tiling


@pytest.fixture(scope="module", autouse=True)
def built():
    entry.build()


def shapes(n, seed):
    rng = random.Random(seed)
    for _ in range(n):
        yield tuple(int(round(math.exp(rng.uniform(0.0, math.log(most))))) for most in (40000, 8192, 160000))


def test_what_the_kernel_relies_on():
    for rows, width, n in shapes(3000, 1):
        for end, args in ((LSE, (False, min(rows, 32768), n, width)), (DLOGITS, (False, rows, n, width)), (GATED, (False, rows, n, width)),
                          (STORE, (True, rows, width, n, 1, 1, True)), (STORE, (True, rows, width, n, 2, 1, True)), (STORE, (True, n, width, rows, 1, 2, True))):
            t = tiling(end, *args)
            m, cols, k = args[1:4]
            stages = -(-k // 64) * (args[4] if len(args) > 4 else 1)
            assert t.ctas in (1, 2) and t.halves in (1, 2) and t.end_warps in (8, 16) and (t.halves == 1 or (end == STORE and t.ctas == 2))
            assert t.tile_n == t.cols * (2 if end == GATED else 1) <= 256 and t.tile_n % (16 * t.ctas) == 0
            assert t.tiles_m * 128 * t.ctas * t.halves >= m and t.tiles_n * t.cols >= cols
            assert 1 <= t.splits <= max(1, stages // 8) and (t.splits == 1 or end == STORE)
            # sixteen warps end tiles of up to eight stages, and those of the loss that are no longer are ended in runs by eight
            assert t.end_warps == 8 or (end != GATED and t.halves == 1 and -(-stages // t.splits) <= 8)
            if end == LSE and width > 512:
                assert t.end_warps == 8


def test_pieces_of_the_vocabulary_cover_it_and_fit():
    for rows, _, vocab in shapes(3000, 2):
        n, each, last = pieces(rows, vocab)
        assert (n - 1) * each + last == vocab and 0 < last <= each and each % 256 == 0
        assert 2 * rows * each <= max(512 << 20, 512 * rows)


def test_shapes_of_the_forms_that_are_tested_on_the_device():
    # (the tests there assert the same: this one tells without a device that the rule has moved a shape to another form)
    import test_gpu_product_forms as values
    import test_gpu_product_waits as waits
    for rows, width, vocab, forms in waits.LOSS + values.LOSS:
        assert forms.items() <= loss_forms(rows, width, vocab).items(), (rows, width, vocab)
    for rows, width, hidden, forms in waits.GATED + values.GATED:
        assert forms.items() <= gated_forms(rows, width, hidden).items(), (rows, width, hidden)
    values.test_no_form_is_left_out()
