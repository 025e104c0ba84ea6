"""How the cross entropy reads bf16 operands of any size (CPU only): what goes straight into LDS makes offsets of 32 bits, so that none may pass them; copies are made of what lies at
addresses that cannot, of few enough classes at a time, and of nothing that needs none."""
import itertools

import pytest

from paper_2408_09697_amd import binding as hb

AT = 0x10000000
CLASSES = [2, 349, 352, 131072, 1100000, 2 ** 22 - 8, 2 ** 22, 5000000, 5000001, 8400000, 8421504, 8421505, 8500000, 8500001, 2 ** 24, 33554431, 33554432, 69000000, 70000001, 2 ** 30, 2 ** 31 - 1024]
ROWS = [1, 4, 32, 33, 511, 512, 513, 8192, 700000]


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("classes", CLASSES)
def test_offsets_stay_within_32_bits(classes, backward):
    for n, d, pad, off in itertools.product(ROWS, (1, 64, 128, 256, 1024, 2 ** 22 + 8, 2 ** 24, 2 ** 31 - 1024), (0, 1, 8), (0, 2)):
        for ld_w in (classes + pad, -(-classes // 8) * 8 + 8 * pad):
            r = hb.heta_xent_reads(n, d, classes, backward, AT, d + pad, AT + off, ld_w)
            assert r["reach_w"] < 2 ** 32 and r["reach_in"] < 2 ** 32, (n, d, ld_w, r)
            assert r["classes"] <= classes and (not r["copy_w"] or n >= 512)


@pytest.mark.parametrize("n,d", [(512, 256), (8192, 256), (700000, 64)])
@pytest.mark.parametrize("classes", [349, 131073, 4200001, 5000001, 8500001, 16900000, 33554400])
def test_many_rows_go_straight_into_lds_whatever_the_classes(n, d, classes):
    """By copies where rows start anywhere or are too long for the input gradient's 256, without where they do not have to be."""
    for backward in (False, True):
        odd = hb.heta_xent_reads(n, d, classes, backward, AT, d, AT + 2)
        assert odd["copy_w"] and odd["logits"] and (not backward or (odd["grad_in"] and odd["grad_w"]))
        even = -(-classes // 8) * 8
        r = hb.heta_xent_reads(n, d, even, backward, AT, d, AT)
        assert r["logits"] and not r["copy_in"] and (not backward or (r["grad_in"] and r["grad_w"]))
        assert bool(r["copy_w"]) == (backward and even * 2 >= 2 ** 24)


def test_few_rows_are_not_copied_for():
    for n, classes, backward in itertools.product((1, 64, 511), (349, 1100000, 5000000, 20000000), (False, True)):
        r = hb.heta_xent_reads(n, 256, classes, backward, AT, 256, AT)
        assert not r["copy_w"] and not r["copy_in"]
        straight = classes % 8 == 0 and not (n == 64 and classes * 2 >= 2 ** 23)
        assert bool(r["logits"]) == straight
        if backward:
            assert bool(r["grad_in"]) == (straight and classes * 2 < 2 ** 24)
