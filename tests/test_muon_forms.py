"""Which forms the product behind an update's X takes; no GPU needed."""
import random

import muon_forms as forms
from paper_2410_12707_amd import binding as B


def test_sizes_for_every_form_take_the_form_they_are_meant_for():
    for which, *form, size in forms.NEXT:
        assert B.measure_muon_update_next_cut(*size)[which] == tuple(form), (which, size)


def test_there_is_no_other_form():
    rng = random.Random(7)
    table = {(which, *form) for which, *form, _ in forms.NEXT}
    for _ in range(20000):
        rows, cols = (max(1, int(round(65536 ** rng.random()))) for _ in range(2))
        if rows * cols >= 1 << 31:
            continue
        for which, form in enumerate(B.measure_muon_update_next_cut(rows, cols)):
            if which == 0 or min(rows, cols) >= 256:  # below that no product is from the h alone
                assert (which, *form) in table, (which, rows, cols, form)
            # X's runs of elements change: an exchange would read and write it in place in two orders
            assert which != 2 or not form[2]
