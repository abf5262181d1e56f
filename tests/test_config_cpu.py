"""`Config` and the POD that is kept for it: any sequence of widths, and a change of any field is seen by the next call."""
import copy
import dataclasses

import numpy as np
import pytest
import torch

from paper_2604_23108_b200 import binding as B

BASE = dict(d_model=64, n_groups=2, experts_per_group=3, k_groups=1, k_experts=2)
MAKE = {"list": list, "tuple": tuple, "range": lambda w: range(w[0], w[1] + 1, w[1] - w[0]), "array": np.array,
        "int16 array": lambda w: np.array(w, np.int16), "tensor": torch.tensor}


def widths(c):
    return list(c.c().group_width)[:3]


@pytest.mark.parametrize("kind", MAKE)
def test_widths_of_every_kind_of_sequence(kind):
    c = B.Config(**BASE, group_width=MAKE[kind]([16, 32]))
    assert widths(c) == [16, 32, 0] and c.c() is c.c()
    c.group_width = MAKE[kind]([24, 40])
    assert widths(c) == [24, 40, 0]
    if kind not in ("tuple", "range"):
        c.group_width[1] = 48                    # in place
        assert widths(c) == [24, 48, 0]


def test_widths_that_are_not_whole_numbers_are_refused():
    for w in ([16.0, 32.5], np.array([16.0, 32.0]), torch.tensor([16.0, 32.0])):
        with pytest.raises(TypeError):
            B.Config(**BASE, group_width=w).c()


def test_a_changed_field_reaches_the_next_call_and_a_copy_is_its_own():
    c = B.Config(**BASE, group_width=[16, 32])
    a = c.c()
    for name, value in (("d_model", 128), ("k_experts", 3), ("alpha_e", 0.5), ("row_align", 1), ("dtype", "f32")):
        setattr(c, name, value)
        b = c.c()
        assert b is not a and getattr(b, name) == (value if name != "dtype" else B.F32)
        a = b
    d = copy.deepcopy(c)
    d.group_width[0] = 8
    e = dataclasses.replace(c, n_groups=1)
    assert widths(d) == [8, 32, 0] and widths(c) == [16, 32, 0] and e.c().n_groups == 1 and c.c().n_groups == 2
