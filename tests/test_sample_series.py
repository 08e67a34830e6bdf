"""The series in which sampling's kernels compute powers of two, against 60 digits: no GPU needed."""
import decimal
import os
import re
from fractions import Fraction

import paper_2309_01507_amd as lpmm


def test_powers_of_two():
    """The coefficients as the source has them, from the 10th power down, for 2^f with |f| <= 1/2: off by less than 2^-50, an eighth of the rounding to whole numbers of 2^-46"""
    path = os.path.join(os.path.dirname(lpmm.lib_path()), "csrc", "sample.hpp")
    with open(path) as f:
        body = re.search(r"double sample_rounded\(.*?\n}", f.read(), re.S).group(0)
    number = r"(-?\d\.\d+(?:e[-+]\d+)?)"
    first = re.search(r"p = fma_by\(f, " + number + ", " + number, body)
    rest = re.findall(r"p = (?:fma_by|__builtin_fma)\(p, f, " + number, body)
    series = [Fraction(float(x)) for x in (*first.groups(), *rest)]
    assert len(series) == 11 and series[-1] == 1
    with decimal.localcontext() as exact:
        exact.prec = 60
        for i in range(-500, 501):
            f, p = Fraction(i, 1000), Fraction(0)
            for c in series:
                p = p * f + c
            want = (decimal.Decimal(f.numerator) / f.denominator * decimal.Decimal(2).ln()).exp()
            assert abs(p - Fraction(want)) < Fraction(1, 2 ** 50), float(f)
