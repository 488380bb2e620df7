"""How far the sum of two halves is from the float32 number that it stands for, as the header states it."""
import os
import re

import numpy as np

from paper_2502_03805_b200 import build


def error(x):
    """Of numbers whose largest lies in [2^14, 2^15), as the kernel scales a query."""
    first = x.astype(np.float16)
    second = (x - first.astype(np.float32)).astype(np.float16)              # the difference is exact
    return np.abs(x.astype(np.float64) - (first.astype(np.float64) + second.astype(np.float64)))


def test_the_stated_bound_holds_and_half_of_it_does_not():
    text = open(os.path.join(build.INCLUDE, "criticalkv.h")).read()
    own, largest = re.search(r"sum of two halves \(its error 2\^(-\d+) of it, or 2\^(-\d+) of the query's largest element", text).groups()
    own, largest = 2.0 ** int(own), 2.0 ** int(largest)
    # the second half has 11 bits for a difference of up to 12
    worst = np.float32(2.0 ** 14 * (1 + 2.0 ** -11 - 2.0 ** -23))
    r = np.random.default_rng(0)
    x = np.concatenate([np.exp2(r.uniform(-40, 15, 2_000_000)).astype(np.float32), np.arange(2 ** 14, 2 ** 15, 2.0 ** -5, dtype=np.float32),
                        np.array([worst], np.float32)])
    bound = np.maximum(own * x.astype(np.float64), largest * 2.0 ** 14)
    assert np.all(error(x) <= bound)
    assert error(np.array([worst]))[0] > 0.99 * own * worst
    assert np.any(error(x) > 0.99 * largest * 2.0 ** 14)
