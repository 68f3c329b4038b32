"""The constants of the draws' exponentials against 60 digits: the arithmetic of the kernels' sums rests on them.  No GPU."""
import os
import re
from decimal import Decimal as D
from decimal import getcontext
from math import comb, factorial

from paper_2605_14305_amd import build as b

getcontext().prec = 60
NUMBER = r"-?(?:0x[0-9a-f.]+p[+-]?\d+|[\d.]+(?:e-?\d+)?)"
SOURCE = open(os.path.join(b.CSRC, "draw_kernels.hip")).read()


def _numbers(text):
    return [float.fromhex(x) if "0x" in x else float(x) for x in re.findall(NUMBER, text)]


def test_reduction_of_the_argument():
    per, = _numbers(re.search(rf"rint\(x \* ({NUMBER})\)", SOURCE).group(1))
    high, = _numbers(re.search(rf"r = fma\(k, ({NUMBER}), x\)", SOURCE).group(1))
    low, = _numbers(re.search(rf"q = fma\(k, ({NUMBER}), r\)", SOURCE).group(1))
    step = D(2).ln() / 64
    assert per == float(1 / step)
    assert -high == float(step) and -low == float(step - D(-high))  # each the double nearest to what it stands for


def test_weights_within_a_bin():
    """exp((t - 1/2) / 32) to degree 5 about the middle, as a polynomial in t, highest first."""
    text = re.search(r"static double weight\(double u\) \{(.*?)\n  \}", SOURCE, re.S).group(1)
    c = [D(0)] * 6
    for k in range(6):
        for j in range(k + 1):
            c[j] += comb(k, j) * D("-0.5") ** (k - j) / (D(32) ** k * factorial(k))
    assert _numbers(text[text.index("return"):]) == [float(x) for x in reversed(c)]


def test_steps_of_bins():
    down = re.search(r"kDown\[8\] = \{(.*?)\};", SOURCE, re.S).group(1)
    up = re.search(r"kUp\[7\] = \{(.*?)\};", SOURCE, re.S).group(1)
    assert _numbers(down) == [float((-D(i) / 32).exp()) for i in range(8)]
    assert _numbers(up) == [float((D(16) * i).exp()) for i in range(7)]
