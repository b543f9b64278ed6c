"""What the bins of a top-p row know of their masses, computed as the kernel does, against the slack that its windows leave for it."""
import re
from pathlib import Path

import numpy as np

TEXT = (Path(__file__).resolve().parent.parent / "paper_2605_13319_b200" / "csrc" / "serving" / "shape.cuh").read_text()


def _constant(name):
    return float(re.search(r"\b" + name + r" = ([0-9.e+-]+)f?[;,]", TEXT).group(1))


def test_the_slack_covers_what_a_bin_loses():
    f32, width = np.float32, _constant("kShapeWidth")
    d0 = f32(0.5) / f32(width)
    f = np.arange(0, 1 << 16, dtype=np.float64) / (1 << 16)                  # places inside a bin
    inner = (f * (4096.0 / width ** 2) + float(-(f32(8192) + f32(8192) * d0) / f32(width))).astype(f32)
    big = f32(8388608) + f32(8192) * (f32(1) + d0 + f32(0.5) * d0 * d0)      # (rounded to a whole number)
    steps = (f * inner + float(big)).astype(f32).astype(np.float64) - 8388608.0
    weight = np.exp(-(f - 0.5) / width) * 8192.0
    worst = np.abs(steps / weight - 1).max()
    place = 4096 * 2.0 ** -24 / width                                        # half a step of fp32 at the last bins, relative
    assert 6e-5 < worst and worst + 4 * place <= _constant("kShapeSlack"), (worst, place)
    # a prefix against a share of the whole: both are off by the slack
    share = 1 + 2 * _constant("kShapeSlack") + 4 * _constant("kShapeSlack") ** 2
    assert share < 1 + 3 * _constant("kShapeSlack")
