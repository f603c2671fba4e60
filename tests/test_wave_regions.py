"""The waves of an attention block do not wait for one another between the rows they give out through LDS and the loads behind them that make some of these rows again: a wave that was quick
would load over rows that another has not given out yet, unless each keeps to one part of LDS for both.  Every such place of a source has its part from wave_region, whose parts lie side by
side.  No GPU needed."""
import os
import re

import pytest

from paper_2411_15871_amd import build as B


@pytest.mark.parametrize("name", ["attn_window_bf16.h", "attn_docs_bf16.h"])
def test_each_wave_keeps_to_its_part(name):
    source = open(os.path.join(B.CSRC, name)).read()
    assert len(re.findall(r"wave_region<\w+, D>\(smem, wave\)", source)) >= 8  # forward, dQ, dK/dV: rows in either type (forward, dK/dV) or one, and what is made again
    own = [line for line in source.splitlines() if re.search(r"smem\)? \+ wave \*", line)]
    assert not own, own


def test_the_parts_lie_side_by_side():
    source = open(os.path.join(B.CSRC, "attn_bf16.hip")).read()
    body = re.search(r"T\* wave_region\(char\* smem, int wave\) \{ return reinterpret_cast<T\*>\(smem \+ wave \* (.*?)\); \}", source).group(1)
    for d in (64, 128):
        size = eval(body.replace("sizeof(float)", "4").replace("D", str(d)))
        assert size == 32 * d * 4 and size >= 64 * d * 2  # 32 rows of float32 (or bf16) on their way out; a tile of 64 rows of bf16 for those made again
