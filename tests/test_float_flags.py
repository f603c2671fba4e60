"""Infinities and NaNs are numbers that kernels meet (a token or a gradient may hold them) and that some of them look for: no source is built on the promise that there are none, under
which the compiler may drop such a test.  No GPU needed."""
from paper_2411_15871_amd import build as B


def test_no_source_is_built_without_nans_and_infinities():
    for flags in [B.FLAGS] + list(B.EXTRA_FLAGS.values()):
        for f in flags:
            assert "honor" not in f and "finite-math" not in f and "fast" not in f and "unsafe-math" not in f, f
