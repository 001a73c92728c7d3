"""The optimizer's arguments: what needs no tensor."""
import warnings

import pytest

from paper_2608_27888_gb300 import build as B

B.build()
from paper_2608_27888_gb300.optim import AdamW  # noqa: E402


def test_a_decay_that_8_bits_do_not_follow_draws_a_warning():
    for beta2 in (0.0, 0.98, 0.99):
        with pytest.warns(UserWarning, match="8 bits"):
            AdamW([], bits=8, beta2=beta2)
    with warnings.catch_warnings():
        warnings.simplefilter("error")
        AdamW([], bits=8)
        AdamW([], bits=8, beta2=0.995)
        AdamW([], bits=32, beta2=0.9)
