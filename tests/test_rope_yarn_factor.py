"""YaRN is a method for contexts longer than the trained one: factors below 1 are refused, and a factor
of 1 changes nothing."""
import math

import pytest

from paper_2609_36757_amd import fastvr


@pytest.mark.parametrize("factor", [0.5, math.nextafter(1.0, 0.0), 1e-3, math.nan, math.inf])
def test_factors_that_lengthen_nothing_are_refused(factor):
    with pytest.raises(ValueError, match="factor"):
        fastvr.rope_inv_freq(32, scaling="yarn", factor=factor, original_len=4096)


def test_a_factor_of_one_is_the_plain_table():
    assert fastvr.rope_inv_freq(32, scaling="yarn", factor=1.0, original_len=4096)[1] == 1.0
    plain = fastvr.rope_inv_freq(32)[0]
    # f k + f (1 - k): two products and a sum, each off by half a step at most
    for a, b in zip(fastvr.rope_inv_freq(32, scaling="yarn", factor=1.0, original_len=4096)[0], plain):
        assert abs(a - b) <= 3 * 2.0 ** -53 * b
