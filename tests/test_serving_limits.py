"""Sizes that a call over 4-bit weights does not take are refused before anything is launched."""
import pytest

from paper_2601_03700_amd import binding as B

A = 1 << 20          # an aligned address that is never read


def head(vocab, rows):
    return B.lib().adept_final_logits_quant(256, vocab, 1e-6, A, A, A, A, A, rows, A, None, A, A, A, A,
                                            None)


@pytest.mark.parametrize("vocab,rows", [(100, -1), (100, 64 * 65535 + 1), (50257, 21297),
                                        (32000, 33425), (1 << 26, 16)])
def test_a_head_over_too_many_rows(vocab, rows):
    """The bound of the product, before the rows' norm."""
    assert head(vocab, rows) == -1
    assert b"final_logits_quant: bad max_rows" in B.lib().adept_last_error()
