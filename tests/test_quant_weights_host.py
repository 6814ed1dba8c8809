"""binding.QuantWeights made of given codes and scales: what does not hold the matrices is refused,
on the host; the kernels would read behind it."""
import pytest
import torch

from paper_2601_03700_amd import binding as B

CB, SB = 2 * 2 * 1024, 2 * 2 * 64      # of 17 x 130: two blocks of rows, two of k


def u8(*shape):
    return torch.zeros(shape, dtype=torch.uint8)


def test_what_holds_the_matrices():
    assert (B.lib().adept_quant_codes_bytes(17, 130), B.lib().adept_quant_scales_bytes(17, 130)) == (CB, SB)
    assert B.QuantWeights(17, 130, u8(3, CB), u8(3, SB)).n_mats == 3
    made = B.quant_weights(17, 130, "cpu", 2)
    again = B.QuantWeights(made.n, made.k, made.codes, made.scales)
    assert again.n_mats == 2 and again.codes is made.codes


@pytest.mark.parametrize("n,k,codes,scales", [
    (17, 130, (3, CB - 1024), (3, SB)), (17, 130, (3, CB), (3, SB - 64)), (17, 130, (3, CB), (2, SB)),
    (33, 130, (3, CB), (3, SB)), (17, 257, (3, CB), (3, SB)), (17, 130, (3 * CB,), (3 * SB,)),
    (17, 130, (0, CB), (0, SB)), (0, 130, (3, 0), (3, 0)), (17, -1, (3, 0), (3, 0))], ids=str)
def test_sizes_that_do_not_fit(n, k, codes, scales):
    with pytest.raises(B.AdeptError, match="quant_weights"):
        B.QuantWeights(n, k, u8(*codes), u8(*scales))


def test_types_strides_and_devices():
    bad = [(u8(3, CB).float(), u8(3, SB)), (u8(3, CB), u8(3, SB).to(torch.int8)),
           (u8(6, CB)[::2], u8(3, SB)), (u8(3, CB), u8(3, 2 * SB)[:, :SB]),
           (u8(CB, 3).t(), u8(3, SB)), (u8(3, CB), u8(3, SB).to("meta"))]
    for codes, scales in bad:
        with pytest.raises(B.AdeptError, match="quant_weights"):
            B.QuantWeights(17, 130, codes, scales)
