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


def args(**change):
    a = B.LayerArgs()
    a.n_layers, a.d_model, a.n_heads, a.head_dim, a.d_ff, a.family = 3, 128, 2, 64, 256, B.FAMILY_LLAMA
    a.n_tok = a.n_seq = 2
    for k, v in change.items():
        setattr(a, k, v)
    return a


def layers(a, n_mats=3, device="cpu"):
    d, q, f = a.d_model, a.n_heads * a.head_dim, a.d_ff
    make = lambda n, k: B.quant_weights(n, k, device, n_mats)
    return B.quant_layers(a, make(3 * q, d), make(d, q), make(f, d),
                          None if a.family == B.FAMILY_GPT2 else make(f, d), make(d, f))


@pytest.mark.parametrize("change", [dict(n_layers=4), dict(d_model=256), dict(n_heads=4), dict(head_dim=128),
                                    dict(d_ff=512), dict(family=B.FAMILY_GPT2)], ids=str)
def test_a_step_of_other_layers_than_the_weights(change):
    """The kernels would read behind the weights."""
    with pytest.raises(B.AdeptError, match="layer_step_quant: weights of 3 layers"):
        B.layer_step_quant(args(**change), layers(args()), 1)


def test_steps_of_the_weights_layers():
    for a, w in ((args(), layers(args())), (args(n_layers=2), layers(args())),
                 (args(family=B.FAMILY_GPT2), layers(args(family=B.FAMILY_GPT2))),
                 (args(n_heads=1, head_dim=128), layers(args()))):
        with pytest.raises(B.AdeptError, match="current HIP device"):    # the sizes pass
            B.layer_step_quant(a, w, 1)


def test_layers_on_one_device():
    a = args()
    on = lambda d: [B.quant_weights(n, k, d, 3) for n, k in ((384, 128), (128, 128), (256, 128),
                                                             (256, 128), (128, 256))]
    mixed = on("cpu")
    mixed[4] = on("meta")[4]
    with pytest.raises(B.AdeptError, match="one device"):
        B.quant_layers(a, *mixed)
