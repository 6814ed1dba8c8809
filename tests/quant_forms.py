"""The forms of the 4-bit product (gemm_direct.hip: blocks of 16 weight rows, waves), which one a
size takes, and sizes that take each of them with each epilogue."""
import math
import os
import re

import adept_inputs as ai

SOURCE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                      "paper_2601_03700_amd", "csrc", "gemm_direct.hip")


def _read():
    """The forms and the estimate's numbers, as the source has them."""
    with open(SOURCE) as f:
        text = " ".join(f.read().split())
    forms = re.search(r"QuantForm forms\[\] = \{((?:\{\d+, \d+\}(?:, )?)+)\};", text).group(1)
    forms = [(int(a), int(b)) for a, b in re.findall(r"\{(\d+), (\d+)\}", forms)]
    num = r"([\d.]+)"
    t = re.search(r"const double wgs = ceil_div\(\(long\)ceil_div\(n_weights, 16 \* f\.nb\) \* "
                  r"ceil_div\(rows, 16\), 256\); const int rounds = ceil_div\(pieces, f\.w\); "
                  r"const double t = wgs \* f\.w \* \(rounds \* \(" + num +
                  r" \* std::min\(rows, 16\) / 16 \+ " + num + r" \* f\.nb\) \+ " + num + r"\) \+ " + num +
                  r" \* rounds \* std::ceil\(wgs \* f\.w / 16\);", text)
    assert t, "the estimate of quant_form has another form: form() below has to follow it"
    return forms, [float(x) for x in t.groups()]


FORMS, (ROW, WEIGHT, FIXED, ROUND) = _read()


def form(rows, n, k):
    """What quant_form chooses for n weight rows."""
    up = lambda a, b: -(-a // b)

    def cost(f):
        nb, w = f
        wgs, rounds = up(up(n, 16 * nb) * up(rows, 16), 256), up(up(k, 128), w)
        return (wgs * w * (rounds * (ROW * min(rows, 16) / 16 + WEIGHT * nb) + FIXED) +
                ROUND * rounds * math.ceil(wgs * w / 16))

    return min(FORMS, key=cost)            # of equal ones the first


def llama(d_model, heads, head_dim, d_ff):
    return ai.DecoderShape(n_layers=2, d_model=d_model, n_heads=heads, head_dim=head_dim, d_ff=d_ff,
                           vocab=128)


def gpt2(d_model, heads, head_dim, d_ff):
    return ai.DecoderShape(n_layers=2, d_model=d_model, n_heads=heads, head_dim=head_dim, d_ff=d_ff,
                           vocab=128, family="gpt2", max_pos=128)


# (layers, rows): one row for each sequence, a prompt and a decode pass
LAYERS = [
    (llama(64, 2, 128, 640), 5), (llama(64, 4, 64, 1152), 49), (llama(576, 4, 64, 128), 33),
    (llama(2112, 4, 64, 128), 50), (llama(64, 6, 128, 128), 49), (llama(64, 12, 64, 256), 50),
    (llama(576, 2, 128, 128), 17), (llama(1088, 2, 128, 128), 24), (llama(3136, 8, 64, 640), 49),
    (llama(3136, 4, 128, 128), 50), (llama(1088, 2, 128, 3200), 64),
    (gpt2(64, 3, 64, 576), 49), (gpt2(64, 11, 64, 2112), 49), (gpt2(2112, 1, 64, 64), 50),
    (gpt2(640, 1, 64, 64), 64), (gpt2(3136, 6, 64, 1088), 64), (gpt2(1088, 1, 128, 3328), 49),
    # the widths of the benchmark's decoders: O of 4096 for 24 rows, all of 1600 for 64
    (llama(4096, 32, 128, 512), 24), (gpt2(1600, 25, 64, 6400), 64)]

# (rows, n, k) of plain products: each form with one and with several blocks of rows where a size
# of it takes it, columns and k that end inside a block
PRODUCTS = [(1, 60, 56), (33, 100, 136), (3, 70, 584), (24, 301, 1000), (5, 50, 1096),
            (50, 500, 1640), (49, 1085, 3320), (24, 4096, 4096), (64, 1600, 6400), (49, 2125, 72),
            (9, 4108, 3656), (17, 11008, 200), (5, 32000, 264), (12, 8200, 520)]


def layer_forms(shape, rows):
    """(epilogue, form) of each product of a layer."""
    d, q, f = shape.d_model, shape.n_heads * shape.head_dim, shape.d_ff
    if shape.family == "gpt2":
        return [("qkv, biased", form(rows, 3 * q, d)), ("residual, biased", form(rows, d, q)),
                ("tanh GELU", form(rows, f, d)), ("residual, biased", form(rows, d, f))]
    return [(f"qkv, rotary {shape.head_dim}", form(rows, 3 * q, d)), ("residual", form(rows, d, q)),
            ("SwiGLU", form(rows, 2 * f, d)), ("residual", form(rows, d, f))]


KINDS = ["qkv, biased", "residual, biased", "tanh GELU", "qkv, rotary 64", "qkv, rotary 128",
         "residual", "SwiGLU"]
