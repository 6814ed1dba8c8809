"""The sizes of test_gpu_quant_forms.py take every form of the 4-bit product with every epilogue."""
from tests import quant_forms as Q


def test_every_form_of_every_epilogue_of_a_layer():
    got = {f for shape, rows in Q.LAYERS for f in Q.layer_forms(shape, rows)}
    assert got == {(kind, f) for kind in Q.KINDS for f in Q.FORMS}


def test_every_form_of_plain_products():
    """For one block of 16 rows and for several."""
    for many in (False, True):
        got = {Q.form(*p) for p in Q.PRODUCTS if (p[0] > 16) == many}
        assert got == set(Q.FORMS)
