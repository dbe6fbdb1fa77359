"""The sizes of tests/product_forms.py reach every form of the layer operators'
products, and the rules choose no form beyond those (no GPU needed)."""
import os
import random

import pytest

import paper_2609_14706_amd as ff
from product_forms import FEW, LENGTHS, LINEAR, ORTHO, linear_form, ortho_form

TILES = {(8, 8, 2), (6, 8, 2), (4, 8, 3), (4, 6, 3), (4, 4, 2), (4, 4, 4), (2, 4, 3)}
BYTES = {"bf16": 2, "int8": 1}


@pytest.fixture(scope="module", autouse=True)
def built():
    if not os.path.exists(ff.LIB_PATH):
        from paper_2609_14706_amd.build import build
        build()


@pytest.mark.parametrize("kind", ["bf16", "int8"])
def test_linear_layers(kind):
    forms = [linear_form(*s, BYTES[kind]) for s in LINEAR[kind]]
    assert {f[:3] for f in forms if f[3] == 1} == TILES
    assert {f[:3] for f in forms if f[3] > 1} == {(2, 4, 3), (4, 4, 2), (4, 4, 4)}
    few = {linear_form(*s, BYTES[kind])[1:] for s in FEW[kind]}
    want = {(nt, 1, w) for nt in (1, 2, 4) for w in (4, 8, 16)} | {(2, 2, 4), (2, 2, 8), (4, 2, 4)}
    assert few == want
    lengths = {linear_form(T, 64 * p * 2 // BYTES[kind], m, BYTES[kind])[:3] for T, m in LENGTHS for p in range(1, 10)}
    assert {(8, 8, 2), (6, 8, 2), (4, 6, 3), (4, 4, 2)} <= lengths
    # whatever the sizes, nothing else is chosen
    rng = random.Random(5)
    for _ in range(3000):
        T, n, m = (int(2 ** rng.uniform(0, b)) for b in (13, 16, 16))
        f = linear_form(T, n, m, BYTES[kind])
        assert f[1:] in want if f[0] == "few" else f[:3] in TILES


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_updates(kind):
    forms = [ortho_form(*s, kind == "bf16") for s in ORTHO[kind]]
    assert {f[0] for f in forms} == ({0, 1, 2} if kind == "bf16" else {0, 2})
    steps = [f for f in forms if f[0] == 0]
    assert {f[4] for f in steps} == set(range(7)) and {f[3] for f in steps} == set(range(5))
    assert {f[1] for f in steps if f[2] == 1} == set(range(5))
    assert {f[1] for f in steps if f[2] > 1} == ({1, 4} if kind == "bf16" else {0, 1, 3, 4})
