"""The operators together, as examples/layer_block.py uses them: a block is
trained with orthogonalised updates, its tokens give its layers' curvature, its
weights become codes, and it runs from them."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    spec = importlib.util.spec_from_file_location("layer_block", os.path.join(ROOT, "examples", "layer_block.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


@pytest.mark.parametrize("hidden,inner,tokens", [(256, 512, 2048), (120, 333, 1001)])
def test_block(gpu, hidden, inner, tokens):
    r = _example().run(hidden, inner, tokens, steps=20)
    assert r["losses"][-1] < 0.5 * r["losses"][0]
    # steps of about gamma = 0.01 on weights of 0.04 to 0.09: a uniform error of
    # 0.01 / sqrt(12), at most a tenth of them, kept below that by the curvature
    assert r["codes against weights"] < 0.15
    # rows rounded to 1/254 of their largest entry (3 to 4 times their rms), twice:
    # below 2% of a row's norm each
    assert r["8-bit rows against bf16 rows"] < 0.04
    # a token alone is rounded as in the batch, but for sums in another order
    assert r["one token against the batch"] < 0.01
