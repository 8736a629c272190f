"""The serving example: prompts at once and then position by position gives what
the same positions give in one pass.  The two run different kernels (decode and
prefill products, one row block and several, other splits of a softmax), whose
float32 results differ in the last bits; a value that falls on the other side of
an int8 step (1/254 of a token's largest at most) or of a 4-bit one changes its
token by about 1e-3, so the bound is a sanity bound of 2e-2."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("kw", [dict(), dict(layers=1, n=256, n_ff=704, heads=4, kv_heads=1, prompts=(33, 64, 1, 20), steps=3, T=1),
                                dict(layers=1, n=256, n_ff=704, heads=2, kv_heads=2, prompts=(300,), steps=2)])
def test_incremental_equals_at_once(gpu, kw):
    spec = importlib.util.spec_from_file_location("serve_batch", os.path.join(ROOT, "examples", "serve_batch.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    assert m.run(log=lambda *a: None, **kw) <= 2e-2
