"""The limits of test_gpu_attn_precision.py tell the kernels' arithmetic from the same without what it does about its roundings."""
import numpy as np
import pytest

import attn_emulate as emulate
import attn_ref as ref


@pytest.mark.parametrize("name", ["short", "short_full", "few", "parts", "rows_in_128s", "rows_in_128s_full"])   # (the others' arithmetic is one of these)
def test_limits_of_gradients(name):
    lens_q, lens_k, H, Hk, dims, causal, exact_ds, *_ = emulate.PASSES[name]
    lens_k, dh = lens_k or lens_q, dims[0]
    Q, K, V, dY = map(ref.f64, emulate.inputs(lens_q, lens_k, H, Hk, dh, 12.0))
    args = Q, K, V, lens_q, lens_k, causal, dh ** -0.5, dY
    want, rounded = emulate.exact(*args), emulate.prompt(*args, exact_ds)
    limit = {x: emulate.FACTOR * emulate.off(rounded[x], want[x]) for x in want}
    for mistake in ("no correction", "correction turned round") + (("one dS",) if exact_ds else ()):
        wrong = emulate.prompt(*args, exact_ds, mistake)
        assert all(emulate.off(wrong[x], want[x]) > limit[x] for x in ("dQ", "dK")), mistake


@pytest.mark.parametrize("name", emulate.TOKENS)
def test_limits_of_single_tokens(name):
    lens, H, Hk, dh, _ = emulate.TOKENS[name]
    Q, K, V = map(ref.f64, emulate.inputs([1] * len(lens), lens, H, Hk, dh, 1.0)[:3])
    args = Q, K, V, lens, dh ** -0.5
    want = emulate.decode(*args, exact=True)
    assert emulate.off(emulate.decode(*args, mistake="one weight"), want) > emulate.FACTOR * emulate.off(emulate.decode(*args), want)


def test_reference_of_single_tokens():
    """Without roundings it is the definition."""
    lens, H, Hk, dh, _ = emulate.TOKENS["four_heads"]
    Q, K, V = map(ref.f64, emulate.inputs([1] * len(lens), lens, H, Hk, dh, 1.0)[:3])
    want = ref.prompt(Q, K, V, [1] * len(lens), lens, False, dh ** -0.5)["Y"][0]
    np.testing.assert_allclose(emulate.decode(Q, K, V, lens, dh ** -0.5, exact=True), want, rtol=1e-10, atol=1e-12)
