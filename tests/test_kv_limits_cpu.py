"""Sizes and values at which the paged key-value cache's calls have to refuse, on the CPU: nothing is launched."""
import ctypes

import pytest

from tests.test_kv_cpu import FAKE, L, R, cache  # noqa: F401  (fixtures)


def test_decode_step_of_rows_past_32_bit_offsets(R, L):  # noqa: F811
    """The step's products address their rows by 32-bit byte offsets: n_seq * d as well as n_seq * ffn stays below 2^31."""
    layer = R.LayerWeights(*[FAKE] * 9)

    def call(d, heads, ffn, n_seq):
        cfg = R.model_cfg(d=d, n_heads=heads, head_dim=128, ffn=ffn, n_layers=1, rms_eps=1e-6, rope_base=1e4, dt_code=R.RIFT_BF16)
        c = cache(heads=heads)
        size = L.riftkv_decode_workspace_size(ctypes.byref(cfg), ctypes.byref(c), n_seq, 4)
        # a workspace that is always too small, so that nothing is launched
        return size, L.riftkv_decode_step(ctypes.byref(cfg), ctypes.byref(layer), FAKE, ctypes.byref(c), FAKE, n_seq, 4, FAKE, FAKE,
                                          FAKE, FAKE, 0, None)

    for d, ffn, most in ((65536, 4096, (1 << 15) - 1), (65536, 8192, (1 << 15) - 1), (4096, 65536, (1 << 15) - 1)):
        size, status = call(d, d // 128, ffn, most)
        assert size > 0 and status == 5, (d, ffn, most)
        for n in (most + 1, 40000, 65535):
            assert call(d, d // 128, ffn, n) == (0, 2), (d, ffn, n)


@pytest.mark.parametrize("base, factor, rotary_dim", [(1e300, 1e10, 64), (10000.0, 1e200, 4), (1.7e308, 2.0, 128)])
def test_a_base_that_overflows(R, base, factor, rotary_dim):  # noqa: F811
    """base * factor^(R / (R - 2)) past float64: every frequency but the first would be 0."""
    with pytest.raises(R.RiftError) as e:
        R.riftkv_rope_freqs(rotary_dim, base=base, scaling="base", factor=factor)
    assert e.value.status == 7
    freqs, _ = R.riftkv_rope_freqs(rotary_dim, base=1e300, scaling="base", factor=1.0)
    assert (freqs > 0).all()


def test_a_magnitude_past_float32(L):  # noqa: F811
    """The factor on the pairs is applied in float32, where this one is infinite."""
    import numpy as np
    f = np.ones(32)

    def call(mag):
        return L.riftkv_rope(FAKE, 128, 2, FAKE, 128, None, 0, 0, None, 0, 1, FAKE, 0, 64, 64, 0, f.ctypes.data, mag, None)   # no rows

    for mag in (1e39, -3.5e38, float("inf")):
        assert call(mag) == 7, mag
    assert call(3.4e38) == 0 and call(0.0) == 0
