"""Gated blocks, 8-bit checkpoints and adapters without a GPU: NaN in the oracle, sizes at the limits, operands of another device."""
import numpy as np
import pytest

from oracle import block_oracle as o


@pytest.mark.parametrize("kind", ["silu", "gelu", "relu"])
def test_nan_has_no_value_and_no_slope(kind):
    v, d, _, _ = o.act(np.array([np.nan, 1.0, -1.0]), kind)
    assert np.isnan(v[0]) and np.isnan(d[0]) and np.isfinite(v[1:]).all() and np.isfinite(d[1:]).all()
