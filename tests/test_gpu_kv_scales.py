"""kvprm_write_kv into fp8 pages whose scale is already far above (or below) what the new rows need, bit for bit
against the oracle: a scale never falls while its page holds earlier tokens."""
import numpy as np
import pytest

from test_gpu_kv_rows import Cache, _rows, _say, _write

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("scale", [2.0 ** -126, 1.5 * 2.0 ** -101, 2.0 ** 119, 2.0 ** 121, 1.25 * 2.0 ** 122, 2.0 ** 126,
                                   1.5 * 2.0 ** 125])
def test_write_beside_far_scales(dtype, scale):
    _say("far scales", dtype, scale)
    counts = [1, 3, 16, 2]
    c = Cache("fp8", 64, [0, 5, 15, 31], counts, seed=21)
    for s in c.scale:
        s[:] = np.float32(scale)
    c.upload()
    _write(c, _rows(sum(counts), 64, dtype, 22, sizes=(1e-30, 1.0, 1e36)), dtype, counts)
    c.check()
