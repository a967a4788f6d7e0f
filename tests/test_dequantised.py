"""explore.dequantised reads scale bytes as the products do, those included that mmasim.quantize does not write (on the CPU)."""
import numpy as np
import pytest
import torch

import rows_ref as ref
from paper_2511_10909_b200 import explore, mmasim


@pytest.mark.parametrize("fmt", ref.FORMATS)
def test_every_scale_byte(fmt):
    block = mmasim.SCALE_BLOCK.get(fmt, 32)
    g = np.random.default_rng(1)
    M, K = 256, 2 * block
    codes = g.integers(0, 16 if fmt in ("mxf4", "nvf4") else 0x78, (M, K)).astype(np.uint8)
    codes[:, :2] = 0                        # a NaN scale reaches zeros too
    sf = np.tile(np.arange(256, dtype=np.uint8)[:, None], (1, 2)) if fmt in mmasim.SCALE_BLOCK else None
    rs = (g.random(M).astype(np.float32) + 0.5) if fmt in ("e4m3", "e5m2", "nvf4") else None
    tensor = lambda a: None if a is None else torch.from_numpy(np.ascontiguousarray(a))
    got = explore.dequantised(mmasim.Quantized(tensor(ref.pack(codes, fmt)), tensor(sf), tensor(rs)), fmt).numpy()
    seven = None if sf is None else sf & 0x7F if fmt == "nvf4" else sf           # UE4M3 has no sign: the products leave the bit out
    want = ref.code_values(codes, fmt) * ref.units((codes, seven, rs), fmt, K)
    assert np.array_equal(got, want, equal_nan=True)
    if sf is not None:
        assert np.isnan(got[0x7F if fmt == "nvf4" else 255]).all()
