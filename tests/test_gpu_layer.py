"""explore.quantised_layer: a network's layer through the norm, the quantiser, the units' models and the weight-only product."""
import numpy as np
import pytest
import torch

import rows_ref as ref

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
def test_quantised_layer(dtype):
    from paper_2511_10909_b200 import explore, mmasim
    g = torch.Generator().manual_seed(21)
    T, N, K = 24, 160, 512
    x, res, W = (torch.randn(s, generator=g).to(ref.DTYPES[dtype]) for s in ((T, K), (T, K), (N, K)))
    W = W / K ** 0.5
    gain = 1 + 0.1 * torch.randn(K, generator=g)
    r = explore.quantised_layer(x.cuda(), gain.cuda(), W.cuda(), residual=res.cuda())
    h = (x.float() + res.float()).to(x.dtype).double().numpy()
    y, _ = ref.rms_norm(h, gain.double().numpy(), 1e-6)
    real = y @ W.double().numpy().T
    for (arch, fmt), s in r.items():
        assert s["unit"]["count"] == s["format"]["count"] == T * N
        # what the formats cost, from the definitions alone: FP32 noise before the rounding moves few codes
        qa, qb = ref.quantize(y.astype(np.float32), fmt), ref.quantize(W.float().numpy(), fmt)
        value = lambda q: ref.code_values(q[0], fmt) * ref.units(q, fmt, K)
        want = np.sqrt(np.mean((value(qa) @ value(qb).T - real) ** 2))
        assert abs(s["format"]["rms"] - want) < 0.02 * want, (fmt, s["format"]["rms"], want)
        if "weight_only" in s:                              # (the activations are not quantised: less)
            assert 0.3 * want < s["weight_only"]["rms"] < 0.95 * want
    # the units: 13 bits behind the largest term cost as much as the format does, 25 and 35 bits next to nothing
    unit = {k: s["unit"]["rms"] / s["format"]["rms"] for k, s in r.items()}
    assert unit["hopper", "e4m3"] > 20 * unit["blackwell", "e4m3"]
    assert all(u < 1e-3 for k, u in unit.items() if k[0] == "blackwell")


def test_dequantised_is_what_the_products_take():
    """A product with the identity gives the values back, through the models that are exact for one term."""
    from paper_2511_10909_b200 import explore, mmasim
    x = torch.randn((40, 64), generator=torch.Generator().manual_seed(3)).cuda()
    for fmt in ref.FORMATS:
        q = mmasim.quantize(x, fmt)
        v = explore.dequantised(q, fmt)
        c, sf, s = (None if t is None else t.cpu().numpy() for t in q)
        want = ref.code_values(ref.unpack(c, fmt), fmt) * ref.units((c, sf, s), fmt, 64)
        assert np.array_equal(v.cpu().numpy(), want)
