"""windq_adamw where its tensors take more than one launch, and either form of one."""
import pytest
import torch

from test_gpu_adamw import make, run, steps32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("count", [16, 17, 224, 225, 300, 450])
def test_as_many_tensors_as_there_are(windq, bits, count):
    """Bit for bit the formula's fp32 steps."""
    sets = [make(1 + (i * 97) % 700, bits, torch.float32, torch.bfloat16, i) for i in range(count)]
    dev, scales, cp = run(windq, sets, bits, 21, 1e-2, 0.05, 0.5, True)
    for i, (p, g, m, v, ms, vs) in enumerate(sets):
        wp, wm, wv, wms, wvs = steps32(p.float().numpy(), g.float().numpy(), m, v, ms, vs, 21, 1e-2, 0.05, 0.5, bits)
        assert torch.equal(dev["p"][i].cpu(), torch.from_numpy(wp)) and torch.equal(cp[i].cpu(), torch.from_numpy(wp).to(torch.bfloat16))
        assert torch.equal(dev["m"][i].float().cpu(), torch.from_numpy(wm)) and torch.equal(dev["v"][i].float().cpu(), torch.from_numpy(wv))
        if bits == 8:
            assert torch.equal(scales[0][i].cpu(), torch.from_numpy(wms)) and torch.equal(scales[1][i].cpu(), torch.from_numpy(wvs))
