"""GPU tests of the operators around the layer at the places where a bound of test_gpu_operators.py leaves room for a whole code, a
lost product or another kernel: exact codes, gates far out, each way in which a scored layer is routed."""
import numpy as np
import pytest

from oracle import operators as orc

pytestmark = pytest.mark.gpu
h = 2.0 ** -24                                             # fp32's half unit in the last place


@pytest.fixture(scope="module")
def amd():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    import paper_2512_17073_amd as amd
    amd.lib()
    return amd


def _normal(rng, *shape):
    return rng.standard_normal(shape, dtype=np.float32)


def _bf16(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).bfloat16().cuda()


def _f64(t):
    return t.double().cpu().numpy()


def _bytes(t):
    import torch
    return t.view(torch.uint8).cpu().numpy()


# ------------------------------------------------------------------------------------------ 8-bit activations
@pytest.mark.parametrize("power", [0, 100, -60, -85, -110, -125])
def test_codes_are_those_of_two_divisions(amd, power):
    """Every significand of bf16 as a block's largest magnitude, and as the other values of the block what lies closest to the middles
    between two codes: scales and codes are those of fp32 divisions, bit for bit.  (What a unit of the last place of the scale
    or of the quotient can change is a tie, and that by a whole code.)"""
    import torch
    codes = orc.e4m3_values()[:127]                        # 0 .. 448
    middles = (codes[1:] + codes[:-1]) / 2
    rng = np.random.default_rng(power + 200)
    rows = []
    for m in range(128):
        top = (1 + m / 128) * 2.0 ** power
        near = middles * (top / 448)
        near = np.concatenate([near, near * (1 + 2.0 ** -8), top * rng.uniform(0, 1, 127 * 8 - 256 + 4)])
        near = np.minimum(near, top * (1 - 2.0 ** -7)) * rng.choice([-1.0, 1.0], near.size)
        blocks = np.full((8, 128), top)
        blocks[:, 1:] = rng.permutation(near)[:8 * 127].reshape(8, 127)
        rows.append(blocks.reshape(-1))
    x = torch.from_numpy(np.array(rows)).bfloat16()
    v = x.float().view(128, 8, 128)
    scale = (v.abs().amax(-1) / torch.tensor(448.0)).clamp_min(2.0 ** -126)
    want = (v / scale[..., None]).clamp(-448, 448).to(torch.float8_e4m3fn)
    got, got_scale = amd.quantize_fp8(x.cuda())
    assert torch.equal(got_scale.cpu(), scale)
    assert np.array_equal(_bytes(got), _bytes(want.view(128, 1024)))
