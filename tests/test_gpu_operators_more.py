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


def test_swiglu_of_gates_far_out(amd):
    """Gates down to -170 with up values that bring the product back among the normal numbers, and gates up to the largest, each in
    a block of its own, whose scale therefore follows its magnitude: eight units of fp32's last place, as for ordinary gates."""
    import torch
    pairs = [(g, u) for g in (-60.0, -69.0, -69.5, -80.0, -87.0, -87.5, -88.0, -89.0, -92.0, -100.0, -104.0, -120.0, -150.0, -170.0)
             for u in (1e30, -3e38) if np.log2(-g) + g / np.log(2) + np.log2(abs(u)) > -100]
    pairs += [(-69.0, 1e-6), (-70.0, 1e-6), (-200.0, 3e38), (-3e38, 3e38), (88.0, 1.0), (100.0, 2.0), (3e38, 0.5), (3e38, -1e-30)]
    x = np.zeros((len(pairs), 256), np.float32)
    for i, (g, u) in enumerate(pairs):
        x[i, i % 128], x[i, 128 + i % 128] = g, u
    x = _bf16(x)
    v = _f64(x)
    with np.errstate(over="ignore"):
        v = v[:, :128] * v[:, 128:] / (1.0 + np.exp(-v[:, :128]))
    codes, scales = amd.quantize_fp8(x, swiglu=True)
    top = np.abs(v).max(1)
    want = np.where(top == 0, 1.0, np.maximum(top / 448, 2.0 ** -126))
    got = scales.cpu().numpy()[:, 0].astype(np.float64)
    gone = top < 2.0 ** -149                               # (below every number: whichever of a zero's scale and the smallest)
    assert np.all((np.abs(got - want) <= 10 * h * want) | (gone & ((got == 1) | (got == 2.0 ** -126))))
    largest = orc.e4m3_values()[_bytes(codes)].reshape(len(pairs), 128)
    assert np.array_equal(np.abs(largest).max(1)[~gone], np.full((~gone).sum(), 448.0))
    assert np.array_equal(np.sign(largest).sum(1)[~gone], np.sign(v).sum(1)[~gone])
