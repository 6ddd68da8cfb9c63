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


# ------------------------------------------------------------------------------------------ scored routing
def _layer(amd, H, E, k, T, wg, bias=None):
    """(layer, its gate in fp64) for a gate [E][H] that is rounded to bf16."""
    import torch
    bits = _bf16(wg).view(torch.int16).cpu().numpy().view(np.uint16)
    L = amd.Layer(hidden=H, ffn=64, n_experts=E, top_k=k, top_n=0, bits=2, group=64, rank=0, max_tokens=T)
    L.set_gate(bits, bias)
    return L, (bits.astype(np.uint32) << 16).view(np.float32).astype(np.float64)


def _check_route(L, wg, x, k, rule, bias=None):
    """The definition's selections and, within two units of fp32's last place, its weights."""
    idx, w = L.route(x)
    logits = _f64(x) @ wg.T + (0.0 if bias is None else bias.astype(np.float64))
    ridx, rw = orc.route_scored(logits, k, **rule)
    assert np.array_equal(idx.cpu().numpy(), ridx)
    assert np.all(np.abs(w.cpu().numpy().astype(np.float64) - rw) <= 2 * h * np.abs(rw) + 2.0 ** -149)


def test_scored_routing_of_tiny_tokens_by_a_huge_gate(amd):
    """Tokens whose squares fp32 does not hold, among ordinary ones, and a gate that makes ordinary logits of them."""
    rng = np.random.default_rng(21)
    T, H, E, k = 512, 16384, 64, 6
    x = _normal(rng, T, H) * 2.0 ** -64
    x[::3] = 2.0 ** -64 * rng.choice([-1.0, 1.0], (len(x[::3]), H))
    x[1::7] *= 2.0 ** -6
    x[5] *= 4.0
    gate = _normal(rng, E, H) * 2.0 ** 57
    gate[1::2] = gate[::2] * (1 + 2.0 ** -7)               # (close keys)
    L, wg = _layer(amd, H, E, k, T, gate)
    rule = dict(score="sigmoid", groups=8, top_groups=4, group_best=2, renormalize=True)
    L.set_routing(**rule)
    _check_route(L, wg, _bf16(x), k, rule)


@pytest.mark.parametrize("groups,top", [(1, 1), (16, 6)])
def test_scored_routing_where_the_matrix_cores_lose_small_products(amd, groups, top):
    """Large products that cancel, +256 and -256 around every 240 small ones that lie just below 2^-24 of the running sum: a product in
    32 bits loses the small ones, whose sum decides between experts that a bias has put level."""
    rng = np.random.default_rng(22)
    T, H, E, k = 640, 2048, 128, 8
    at = np.arange(H) % 256
    large, small = (at == 0) | (at == 255), (at >= 8) & (at < 248)
    x = np.where(large, 16.0, 0.0) * np.ones((T, 1))
    x[:, small] = 2.0 ** -4 * (rng.random((T, small.sum())) < rng.random((T, 1)))
    gate = np.where(at == 0, 16.0, np.where(at == 255, -16.0, 0.0)) * np.ones((E, 1))
    gate[:, small] = 1.984375 * 2.0 ** -13 * (rng.random((E, small.sum())) < rng.random((E, 1)))
    # (levelled for a token with half of the small values; a third of the experts in the choice at all)
    bias = -0.5 * (gate[:, small].sum(1) * 2.0 ** -4) + 1e-3 * rng.standard_normal(E) - 2.0 * (np.arange(E) % 3 != 0)
    bias = bias.astype(np.float32)
    L, wg = _layer(amd, H, E, k, T, gate, bias)
    rule = dict(score="sigmoid", groups=groups, top_groups=top, group_best=1, renormalize=True)
    L.set_routing(**rule)
    _check_route(L, wg, _bf16(x), k, rule, bias)


@pytest.mark.parametrize("max_tokens", [16, 600])
def test_a_gate_is_set_in_the_time_of_its_copy(amd, max_tokens):
    """No pass of the host over the gate's values: a copy of as many bytes from pageable memory, half of it again for the spread, and a few
    calls of a few tens of microseconds each."""
    import time
    import torch
    H, E = 16384, 256
    rng = np.random.default_rng(23)
    L, _ = _layer(amd, H, E, 2, max_tokens, _normal(rng, E, H))
    bits = rng.integers(0, 1 << 14, (E, H)).astype(np.uint16)
    host, there = torch.from_numpy(bits.view(np.int16)), torch.empty((E, H), dtype=torch.int16, device="cuda")

    def least(call):
        took = []
        for _ in range(12):
            torch.cuda.synchronize()
            t = time.perf_counter()
            call()
            torch.cuda.synchronize()
            took.append(time.perf_counter() - t)
        return min(took)

    copy, whole = least(lambda: there.copy_(host)), least(lambda: L.set_gate(bits))
    assert whole <= 1.5 * copy + 1e-4, (whole, copy)


@pytest.mark.parametrize("T,H,E,k,score,groups,top,best,renorm,bias", [
    # sigmoid scores of fewer tokens than the bounds are for, softmax scores of any number: the fp64 gate by 16 x 16 tiles,
    (256, 2048, 128, 8, "sigmoid", 8, 4, 2, True, True),
    (511, 2240, 60, 4, "sigmoid", 6, 3, 2, False, False),
    (301, 1152, 250, 7, "sigmoid", 25, 9, 1, True, True),
    (513, 2240, 60, 4, "softmax", 1, 1, 1, False, True),
    (2047, 2048, 64, 6, "softmax", 8, 3, 2, True, True),
    # and by 32 x 32 tiles
    (1100, 1024, 128, 8, "softmax", 8, 4, 1, False, True),
    (1031, 576, 256, 16, "softmax", 64, 20, 2, True, False),
    (4096, 256, 130, 9, "softmax", 1, 1, 1, True, True),
])
def test_scored_routing_behind_the_tiled_gate(amd, T, H, E, k, score, groups, top, best, renorm, bias):
    rng = np.random.default_rng([T, H, E, 3])
    gate_bias = 0.3 * _normal(rng, E) if bias else None
    L, wg = _layer(amd, H, E, k, T, _normal(rng, E, H) / np.sqrt(H), gate_bias)
    x = _normal(rng, T, H)
    x[3] = 0.0
    select = (0.05 if score == "sigmoid" else 0.3 / E) * _normal(rng, E) if bias else None
    if bias:
        select[E // 2] = -np.inf
    rule = dict(score=score, select_bias=select, groups=groups, top_groups=top, group_best=best, renormalize=renorm, scale=2.5)
    L.set_routing(**rule)
    _check_route(L, wg, _bf16(x), k, rule, gate_bias)


@pytest.mark.parametrize("T,score", [(300, "sigmoid"), (300, "softmax"), (1030, "softmax")])
def test_forward_by_a_rule_behind_the_tiled_gate(amd, T, score):
    """The whole layer against its four calls, tokens of very different magnitudes, whose exponents that pass also hands on."""
    from oracle import fixtures
    from workload import configs
    rng = np.random.default_rng(24)
    H = 2048
    cfg = configs.TINY.with_(tokens=T, n_experts=128, top_k=4, hidden=H, ffn=64, name="scored")
    L = amd.Layer.from_config(cfg, max_tokens=T)
    L.load(fixtures.build_layer(cfg))
    L.set_routing(score, groups=8, top_groups=4, group_best=2, renormalize=True, scale=1.5)
    x = _bf16(_normal(rng, T, H) * 2.0 ** rng.integers(-24, 6, (T, 1)))
    idx, w = L.route(x)
    _, offsets, row_pair, pair_row, _ = L.permute(idx)
    y = _f64(L.expert_ffn(x, offsets, row_pair))
    want = (y[pair_row.cpu().numpy().reshape(T, 4)] * _f64(w)[..., None]).sum(1)
    # (rows rounded to bf16 before the sum here, and perhaps not there; the result rounded once)
    assert np.all(np.linalg.norm(_f64(L.forward(x)) - want, axis=1) <= 2.0 ** -7 * np.linalg.norm(want, axis=1))
