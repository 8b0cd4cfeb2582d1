"""AdamW with 8-bit states on parameters whose gradients end, or are small beside their
block's."""
import numpy as np
import pytest
import torch

import paper_2608_22646_gb300 as cai
from tests import train_ref as ref
from tests.test_adamw_gpu import BF16, F32, host

pytestmark = pytest.mark.gpu


def state(n, offset=0):
    """Zero states and parameters, `offset` elements off the vectors' boundaries."""
    def zeros(k, dtype):
        return torch.zeros(k + offset, dtype=dtype, device="cuda")[offset:]
    u8 = torch.uint8
    return dict(param=zeros(n, F32), m=zeros(n, u8), v=zeros(n, u8), m_scale=zeros((n + 31) // 32, u8),
                v_scale=zeros((n + 31) // 32, u8), decay=0.0)


@pytest.mark.parametrize("offset", [0, 1])
def test_a_parameter_whose_gradient_has_ended_rests(offset):
    """Its m is multiplied by 0.9 a step and rounded without bias: after k steps it is
    not 0 with a probability of 0.9^k m / (the smallest code) at most.  From step 200,
    where m is below the block's largest, 2^18 of the smallest code, to step 1000 that is
    2^18 0.9^800 < 1e-31.  From there on the parameter is what it is."""
    n, steps = 32 * 16 + 7, 4000
    t = state(n, offset)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    idle = torch.arange(n, device="cuda") % 5 == 3
    with cai.cai_adamw_init([t], 8) as opt:
        for step in range(1, steps + 1):
            grad = torch.randn(n + offset, generator=g, device="cuda")[offset:]
            if step > 200:
                grad[idle] = 0.0
            cai.cai_adamw_step(opt, [grad], lr=1e-3, step=step, seed=4)
            if step == 1000:
                held, still = t["param"].clone(), t["m"].clone()
    assert (still[idle] == 0).all() and (t["m"][idle] == 0).all()
    assert torch.equal(held[idle], t["param"][idle]) and (held[~idle] != t["param"][~idle]).all()


def packed_m(x, bits, had_root, share):
    """ref.packed's codes and powers, with 0 for numbers it would keep at the smallest code
    alone for their not being 0, where `share` is below that code's number and there was
    a root."""
    code, power = ref.packed(x, bits)
    scale = np.repeat(np.exp2(power.astype(np.float64) - 127), 32)[:len(x)]
    cut = np.abs(x.astype(np.float64)) / scale * 512  # of the smallest number, where below it
    up = np.floor(cut * 2 ** 20) + bits.astype(np.float64) * 16 >= 2 ** 20
    ends = (power[np.arange(len(x)) // 32] != 255) & (cut < 1) & ~up & had_root & (np.abs(share) < scale / 512)
    return np.where(ends, 0, code).astype(np.uint8), power


@pytest.mark.parametrize("gdtype", [F32, BF16])
@pytest.mark.parametrize("offset", [0, 1])
@pytest.mark.parametrize("scale", [None, 0.5])
def test_small_numbers_among_large_ones(gdtype, offset, scale):
    """Gradients from far below the smallest code of their block to above it, of either
    sign or 0, under m and roots of small codes or none: every code to the last bit."""
    n, lr, step, b1, b2, seed = 32 * 700 + 13, 1e-3, 9, 0.9, 0.99, 77
    rng = np.random.default_rng(3)
    t = state(n, offset)
    lead = np.arange(n) % 32 == 0  # the block's largest, as is its gradient
    m = np.where(lead, 120, rng.integers(0, 4, n)) + 128 * rng.integers(0, 2, n)
    root = np.where(lead, 120, rng.integers(0, 3, n))
    for k, x in (("m", m), ("v", root)):
        t[k].copy_(torch.from_numpy(x.astype(np.uint8)))
        t[k + "_scale"].fill_(120)
    size = np.exp2(rng.uniform(-20, 0, n) - 7 - 9 + 4) * rng.choice([-1, 0, 1], n, p=[0.4, 0.2, 0.4])
    grad = torch.zeros(n + offset, dtype=gdtype, device="cuda")[offset:]
    grad.copy_(torch.from_numpy(np.where(lead, 1.0, size)))
    g = host(grad) if scale is None else host(grad) * np.float32(scale)
    before = [ref.unpacked(t[k].cpu().numpy(), t[k + "_scale"].cpu().numpy()).astype(np.float32) for k in "mv"]
    _, m1, _, root1 = ref.adamw(host(t["param"]), g, before[0], None, before[1], lr, step, b1, b2, 1e-8, 0.0)
    h = ref.dither(seed, step, 0, np.arange(n))
    want = packed_m(m1, h & np.uint64(0xffff), before[1] != 0, g * np.float32(1 - b1)) + ref.packed(root1, h >> np.uint64(16))
    floored = ref.packed(m1, h & np.uint64(0xffff))[0]
    assert (floored != want[0]).sum() > 100 and ((want[0] & 127) == 1).sum() > 100  # (both kinds are there)
    scales = None if scale is None else torch.tensor([scale], device="cuda")
    with cai.cai_adamw_init([t], 8) as opt:
        cai.cai_adamw_step(opt, [grad], lr=lr, step=step, beta1=b1, beta2=b2, seed=seed, grad_scale=scales)
    for k, x in zip(("m", "m_scale", "v", "v_scale"), want):
        np.testing.assert_array_equal(t[k].cpu().numpy(), x, err_msg=k)


def test_zeros_stay_zeros():
    """Gradients of -0 and states of 0 and, with beta1 = 0, of any sign leave codes of 0."""
    n = 64
    t = state(n)
    t["m"].copy_(torch.arange(n, device="cuda").to(torch.uint8) + 128)
    t["m_scale"].fill_(100)
    with cai.cai_adamw_init([t], 8) as opt:
        cai.cai_adamw_step(opt, [torch.full((n,), -0.0, device="cuda")], beta1=0.0, step=1)
    assert (t["m"] == 0).all() and (t["v"] == 0).all() and (t["param"] == 0).all()
