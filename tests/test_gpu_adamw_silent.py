"""The 8-bit states over thousands of steps: elements whose gradients fall silent beside one that stays active."""
import math

import numpy as np
import pytest
import torch

from paper_2006_07405_b200 import binding as B

pytestmark = pytest.mark.gpu
LEVELS = [0.3, 0.05, 3e-3, 7e-4]        # of sqrt(v), as a share of the block's largest


def _decay(encode, beta2, steps, blocks):
    """sqrt(v) of silent elements after `steps` steps against the start, by level; one element a block keeps the scale up.
    encode(r, step) gives what is held of the roots r [blocks, 256], in place of the state."""
    r = np.repeat(np.repeat(np.array(LEVELS), 64)[None, :], blocks, 0)
    r[:, 0] = 1.0
    r = encode(r, 0)
    start = r.copy()
    for step in range(1, steps + 1):
        r = encode(np.sqrt(beta2 * r * r + (1 - beta2) * (np.arange(256) == 0)), step)
    return [r[:, max(1, 64 * i):64 * i + 64].mean() / start[:, max(1, 64 * i):64 * i + 64].mean() for i in range(4)]


@pytest.mark.parametrize("beta2,steps", [(0.99, 200), (0.999, 2000)])
def test_8_bit_second_moment_of_silent_elements_beside_an_active_one(beta2, steps):
    """One element of each block keeps a gradient of one and with it the scale; the others' gradients are zero, and sqrt(v)
    should fall by e = 1 - sqrt(beta2) a step.  A code goes up when s - q^2 > u (2 q + 1), u a multiple of 1/4096: with a chance of
    at least the due one and less than 1/4096 above it.  So the mean of s = q^2 falls by e s a step, less at most (2 q + 1) / 4096:
    with r = sqrt(s), r' = -e r / 2 + 1/4096 + 1/(8192 r), whose solution from r0 is below (r0 - k) exp(-e t / 2) + k for
    k = (1 + 1/(2 r1)) / (2048 e), r1 the least r on the way.  Spread: a step moves s by at most 2 q + 1 with chance p <= e q / 2 + 1/4096 or so, so
    its variance after t steps is under t p (2 q + 1)^2; six deviations of a mean over 63 * 64 elements or more are allowed.
    Rounding to the nearest code instead holds every level still."""
    blocks = 64
    n = 256 * blocks
    w, g = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    g[::256] = 1.0
    m, v = torch.zeros(n, dtype=torch.int8, device="cuda"), torch.zeros(n, dtype=torch.uint8, device="cuda")
    ms, vs = torch.zeros(blocks, device="cuda"), torch.zeros(blocks, device="cuda")
    plan = B.a2sgd_adamw_create([w], [g], m, v, ms, vs)
    r = torch.tensor(LEVELS, device="cuda").repeat_interleave(64).repeat(blocks, 1)
    r[:, 0] = 1.0
    m32, v32 = torch.zeros(n, device="cuda"), torch.empty(n, device="cuda")
    B.a2sgd_adamw_write_state(plan, m32, (r * r).reshape(-1))
    B.a2sgd_adamw_read_state(plan, m32, v32)
    start = v32.double().sqrt().view(blocks, 256).cpu().numpy()
    for step in range(1, steps + 1):
        B.a2sgd_adamw_step(plan, lr=0.0, step=step, beta2=beta2)
    B.a2sgd_adamw_read_state(plan, m32, v32)
    end = v32.double().sqrt().view(blocks, 256).cpu().numpy()
    assert np.all(np.abs(end[:, 0] - 1.0) < 0.02)
    e = 1.0 - math.sqrt(beta2)

    def nearest(r, step):
        scale = r.max(axis=1, keepdims=True)
        q = np.sqrt(r / scale) * 255
        low, high = np.floor(q), np.ceil(q)
        return np.where(q * q - low * low < high * high - q * q, low, high) ** 2 / 255 ** 2 * scale

    held = _decay(nearest, beta2, steps, 2)
    for i in range(4):
        part = slice(max(1, 64 * i), 64 * i + 64)
        q0 = 255 * math.sqrt(start[:, part].mean())
        exact = math.exp(-e * steps)
        r1 = max(2.0, q0 * math.exp(-e * steps / 2))
        k = (1 + 1 / (2 * r1)) / (2048 * e)
        most = ((q0 - k) * math.exp(-e * steps / 2) + k) ** 2 / q0 ** 2
        spread = 6 * math.sqrt(steps * (e * q0 / 2 + 1 / 2048) * (2 * q0 + 1) ** 2 / (63 * blocks)) / q0 ** 2
        ratio = end[:, part].mean() / start[:, part].mean()
        assert exact * (1 - 1e-3) - spread <= ratio <= most + spread
        if beta2 == 0.999:
            assert held[i] > most + spread
