"""Products of more outputs than one launch of the obvious grid could have: a launch has fewer than 2^32 threads."""
import numpy as np
import pytest
import torch

import mx_oracle as O
import paper_2410_15240_amd as F

pytestmark = pytest.mark.gpu

BLOCK = np.arange(1, 17, dtype=np.uint8)    # 16 bytes of codes: E2M1 pairs


@pytest.fixture(autouse=True)
def memory_back():
    yield
    torch.cuda.empty_cache()


def weights(n, k, rows):
    """n x k weights of zeros but in `rows`: block b of rows[i] holds the codes above, rolled by i + b."""
    w = F.MX4.view(torch.zeros(F.MX4.nbytes(n, k), dtype=torch.uint8, device="cuda"), n, k)
    nb = O.blocks(k)
    codes = np.stack([np.concatenate([np.roll(BLOCK, i + b) for b in range(nb)]) for i in range(len(rows))])
    codes.reshape(len(rows), nb, 16)[:, -1, -(-(k - 32 * (nb - 1)) // 2):] = 0
    if k % 2:
        codes.reshape(len(rows), nb, 16)[:, -1, (k - 32 * (nb - 1)) // 2] &= 15
    scales = np.full((len(rows), nb), 128, np.uint8)
    for i, r in enumerate(rows):
        w.codes[r] = torch.from_numpy(codes[i]).cuda()
        w.scales[r] = 128
    return w, O.values(codes, scales, k)


@pytest.mark.parametrize("n,k,m,dtype", [
    (1 << 27, 512, 1, torch.bfloat16), ((1 << 27) + 5, 512, 1, torch.float32), ((1 << 26) + 9, 512, 2, torch.bfloat16),
    ((1 << 28) + 3, 512, 3, torch.float32),     # few enough tokens for tiles of 32
    ((1 << 31) - 1, 7, 3, torch.bfloat16),      # 2^24 tiles of 128
])
def test_linear_of_more_outputs_than_a_launch_has_threads(n, k, m, dtype):
    rows = sorted({0, 1, 12345, (1 << 25) - 1, 1 << 25, (1 << 26) - 1, (1 << 26) - 8, min(1 << 26, n - 2), n // 2, n - 2, n - 1})
    w, v = weights(n, k, rows)
    x = np.random.default_rng(n % 1000 + m).integers(-8, 9, (m, k)).astype(np.float64)
    y = torch.full((m, n), 7, dtype=torch.bfloat16, device="cuda")
    F.mx4_linear(torch.from_numpy(x).to(dtype).cuda(), w, out=y)
    want = torch.from_numpy(x @ v.T).to(torch.bfloat16)
    for i, r in enumerate(rows):
        assert torch.equal(y[:, r].cpu(), want[:, i]), r
        y[:, r] = 0
    assert all(not bool(part.any()) for row in y for part in row.split(1 << 28))


def test_input_gradient_of_more_inputs_than_a_launch_has_threads():
    n, k = 3, (1 << 31) - 1
    w, v = weights(n, 64, [0, 1, 2])
    wide = F.MX4.view(torch.zeros(F.MX4.nbytes(n, k), dtype=torch.uint8, device="cuda"), n, k)
    blocks = [0, 1, 2, 12345, (1 << 26) - 2]
    for b in blocks:
        wide.codes[:, 16 * b:16 * b + 16] = w.codes[:, :16]
        wide.scales[:, b] = 128
    dy = np.random.default_rng(3).integers(-8, 9, (2, n)).astype(np.float64)
    got = F.mx4_linear_grad_input(torch.from_numpy(dy).bfloat16().cuda(), wide)
    want = torch.from_numpy(dy @ v[:, :32]).bfloat16()
    for b in blocks:
        assert torch.equal(got[:, 32 * b:32 * b + 32].cpu(), want)
        got[:, 32 * b:32 * b + 32] = 0
    assert all(not bool(part.any()) for row in got for part in row.split(1 << 28))
