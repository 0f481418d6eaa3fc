"""The operators around a model's layers on the GPU at the shapes that take their rarer ways."""
import pytest
import torch

import model_oracle as O
import paper_2410_15240_amd as F
import test_gpu_model as T
from test_gpu_model import close, generator, rows

pytestmark = pytest.mark.gpu

TYPES = O.TYPES


# ---- norm --------------------------------------------------------------------------------------------------

def test_the_gradients_of_weights_of_more_columns_than_one_launch_sums():
    """No rows, so that the sums are all that there is to do: zeros, for 2^28 columns and more."""
    k = (1 << 28) + 70
    used = torch.ones(2 * k, device="cuda")     # (what the gradients are written over)
    del used
    w, post = torch.ones(2, k, device="cuda", dtype=torch.bfloat16)
    x = torch.empty(0, k, device="cuda", dtype=torch.bfloat16)
    _, _, saved = F.mx8_norm(x, w, post_weight=post)
    _, _, _, dw, dpost = F.mx8_norm_grad(x, w, saved, post_weight=post)
    assert dw.shape == dpost.shape == (k,) and not bool(dw.any()) and not bool(dpost.any())
    del w, post, dw, dpost
    torch.cuda.empty_cache()
