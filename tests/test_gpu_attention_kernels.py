"""Every kernel of attention and its gradients by its values: 128 and 256 rows and keys a
workgroup, few rows and few keys, keys in parts, in every mode at both widths, batched and
packed, against the plain 64-bit form. Needs an MI355X."""
import pytest
import torch

import attention_kernel_cases as K
from test_gpu_attention import run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def H():
    assert torch.cuda.is_available(), "no GPU"
    from paper_2609_34244_amd import heddle
    heddle.lib()
    return heddle


@pytest.mark.parametrize("name", K.cases())
def test_kernels(H, name):
    c = dict(K.cases()[name])
    c["dtype"] = {"bf16": torch.bfloat16, "fp16": torch.float16}[c["dtype"]]
    run(H, 3, **c)
