"""How the FP8 operators are called: sizes one after the other without a workspace of the caller's, empty batches, results of
more bytes than 32 bits count, stream capture, threads, scales that change in place."""
import numpy as np
import pytest
import torch

import fp8_ref as R
from gpu_util import dev
from paper_2307_09782_b200 import binding, gated_ffn
from test_gpu_fp8_block import acts, bf16_tensor, check_values, sum_tol, weight

pytestmark = pytest.mark.gpu


def test_kept_workspace_over_sizes():
    """Raw activations of sizes whose needs are not ordered like M (K + 128)."""
    w = {K: binding.quantize_weight_fp8_block(torch.randn((48, K), device=dev())) for K in (256, 512, 1024, 4096)}
    with torch.cuda.stream(torch.cuda.Stream()):  # a stream that has no workspace yet
        for M, K in ((2048, 512), (300, 4096), (100, 1024), (27, 4096), (8192, 256), (700, 4096)):
            x = torch.randn((M, K), device=dev()).to(torch.bfloat16)
            y = binding.fp8_block_linear(w[K], x=x)
            assert torch.equal(y, binding.fp8_block_linear(w[K], q=binding.quantize_fp8_block(x))), (M, K)
        torch.cuda.synchronize()
