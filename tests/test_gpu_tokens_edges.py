"""Operators on token tables on the GPU where their paths part: small tables with many
scores, offsets of the type's lowest value, rows and tokens that take no part, gradients
of sizes far apart.  References in 64 bits, bounds from the roundings."""
from __future__ import annotations

import pytest
import torch

import tokens_ref as ref
from test_gpu_tokens import BF, F16, F32, INF, LOWEST, grid_rows, ids, rows, tk, within  # noqa: F401

pytestmark = pytest.mark.gpu


# ---- the k best of small tables with many scores --------------------------------------
@pytest.mark.parametrize("B,M,V", [(1, 4_096, 4_096), (1, 8_192, 2_048), (8, 512, 4_096), (1, 8_200, 1_793),
                                   (1, 4_100, 3_841)])
@pytest.mark.parametrize("k", [1, 2])
@pytest.mark.parametrize("dt", [BF, F16])
def test_best_of_small_tables_with_many_scores(tk, B, M, V, k, dt):
    """From a workspace full of large scores, and then of another call's."""
    D, scale = 32, 0.125
    n = tk.logprobs_workspace_bytes(B, M, V, D, k, dt)
    ws = (rows((n // 4 + 1,), F32, 300).abs() * 1e30).view(torch.uint8)
    for seed in (301, 311):
        X, W, t = grid_rows((B, M, D), dt, seed), grid_rows((B, V, D), dt, seed + 1), ids(B, M, V, seed + 2)
        for masked in (False, True):
            bias = None
            if masked:
                bias = torch.zeros((B, V), device="cuda")
                bias[rows((B, V), F32, seed + 3) > 0.3] = -INF
                bias[:, :V // 3] = -INF  # no token of the first columns
            got = tk.tokens_logprobs(X, W, t, k=k, scale=scale, bias=bias, ws=ws)
            want = ref.logprobs(X, W, t, scale, bias, k)
            what = f"{B, M, V} k={k} masked={masked}"
            assert torch.equal(got[3], want[3]), f"alternatives {what}"
            within(got[4], want[4], ref.logprob_bound(X, W, scale, bias).unsqueeze(-1), f"top logprob {what}")
            again = tk.tokens_logprobs(X, W, t, k=k, scale=scale, bias=bias,
                                       ws=torch.full_like(ws, 0x42))
            assert torch.equal(got[3], again[3]) and torch.equal(got[4], again[4])
