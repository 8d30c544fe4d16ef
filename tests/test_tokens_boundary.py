"""The C ABI of the operators on token tables without a GPU: exports, and arguments
rejected on the host before any HIP call."""
import ctypes
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "flashtokens.h")
LIB = os.path.join(ROOT, "paper_2608_12629_amd", "libflashkmeans.so")
EINVAL, EUNSUP, EWS = -1, -2, -3
F32, BF16, F16 = 0, 1, 2
P = 4096  # a pointer that is aligned, never followed


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(LIB):
        pytest.fail(f"{LIB} not built (run __graft_entry__.build())")
    from paper_2608_12629_amd import tokens
    return tokens.lib


def test_every_declared_call_is_exported(lib):
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(tokens_\w+)\s*\(", text)))
    assert names == ["tokens_embed", "tokens_embed_grad", "tokens_embed_grad_workspace_bytes",
                     "tokens_logprobs", "tokens_logprobs_grad", "tokens_logprobs_grad_workspace_bytes",
                     "tokens_logprobs_workspace_bytes"]
    for n in names:
        assert hasattr(lib, n), n


BAD_SIZES = [((0, 4, 8, 16), EINVAL), ((1, 0, 8, 16), EINVAL), ((1, 4, 0, 16), EINVAL),
             ((1, 4, 8, 0), EINVAL), ((1, -1, 8, 16), EINVAL), ((65536, 4, 8, 16), EUNSUP),
             ((1, (1 << 24) + 1, 8, 16), EUNSUP), ((1, 4, (1 << 20) + 1, 16), EUNSUP),
             ((1, 4, 8, 8193), EUNSUP)]


@pytest.mark.parametrize("size,status", BAD_SIZES)
def test_sizes_are_refused(lib, size, status):
    B, M, V, D = size
    big = 1 << 62
    assert lib.tokens_embed(P, BF16, P, B, M, V, D, 1.0, P, None) == status
    assert lib.tokens_embed_grad(P, BF16, P, B, M, V, D, 1.0, 0, P, BF16, P, big, None) == status
    assert lib.tokens_logprobs(P, P, BF16, None, P, B, M, V, D, 1.0, 0, P, P, P, None, None, P, big,
                               None) == status
    assert lib.tokens_logprobs_grad(P, P, BF16, None, P, P, None, P, None, B, M, V, D, 1.0, P, P, P, big,
                                    None) == status
    assert lib.tokens_embed_grad_workspace_bytes(B, M, V, D, BF16) == 0
    assert lib.tokens_logprobs_workspace_bytes(B, M, V, D, 0, BF16) == 0
    assert lib.tokens_logprobs_grad_workspace_bytes(B, M, V, D, BF16) == 0


def test_types_are_refused(lib):
    big = 1 << 62
    for dt in (-1, 3):
        assert lib.tokens_embed(P, dt, P, 1, 4, 8, 16, 1.0, P, None) == EINVAL
        assert lib.tokens_embed_grad(P, dt, P, 1, 4, 8, 16, 1.0, 0, P, dt, P, big, None) == EINVAL
        assert lib.tokens_logprobs(P, P, dt, None, P, 1, 4, 8, 16, 1.0, 0, P, P, P, None, None, P, big,
                                   None) == EINVAL
    # the gradient of a lookup comes in its rows' type or fp32
    assert lib.tokens_embed_grad(P, BF16, P, 1, 4, 8, 16, 1.0, 0, P, F16, P, big, None) == EINVAL
    assert lib.tokens_embed_grad(P, F32, P, 1, 4, 8, 16, 1.0, 0, P, BF16, P, big, None) == EINVAL
    # scores take 16-bit rows
    assert lib.tokens_logprobs(P, P, F32, None, P, 1, 4, 8, 16, 1.0, 0, P, P, P, None, None, P, big,
                               None) == EUNSUP
    assert lib.tokens_logprobs_grad(P, P, F32, None, P, P, None, P, None, 1, 4, 8, 16, 1.0, P, P, P, big,
                                    None) == EUNSUP


@pytest.mark.parametrize("bad", [None, P + 2])
def test_pointers_are_refused(lib, bad):
    big = 1 << 62
    for i in range(3):
        a = [P, P, P]
        a[i] = bad
        assert lib.tokens_embed(a[0], BF16, a[1], 1, 4, 8, 16, 1.0, a[2], None) == EINVAL
        assert lib.tokens_embed_grad(a[0], BF16, a[1], 1, 4, 8, 16, 1.0, 0, a[2], BF16, P, big, None) == EINVAL
        assert lib.tokens_logprobs(a[0], a[1], BF16, None, P, 1, 4, 8, 16, 1.0, 0, P, P, a[2], None, None, P,
                                   big, None) == EINVAL
    for i in range(7):
        a = [P] * 7
        a[i] = bad
        assert lib.tokens_logprobs_grad(a[0], a[1], BF16, None, a[2], a[3], None, a[4], None, 1, 4, 8, 16,
                                        1.0, a[5], a[6], P, big, None) == EINVAL
    # a target needs somewhere to go, alternatives too, an entropy's gradient the entropy
    assert lib.tokens_logprobs(P, P, BF16, None, P, 1, 4, 8, 16, 1.0, 0, bad, P, P, None, None, P, big,
                               None) == EINVAL
    assert lib.tokens_logprobs(P, P, BF16, None, P, 1, 4, 8, 16, 1.0, 2, P, P, P, bad, P, P, big, None) == EINVAL
    assert lib.tokens_logprobs(P, P, BF16, None, P, 1, 4, 8, 16, 1.0, 2, P, P, P, P, bad, P, big, None) == EINVAL
    assert lib.tokens_logprobs_grad(P, P, BF16, None, P, P, bad, P, P, 1, 4, 8, 16, 1.0, P, P, P, big,
                                    None) == EINVAL


def test_alternatives_and_factors_are_refused(lib):
    big = 1 << 62

    def call(V, k, scale=1.0):
        return lib.tokens_logprobs(P, P, BF16, None, P, 1, 4, V, 16, scale, k, P, P, P, P, P, P, big, None)
    assert call(8, -1) == EINVAL
    assert call(8, 9) == EINVAL
    assert call(64, 33) == EUNSUP
    for scale in (float("nan"), float("inf"), float("-inf")):
        assert call(8, 1, scale) == EINVAL
        assert lib.tokens_logprobs_grad(P, P, BF16, None, P, P, None, P, None, 1, 4, 8, 16, scale, P, P, P,
                                        big, None) == EINVAL


def test_workspaces_are_refused(lib):
    n = lib.tokens_embed_grad_workspace_bytes(1, 4, 8, 16, BF16)
    assert n > 0
    for ws, size in ((None, n), (P + 4, n), (P, n - 1)):
        assert lib.tokens_embed_grad(P, BF16, P, 1, 4, 8, 16, 1.0, 0, P, BF16, ws, size, None) == EWS
    n = lib.tokens_logprobs_workspace_bytes(1, 4, 8, 16, 2, BF16)
    assert n > 0
    for ws, size in ((None, n), (P + 4, n), (P, n - 1)):
        assert lib.tokens_logprobs(P, P, BF16, None, P, 1, 4, 8, 16, 1.0, 2, P, P, P, P, P, ws, size,
                                   None) == EWS
    n = lib.tokens_logprobs_grad_workspace_bytes(1, 4, 8, 16, BF16)
    assert n > 0
    for ws, size in ((None, n), (P + 4, n), (P, n - 1)):
        assert lib.tokens_logprobs_grad(P, P, BF16, None, P, P, None, P, None, 1, 4, 8, 16, 1.0, P, P, ws,
                                        size, None) == EWS


@pytest.mark.parametrize("B,V,D,k", [(1, 1000, 64, 0), (1, 131_072, 4096, 20), (8, 1024, 128, 5),
                                     (1, 50_021, 100, 32), (3, 17, 8, 1), (1, 2048, 256, 0)])
def test_workspaces_never_shrink_as_positions_grow(lib, B, V, D, k):
    sizes = sorted({1 << i for i in range(22)} | {(1 << i) + 1 for i in range(22)} |
                   {3 * (1 << i) for i in range(20)} | set(range(250, 5000, 250)))
    last = [0, 0, 0]
    for M in sizes:
        now = [lib.tokens_embed_grad_workspace_bytes(B, M, V, D, BF16),
               lib.tokens_logprobs_workspace_bytes(B, M, V, D, k, BF16),
               lib.tokens_logprobs_grad_workspace_bytes(B, M, V, D, BF16)]
        assert all(a <= b for a, b in zip(last, now)), (M, last, now)
        last = now
    assert lib.tokens_embed_grad_workspace_bytes(B, 1000, V, D, BF16) <= \
        lib.tokens_embed_grad_workspace_bytes(B, 1000, 2 * V, D, BF16)


def test_largest_sizes_have_workspaces(lib):
    """Sizes near every limit at once: the arithmetic must not overflow."""
    n = lib.tokens_logprobs_grad_workspace_bytes(65535, (1 << 23) - 64, 1 << 20, 8192, BF16)
    assert n > 65535 * ((1 << 23) - 64) * 8192 * 2  # at least a copy of X
    n = lib.tokens_logprobs_workspace_bytes(65535, 1 << 24, 1 << 20, 8191, 32, BF16)
    assert n > 65535 * (1 << 24) * 8192 * 2


def test_gradients_of_too_many_positions_are_refused(lib):
    for M in ((1 << 23) - 63, 1 << 24):
        assert lib.tokens_logprobs_grad_workspace_bytes(1, M, 8, 16, BF16) == 0
        assert lib.tokens_logprobs_grad(P, P, BF16, None, P, P, None, P, None, 1, M, 8, 16, 1.0, P, P, P,
                                        1 << 62, None) == EUNSUP
    assert lib.tokens_logprobs_grad_workspace_bytes(1, (1 << 23) - 64, 8, 16, BF16) > 0


@pytest.mark.parametrize("D", [128, 130, 200, 256, 257])
def test_gradient_workspaces_never_shrink(lib, D):
    """Across the sizes where dz changes between being stored and not."""
    sizes = [1, 64, 100, 1000, 1025, 2047, 2048, 2049, 4096, 8191, 8192, 8193, 20_000, 100_000, 1 << 20]
    for V in sizes:
        got = [lib.tokens_logprobs_grad_workspace_bytes(1, M, V, D, BF16) for M in sizes]
        assert got == sorted(got), (V, got)
