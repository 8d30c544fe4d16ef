"""Which alignment the C ABI of the operators on token tables asks for, without a GPU: a
call with a workspace of 0 bytes that passes its other checks is refused for that."""
import pytest

EINVAL, EWS = -1, -3
BF16 = 1
P = 4096  # never followed


@pytest.fixture(scope="module")
def lib():
    from paper_2608_12629_amd import tokens
    return tokens.lib


@pytest.mark.parametrize("off", [4, 8, 12, 2, 1])
def test_values_of_positions_and_tokens_start_at_any_element(lib, off):
    want = EWS if off % 4 == 0 else EINVAL
    Q = P + off
    assert lib.tokens_embed_grad(P, BF16, Q, 1, 4, 8, 16, 1.0, 0, P, BF16, P, 0, None) == want
    for i in range(7):  # bias, target, logprob, entropy, lse, top_idx, top_logprob
        a = [P] * 7
        a[i] = Q
        assert lib.tokens_logprobs(P, P, BF16, a[0], a[1], 1, 4, 8, 16, 1.0, 2, a[2], a[3], a[4], a[5], a[6],
                                   P, 0, None) == want
    for i in range(6):  # bias, target, lse, entropy, grad_logprob, grad_entropy
        a = [P] * 6
        a[i] = Q
        assert lib.tokens_logprobs_grad(P, P, BF16, *a, 1, 4, 8, 16, 1.0, P, P, P, 0, None) == want


@pytest.mark.parametrize("off", [2, 4, 8])
def test_rows_of_elements_are_aligned(lib, off):
    Q = P + off
    for a in ((Q, P), (P, Q)):
        assert lib.tokens_embed(a[0], BF16, P, 1, 4, 8, 16, 1.0, a[1], None) == EINVAL
        assert lib.tokens_embed_grad(a[0], BF16, P, 1, 4, 8, 16, 1.0, 0, a[1], BF16, P, 0, None) == EINVAL
        assert lib.tokens_logprobs(*a, BF16, None, P, 1, 4, 8, 16, 1.0, 0, P, P, P, None, None, P, 0,
                                   None) == EINVAL
        assert lib.tokens_logprobs_grad(P, P, BF16, None, P, P, None, P, None, 1, 4, 8, 16, 1.0, *a, P, 0,
                                        None) == EINVAL
