"""Calls of the latent cache at the ends of their ranges, refused ahead of the device (no GPU is needed for that)."""
import pytest

from test_latent_refusals_cpu import AT, B, batch, cache, expanded, refused  # noqa: F401 (B is a fixture)


@pytest.mark.parametrize("heads,head", [(1, 64), (1, 128), (16, 128), (1024, 64)])
@pytest.mark.parametrize("n_seq", [1, 2, 1024])
def test_the_workspace_query_and_the_call_take_the_same_sizes(B, heads, head, n_seq):  # noqa: F811
    b = batch(B, n_seq=n_seq)
    most = 2 ** 30 - 127 * n_seq - 1
    for n, taken in ((0, True), (most, True), (most + 1, False), (2 ** 30 - 1, False), (2 ** 30, False), (2 ** 31 - 1, False), (-1, False)):
        def query():
            return B.spm_latent_attend_expanded_workspace(cache(B), b, heads, head, n, 1)
        if taken:                                  # of the call the next refusal is the workspace's, which nobody has
            assert query() >= n * (2 * head + 64) * 2
            refused(B, expanded(B, b=b, heads=heads, head=head, n_tokens=n, work=None), -1, "workspace")
        else:
            refused(B, query, -1, "n_tokens")
            refused(B, expanded(B, b=b, heads=heads, head=head, n_tokens=n), -1, "n_tokens")


@pytest.mark.parametrize("n_tokens", [2 ** 31, 2 ** 32 + 100, -2 ** 31 - 1])
def test_a_number_of_tokens_is_not_cut_to_32_bits(B, n_tokens):  # noqa: F811
    for call in (lambda: B.spm_latent_attend_expanded_workspace(cache(B), batch(B), 16, 128, n_tokens, 1), expanded(B, n_tokens=n_tokens)):
        with pytest.raises(ValueError, match="32 bits"):
            call()
