"""Sizes of the gated feed-forward block that are refused before anything is launched."""
import pytest

from test_gpu_gated_ffn import BWD, FWD


@pytest.mark.parametrize("tokens,width,hidden", [((1 << 21) + 1, 64, 65536), ((1 << 21) + 1, 65536, 64), (1 << 26, 65536, 65536), (1 << 26, 8, 2056)])
def test_more_elements_than_a_launch_covers_are_refused(tokens, width, hidden):
    import paper_2508_06001_amd as K
    sizes = dict(tokens=tokens, width=width, hidden=hidden, xs=width, nbytes=1 << 60)
    assert K.lib.knap_gated_ffn_fwd(*dict(FWD, **sizes, ys=width).values(), 0) == K.KNAP_ERR_INVALID_ARG
    assert K.lib.knap_gated_ffn_bwd(*dict(BWD, **sizes, dys=width, dxs=width).values(), 0) == K.KNAP_ERR_INVALID_ARG
    assert K.knap_gated_ffn_fwd_workspace_bytes(tokens, width, hidden) == K.knap_gated_ffn_bwd_workspace_bytes(tokens, width, hidden) == 0


def test_the_largest_sizes_have_a_workspace():
    import paper_2508_06001_amd as K
    for tokens, width, hidden in ((1 << 21, 64, 65536), (1 << 26, 2048, 8), (1 << 26, 8, 2048)):
        assert K.knap_gated_ffn_bwd_workspace_bytes(tokens, width, hidden) >= 4 * tokens * hidden
