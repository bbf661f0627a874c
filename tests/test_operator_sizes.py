"""Sizes past what the library's 32-bit arguments hold are refused, not cut down to their lower bits; types that are not built too.  The
tensors are on no device: nothing is allocated."""
import pytest
import torch

import paper_2511_00413_amd as T
from test_operator_refusals import FAKE, L

F32 = torch.float32
WRAP = 1 << 32


def meta(*shape, dtype=F32):
    return torch.empty(shape, dtype=dtype, device="meta")


def test_binding_refuses_sizes_past_32_bits():
    plan = T.tree_gdn_plan([-1], [2])
    i32 = torch.int32
    wide, A, Bc = meta(2, WRAP + 64), meta(WRAP + 64, 4), meta(2, 1, 4)
    x = meta(2, 64)
    for call in (lambda: T.tree_logprob_entropy(meta(2, WRAP + 50), meta(2, dtype=i32)),
                 lambda: T.tree_logprob_entropy_workspace(meta(2, WRAP + 50)),
                 lambda: T.tree_logprob_entropy_workspace(meta(2, 50), WRAP + 5),
                 lambda: T.tree_logprob_entropy(meta(2, 50), meta(2, dtype=i32), top_k=WRAP + 5),
                 lambda: T.tree_logprob_entropy(meta(0, 50), meta(0, dtype=i32), top_k=WRAP + 5),
                 lambda: T.tree_logprob_entropy_bwd(meta(2, WRAP + 50), meta(2, dtype=i32), meta(2), meta(2)),
                 lambda: T.tree_rope_axes(meta(2, WRAP + 1, 32), meta(3, 2, dtype=i32), (4, 6, 6)),
                 lambda: T.tree_scan_fwd(wide, wide, A, Bc, Bc, plan), lambda: T.tree_scan_bwd(wide, wide, A, Bc, Bc, wide, plan),
                 lambda: T.tree_scan_workspace(wide, A, Bc, plan), lambda: T.tree_scan_workspace(meta(WRAP + 2, 64), meta(64, 4), Bc, plan),
                 lambda: T.tree_scan_workspace(meta(WRAP + 2, 64), meta(64, 4), meta(WRAP + 2, 1, 4), plan),
                 lambda: T.tree_scan_step(wide, wide, A, Bc, Bc, meta(2, WRAP + 64, 4)),
                 lambda: T.tree_scan_step(x, x, meta(64, 4), Bc, Bc, meta(WRAP + 2, 64, 4)),
                 lambda: T.tree_conv_step(wide, meta(2, 3, WRAP + 64), meta(WRAP + 64, 4)),
                 lambda: T.tree_conv_step(x, meta(WRAP + 2, 3, 64), meta(64, 4))):
        with pytest.raises(ValueError, match="at most|must lie|must be"):
            call()


def test_workspace_of_types_that_are_not_built():
    plan = T.tree_gdn_plan([-1], [2])
    with pytest.raises(ValueError):
        T.tree_logprob_entropy_workspace(torch.zeros(2, 50).half())
    with pytest.raises(ValueError):
        T.tree_scan_workspace(torch.zeros(2, 64).half(), torch.zeros(64, 4), torch.zeros(2, 1, 4), plan)
    with pytest.raises(ValueError):
        T.tree_scan_workspace(torch.zeros(2, 64), torch.zeros(64, 5), torch.zeros(2, 1, 5), plan)
    assert T.tree_scan_workspace(torch.zeros(2, 64), torch.zeros(64, 4), torch.zeros(2, 1, 4), plan) > 0
    assert T.tree_scan_workspace(torch.zeros(0, 64), torch.zeros(64, 4), torch.zeros(0, 1, 4), T.tree_gdn_plan([-1], [0]), backward=True) > 0


def test_channels_of_a_convolution_step():
    """The last workgroup's channels reach past 2^31 from 2^31 - 1020 on."""
    ok = dict(n=1, c=(1 << 31) - 512, k=2, dt=0, act=1, x=FAKE[0], xs=0, w=FAKE[1], b=None, slots=1, s=FAKE[3], i=None, so=FAKE[5], y=FAKE[6], ys=0)
    assert L.tt_tree_conv_step(*ok.values(), None) == -2 and "channels" in T.last_error()
