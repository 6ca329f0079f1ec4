"""Norms at every number of warps that a row can take (one per 256 columns, up to 32), against the fp64 restatement: sums over warps are
joined 8 or 16 at a time, and rows share a block up to 16 warps of them.  Bounds as in the tests of the norms."""
import numpy as np
import pytest
import torch

from test_gpu_norm import EPS, check_backward, check_forward, make

pytestmark = pytest.mark.gpu

WHOLE = [256 * w for w in (1, 2, 3, 4, 5, 6, 7, 8, 9, 10, 11, 13, 14, 15, 16, 17, 20, 24, 31, 32)]
WIDTHS = WHOLE + [d for w in range(1, 33) for d in (256 * w - 8 * (w % 5 + 1), 256 * w - 1 - w % 7)]


@pytest.mark.parametrize("stream", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("gate,post", [("channel", True), ("row", True), ("channel", False)])
def test_every_number_of_warps(stream, gate, post):
    from paper_2410_17765_b200 import binding

    rs = float(np.float32(0.75))
    for d in WIDTHS:
        N = 19 + d % 3
        v = make(N, d, stream, gate, post, gate == "channel" and d % 2 == 0, seed=d)
        f = binding.norm_forward(v["x"], v["w_pre"], block=v["block"], gate=v["gate"], w_post=v["w_post"], res_scale=rs, eps=EPS)
        check_forward(f, v, rs, stream)
        r = binding.norm_backward(v["dy"], f["x_out"], v["w_pre"], f["rstd_pre"], dx_out=v["dx_out"], block=v["block"], gate=v["gate"],
                                  w_post=v["w_post"], rstd_post=f["rstd_post"], res_scale=rs, eps=EPS)
        check_backward(r, v, f, rs)


@pytest.mark.parametrize("d", [1000, 1024, 2000, 2040, 2304, 2303, 3584, 3841, 4352, 8192])
def test_more_rows_than_the_blocks_hold_at_a_time(d):
    """So that every row group goes round its ring, and the last rows leave some groups without one."""
    from paper_2410_17765_b200 import binding

    N = 148 * 16 * 3 // max(1, d // 512) + 5
    v = make(N, d, torch.bfloat16, "channel", True, True, seed=d)
    f = binding.norm_forward(v["x"], v["w_pre"], block=v["block"], gate=v["gate"], w_post=v["w_post"], eps=EPS)
    check_forward(f, v, 1.0, torch.bfloat16)
    r = binding.norm_backward(v["dy"], f["x_out"], v["w_pre"], f["rstd_pre"], dx_out=v["dx_out"], block=v["block"], gate=v["gate"], w_post=v["w_post"],
                              rstd_post=f["rstd_post"], eps=EPS)
    check_backward(r, v, f, 1.0)
