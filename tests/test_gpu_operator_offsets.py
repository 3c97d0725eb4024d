"""The operators around the layer on arrays of more than 2^31 elements (bytes of codes): places that 32-bit offsets would miss."""
import pytest
import torch

from paper_2503_21135_b200 import binding
from paper_2503_21135_b200 import operators as ops

pytestmark = pytest.mark.gpu


def test_rows_behind_two_to_the_31():
    T, k, d = 140000, 2, 8192                      # 2.3e9 elements of rows
    idx = torch.stack([torch.arange(T) % 3, 3 + torch.arange(T) % 2], 1).int().cuda()
    x = torch.arange(T, device="cuda").float()[:, None].expand(T, 8).contiguous()
    wide = torch.zeros((T, d), dtype=torch.bfloat16, device="cuda")
    wide[:, :8] = (x % 251).bfloat16()             # exact in bf16
    wide[:, -8:] = (x % 127).bfloat16()
    s = ops.dispatch(idx, 5, wide)
    assert s.rows.numel() > 2 ** 31
    src = (s.perm // k).long()
    assert torch.equal(s.rows[:, 0], wide[src, 0]) and torch.equal(s.rows[:, -1], wide[src, -1])
    w = torch.tensor([0.5, 0.25], device="cuda").expand(T, 2).contiguous()
    y = ops.combine(s.rows, s.pos, w, y_dtype=binding.F32)      # 0.75 x, exactly
    assert torch.equal(y[:, 0], 0.75 * wide[:, 0].float()) and torch.equal(y[:, -1], 0.75 * wide[:, -1].float())
    del y
    d_rows, d_w = ops.combine_backward(wide, s.rows, s.pos, w)
    assert torch.equal(d_rows[s.pos[:, 1].long(), -1].float(), 0.25 * wide[:, -1].float())
    sq = 8 * (wide[:, 0].double() ** 2 + wide[:, -1].double() ** 2)
    assert bool(((d_w.double() - sq[:, None]).abs() <= d * 2.0 ** -24 * sq[:, None]).all())


def test_stream_behind_two_to_the_31():
    T, d = 270000, 8192
    r = torch.full((T, d), 2.0, dtype=torch.bfloat16, device="cuda")
    r[-1] = 4.0
    r_out, n = ops.norm_join(r, r, res_scale=1.0, block_scale=0.5, eps=1e-12)
    # y normed is 1 in every row: r' = r + 0.5, n = 1 (eps is far below a half step of either)
    assert r.numel() > 2 ** 31
    assert bool((r_out[:-1] == 2.5).all()) and bool((r_out[-1] == 4.5).all()) and bool((n == 1.0).all())


@pytest.mark.parametrize("T", [1, 20])
def test_codes_behind_two_to_the_31(T):
    N, K, G = 150000, 32768, 128
    codes = torch.zeros((N, K // 2), dtype=torch.uint8, device="cuda")
    params = torch.zeros((N, K // G, 2), dtype=torch.float16, device="cuda")
    at = torch.arange(N, device="cuda")
    codes[at, K // 2 - 1] = (at % 16 * 16).to(torch.uint8)       # the last input index alone counts, with scale 2 in its group
    params[:, -1, 0] = 2.0
    x = torch.zeros((T, K), dtype=torch.bfloat16, device="cuda")
    x[:, -1] = torch.arange(1, T + 1).bfloat16().cuda()
    assert codes.numel() > 2 ** 31
    y = ops.linear(x, codes, params)
    assert torch.equal(y, x[:, -1:].float() * (2.0 * (at % 16).float())[None])
    assert binding.load().dynamo_linear_poll_status(None) == 0
