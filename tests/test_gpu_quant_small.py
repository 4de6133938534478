"""Quantised pages from elsewhere: scales below those that an append writes, and above."""
import pytest
import torch

import quant_harness as Q
from paper_2608_07001_amd import gracekv as gk

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("fmt", [gk.E4M3, gk.E2M1])
@pytest.mark.parametrize("d", [64, 128])
def test_read_every_code_under_every_scale(dtype, fmt, d):
    # a page holds a code's rows under one scale; a value that the type does not hold is the nearest that it does
    per = d * Q.BITS[fmt] // 8
    codes = torch.arange(max(256, per)).remainder(256).to(torch.uint8).view(-1, per)
    n = codes.shape[0]
    K = torch.zeros(256, 1, 16, per, dtype=torch.uint8)
    K[:, 0, :n] = codes
    Ks = torch.arange(256).to(torch.uint8)[:, None, None, None].expand(256, 1, 16, d // 32).contiguous()
    pages = gk.QuantPages(fmt, K.cuda(), K.cuda(), Ks.cuda(), Ks.cuda())
    table = torch.arange(256, dtype=torch.int32, device="cuda")[None]
    cfg = gk.quant_config(pages, dtype, 1, table)
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")        # noqa: E731
    k, v = (torch.full((256 * 16, 1, d), 7.0, dtype=dtype, device="cuda") for _ in range(2))
    gk.quant_read(cfg, pages, table, i32(0), i32(0, 256 * 16), k, v)
    want = Q.values(K, Ks, fmt)[:, 0].reshape(-1, d).to(dtype)
    for x in (k, v):
        got = x.cpu()[:, 0]
        assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(got.nan_to_num(1.0), want.nan_to_num(1.0))
