"""A single row's columns have to lie side by side, as several rows' do: a column-strided or an expanded
operand of one token is refused, through the native marshalling and without it, and nothing is written."""
import pytest
import torch

from gpu_helpers import lib
from paper_2604_11947_amd import resbm as R


def odd_rows(io, n, device):
    """(1, n) operands whose elements do not lie side by side, in memory that would hold them if they did."""
    wide = torch.arange(2 * n, device=device).to(io).view(1, 2 * n)
    return {"every second column": wide[:, ::2], "one element, expanded": wide[:, :1].expand(1, n),
            "transposed": torch.zeros(n, 8, dtype=io, device=device).t()[:1]}


@pytest.mark.parametrize("which", ["every second column", "one element, expanded", "transposed"])
def test_leading_dimension_of_one_row(which):
    t = odd_rows(torch.bfloat16, 64, "cpu")[which]
    with pytest.raises(ValueError, match="contiguous"):
        R._ld(t, 1, 64, "x")


def test_rows_that_do_lie_side_by_side():
    x = torch.zeros(4, 72)
    assert R._ld(x[:1, :64], 1, 64, "x") == 72 and R._ld(x[:, :64], 4, 64, "x") == 72
    assert R._ld(torch.zeros(64, 1).t(), 1, 64, "x") == 64          # a column seen as a row
    assert R._ld(torch.zeros(0, 128)[:, ::2], 0, 64, "x") >= 64      # no rows, nothing is read


@pytest.mark.gpu
@pytest.mark.parametrize("native", [True, False])
def test_ops_refuse_them(native, monkeypatch):
    L = lib()
    if not native:
        monkeypatch.setattr(R, "_marshal", None)
    n, io = 64, L.io_dtype
    ok = lambda: torch.ones(1, n, dtype=io, device="cuda")
    g, rs, dg = torch.ones(n, device="cuda"), torch.ones(1, device="cuda"), torch.zeros(n, device="cuda")
    ws = L.norm_workspace(1, n, "cuda")
    b, W, bws = torch.ones(1, 8, dtype=io, device="cuda"), torch.ones(8, n, device="cuda"), L.workspace(1, n, 8, "cuda")
    for name, bad in odd_rows(io, n, "cuda").items():
        keep = bad.clone()
        calls = [lambda: L.skip_norm_fwd(bad, g, ok()), lambda: L.skip_norm_fwd(ok(), g, bad),
                 lambda: L.skip_norm_fwd(ok(), g, ok(), res=bad), lambda: L.skip_norm_fwd(ok(), g, ok(), h=bad),
                 lambda: L.skip_norm_q8_fwd(bad, g, ok().to(torch.float8_e4m3fn), torch.ones(1, 1, device="cuda")),
                 lambda: L.skip_norm_bwd(bad, g, rs, ok(), ok(), dg, ws=ws), lambda: L.skip_norm_bwd(ok(), g, rs, bad, ok(), dg, ws=ws),
                 lambda: L.skip_norm_bwd(ok(), g, rs, ok(), bad, dg, ws=ws),
                 lambda: L.skip_norm_bwd(ok(), g, rs, ok(), ok(), dg, g_h=bad, ws=ws),
                 lambda: L.decode_fwd(b, W, bad, ws=bws)]
        for call in calls:
            with pytest.raises(ValueError, match="contiguous"):
                call()
        torch.cuda.synchronize()
        assert torch.equal(bad, keep) and not bool(dg.any()), name
