"""A product whose rows are copied first or whose K is in parts needs a workspace, and says what is wrong with one.  CPU only."""
import pytest

import paper_2505_18663_amd as dvdq
from test_rows8_linear8 import H, linear


@pytest.mark.parametrize("M,N,K", [(300, 512, 4001), (70, 1540, 8208), (512, 4096, 5120)])
def test_workspace_refusals(M, N, K):
    need = dvdq.linear8_workspace_bytes(M, N, K)
    assert need > 0
    size = dict(M=M, N=N, K=K, ldx=K, ldw=K, ldy=N)
    assert linear(**size, n=need - 1) == 4 and linear(**size, n=0) == 4
    assert linear(**size, space=H + 8) == 5 and linear(**size, space=None) == 1
