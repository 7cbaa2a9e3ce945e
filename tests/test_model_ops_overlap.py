"""linear's output may be the residual, but no operand that other tokens or channels still read.  CPU only: refused before a launch."""
import paper_2505_18663_amd as dvdq

A, B, C = 0x10000, 0x20000, 0x30000        # never dereferenced


def linear(x=A, w=B, y=C, bias=None, gate=None, gr=0, ldg=64, res=None, M=4, ldy=64):
    return dvdq.lib().dvdq_linear(x, 64, w, 64, bias, 0, gate, gr, ldg, res, 64, M, 64, 64, 0, y, ldy, 0x1000, 1 << 40, None)


def test_output_over_an_operand_is_refused():
    for M in (1, 4, 300):
        assert linear(y=A, M=M) == 3               # tiles of y are written while x is read as the K operand of others
        assert linear(y=B, M=M) == 3
    assert linear(bias=C) == 3                     # one row for all tokens
    assert linear(gate=C, gr=1) == 3 and linear(gate=C, gr=2) == 3
    assert linear(gate=C, gr=4, ldg=72) == 3       # a row per token, in other places
    assert linear(x=A, w=A, y=A) == 3
