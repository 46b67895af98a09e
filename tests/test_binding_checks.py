"""What the descriptor builders and calls of the 8-bit transformer layers refuse, before the library sees a pointer (no GPU)."""
import pytest
import torch

B = pytest.importorskip("paper_2208_01944_gb300.binding", reason="libpalquant.so not built")


def test_rows_that_overlap_are_refused():
    """A pitch below the row's length would otherwise be read as the row's length, past the end of what is there."""
    x, w, y = torch.zeros(4, 8), torch.zeros(5, 8, dtype=torch.int8), torch.zeros(4, 5)
    B.linear_desc(x, w, y)
    flat, codes, out = torch.zeros(64), torch.zeros(64, dtype=torch.int8), torch.zeros(64)
    for bad in ((x[:1].expand(4, 8), w, y), (flat.as_strided((4, 8), (3, 1)), w, y), (x, w[:1].expand(5, 8), y),
                (x, codes.as_strided((5, 8), (7, 1)), y), (x, w, y[:1].expand(4, 5)), (x, w, out.as_strided((4, 5), (4, 1)))):
        with pytest.raises(ValueError):
            B.linear_desc(*bad)
    d = B.linear_desc(x[:1].expand(1, 8), w, y[:1])  # the pitch of one row does not count
    assert (d.M, d.ldx, d.ldy) == (1, 8, 5)
    wide = torch.zeros(4, 11)
    assert B.linear_desc(wide[:, 2:10], w, y).ldx == 11
