"""Saved inputs of more rows than one launch has threads for (2^32 along a grid's first dimension)."""
import pytest
import torch

from paper_1804_02941_amd import binding as dab

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def test_save_and_restore_of_more_rows_than_a_grid_has_along_one_dimension():
    rows = (1 << 30) + 70                                          # 64 rows of one channel a workgroup of 256
    X = torch.empty((rows, 1), dtype=torch.bfloat16, device=DEV).normal_()
    Q, S = dab.dab_ckpt8_save(X)
    back = dab.dab_ckpt8_restore(Q, S, 1, torch.bfloat16)
    # a lone number is kept to 7 bits, halves to even: as the same rows are in calls of few
    for at in range(0, rows, 1 << 27):
        part = slice(at, min(at + (1 << 27), rows))
        q, s = dab.dab_ckpt8_save(X[part])
        assert torch.equal(Q[part], q) and torch.equal(S[part], s)
        assert torch.equal(back[part], dab.dab_ckpt8_restore(q, s, 1, torch.bfloat16))
    assert float((back.float() - X.float()).abs().max()) <= 2.0 ** -7 * float(X.abs().max())


def test_matrices_of_more_rows_than_32_bits_count_are_refused():
    """Not taken for one of as many rows as the number's lower 32 bits say."""
    X = torch.empty(((1 << 32) + 4, 1), dtype=torch.bfloat16, device=DEV)
    few = torch.zeros((4, 1), dtype=torch.bfloat16, device=DEV)
    t = torch.zeros((4,), dtype=torch.int64, device=DEV)
    for call in (lambda: dab.dab_head_loss(few, X, t), lambda: dab.dab_w4_pack(X), lambda: dab.dab_ckpt8_save(X)):
        with pytest.raises(ValueError, match="at most 2147483647 rows"):
            call()
    Q, S = torch.empty(((1 << 32) + 4, 32), dtype=torch.int8, device=DEV), torch.empty(((1 << 32) + 4, 1), dtype=torch.uint8, device=DEV)
    with pytest.raises(ValueError, match="at most 2147483647 rows"):
        dab.dab_ckpt8_restore(Q, S, 1, out=X)
