"""Edges of the C interface of the operators of a model's end that need no GPU."""
import pytest

from paper_2510_09103_amd import binding as B

A = 1 << 20
ROWS = B.rows(A, 64)


@pytest.mark.parametrize("call", [
    lambda: B.adapm_dropout(ROWS, ROWS, B.rows(), 4, 64, 1, B.adapm_dropout_t(1, 2, None, 0.1, 7)),
    lambda: B.adapm_norm_forward(B.adapm_norm_t(4, 64, 1, 0, 1, 0, 1e-5, 7), ROWS, B.rows(), B.rows(), A, B.rows(2 * A, 64), 0, A),
    lambda: B.adapm_norm_forward(B.adapm_norm_t(4, 64, 1, 0, 1, 0, 1e-5, 0), ROWS, B.rows(), ROWS, A, B.rows(2 * A, 64), 0, A,
                                 B.adapm_dropout_t(1, 2, None, 0.1, 7)),
    lambda: B.adapm_norm_backward(B.adapm_norm_t(4, 64, 1, 0, 1, 0, 1e-5, 7), ROWS, B.rows(), ROWS, A, A, ROWS, B.rows(), A, None, A),
    lambda: B.adapm_head_loss(B.adapm_head_t(4, 100, 64, 1, 1, 1.0, 7), ROWS, ROWS, A, 0, A, A, A, A, 1 << 30),
    lambda: B.adapm_head_backward(B.adapm_head_t(4, 100, 64, 1, 1, 1.0, 7), ROWS, ROWS, A, 0, A, 0, B.rows(2 * A, 64), B.rows(4 * A, 64), A, 1 << 30),
])
def test_reserved_fields_are_zero(call):
    with pytest.raises(B.AdapmError, match="reserved") as e:
        call()
    assert e.value.status == B.ADAPM_EINVAL


def test_descriptors_with_reserved_fields_need_no_workspace():
    assert B.adapm_norm_workspace_bytes(B.adapm_norm_t(4, 64, 1, 0, 1, 0, 1e-5, 7)) == 0
    assert B.adapm_head_workspace_bytes(B.adapm_head_t(4, 100, 64, 1, 1, 1.0, 7), ROWS, 1) == 0


def test_a_table_without_a_head_has_no_batch_for_one():
    from paper_2510_09103_amd import workloads as WL
    with pytest.raises(ValueError, match="output head"):
        WL.head_batch(WL.tiny_block(), 4)
