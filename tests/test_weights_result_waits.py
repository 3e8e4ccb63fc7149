"""The weights' kernels take their exponentials straight from matrix products, as attention's take their maxima: no vector instruction in
inline assembly there either."""
from tests import test_matrix_result_waits as waits


def test_no_vector_instruction_in_inline_assembly(tmp_path):
    waits.test_no_vector_instruction_in_inline_assembly("fp4_weights.hip", tmp_path)
