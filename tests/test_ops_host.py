"""What the entry points of the operators on reconstructed weights do without a GPU: sizes, and refusals before a device
is touched."""
import paper_2406_11257_amd as X


def test_sizes_of_coded_matrices():
    L = X.lib()
    for rows, cols, groups in ((0, 5, 1), (5, 0, 0), (1, 1, 1), (3, 128, 1), (3, 129, 2), (50304, 2048, 16), (2 ** 31 - 1, 1, 1)):
        assert L.excp_mx_code_bytes(rows, cols) == rows * groups * 64
        assert L.excp_mx_scale_bytes(rows, cols) == rows * groups * 4
    assert L.excp_mx_code_bytes(2 ** 31, 1) == 0 and L.excp_mx_scale_bytes(1, 2 ** 31) == 0
    codes, scales = X.mx_empty(7, 300, "cpu")
    assert codes.shape == (7, 192) and scales.shape == (7, 12)


def test_a_missing_context_is_an_argument_error():
    L = X.lib()
    assert L.excp_mx_quantize(None, None, 0, 1, 1, 1, None, None, None, None) == X.EXCP_E_ARG
    assert L.excp_mx_dequantize(None, None, None, 1, 1, None, 0, 1) == X.EXCP_E_ARG
    assert L.excp_mx_matmul(None, None, None, None, None, 1, 1, 1, None, 0, 1) == X.EXCP_E_ARG
    assert L.excp_mx_linear(None, None, 0, 1, None, None, 1, 1, 1, None, 0, 1, None, None) == X.EXCP_E_ARG
    assert L.excp_token_logprobs(None, None, 0, 1, 1, 1, None, 0, None, None, None, None, None) == X.EXCP_E_ARG
    assert L.excp_token_logprobs_backward(None, None, 0, 1, 1, 1, None, None, None, None, 0, None, None, None, None, 1) == X.EXCP_E_ARG
