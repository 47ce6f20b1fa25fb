"""The real types of the microscaled operators are none of the integer operators'."""
import pytest
import torch

import paper_2103_14949_amd as hago


@pytest.mark.parametrize("code", [hago.BF16, hago.F16])
def test_integer_operators_have_no_results_of_them(code):
    a, i8 = torch.zeros(2, 8, dtype=torch.int8), hago.QType(hago.I8)
    with pytest.raises(KeyError):
        hago.qdense(a, i8, torch.zeros(4, 8, dtype=torch.int8), i8, acc_dtype=code)
    with pytest.raises(KeyError):
        hago.qconv2d(torch.zeros(1, 3, 4, 4, dtype=torch.int8), i8, torch.zeros(2, 3, 1, 1, dtype=torch.int8), i8, acc_dtype=code)
