"""8-bit products of rows of any spread, within the bound that the matrix instruction keeps to.

It adds products by eights, where what lies below 2^-13 of the largest of the eight is cut: seven of them by less than that each, 7 2^-13 of the terms' magnitudes.  Between the eights, over the blocks
and for the scales 32 bits: (16 + B) 2^-22 of them.  Then the result's rounding."""
import numpy as np
import pytest
import torch

import decoder_reference as ref
from test_gpu_fp8 import TYPES, values

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("spread", [0.0, 1.0, 3.0])
@pytest.mark.parametrize("rows,outputs,inputs", [(3, 70, 900), (16, 500, 4100), (64, 1000, 2100), (100, 1778, 1024), (260, 1100, 100), (600, 700, 1300), (1500, 2300, 300)])
def test_products_of_rows_of_any_spread(kind, spread, rows, outputs, inputs):
    from paper_2007_12216_amd.decoder import Fp8Linear
    x, w = values(kind, rows, inputs, 11, spread), values(kind, outputs, inputs, 12, 0.3)
    x = x.clamp(-1000, 1000)  # half precision's results stay finite
    got = Fp8Linear.from_weights(w.cuda()).forward(x.cuda()).double().cpu().numpy()
    codes, xs = ref.fp8_rows(x.float().numpy())
    want, size = ref.fp8_product(codes, xs, *ref.fp8_weights(w.float().numpy()))
    error = (7 * 2.0 ** -13 + (16 + xs.shape[0]) * 2.0 ** -22) * size
    bound = error + TYPES[kind][1] * (np.abs(want) + error) + 2.0 ** -25
    finite = np.abs(want) + error < 65504
    assert finite.mean() > 0.9 and (np.abs(got - want) <= bound)[finite].all()
