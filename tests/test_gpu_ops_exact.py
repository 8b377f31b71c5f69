"""The operators' arithmetic below the step of their outputs, and values that are not finite, against float64
(tests/ops_oracle.py)."""
import pytest
import torch

import paper_2512_21835_amd as P  # noqa: F401
from tests import ops_oracle as O
from tests.test_gpu_ops import _run_window, _window_case

pytestmark = pytest.mark.gpu


# ([1] * 3 and two KV heads: the keys cut over wavefronts; two prompts and many heads: whole tiles of rows)
@pytest.mark.parametrize("rows,held,hq,hkv", [([1, 1, 1], [5, 300, 900], 8, 2), ([37, 70], [90, 200], 8, 1),
                                              ([37, 1, 70], [90, 0, 200], 72, 9), ([37, 70], [90, 200], 50, 50)])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("window,sinks", [(0, 0), (64, 3)])
def test_probabilities_of_bf16_rows(rows, held, hq, hkv, d, window, sinks):
    """Two bf16 terms, each within half a step of what it stands for, hold a probability to (2^-8)^2 of its value: the
    output is off by no more than 2^-16 of its terms' sizes beyond what fp32 rows are, before its own rounding."""
    b, q, out = c = _window_case(rows, held, hq, hkv, d, "bf16", "bf16")
    got = _run_window(c, window, sinks)
    want, off32, off16 = O.window(b, q, out, b.pool, hq, window, sinks)
    O.assert_within(got, want, O.rounded(want, off32 + off16 * 2.0 ** -8, torch.bfloat16))
