"""What a stage's operator fields refuse, beside tests/test_gpu_stage_ops.py."""
import pytest

import paper_2512_21835_amd as P
from tests.test_gpu_stage_ops import SHAPES, Model

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rank", [-4, -256])
def test_an_adapter_rank_below_zero_is_refused(rank):
    cfg = Model(SHAPES[64]).config()
    cfg.adapter_rank = rank
    with pytest.raises(P.StageError) as e:
        P.stage_destroy(P.stage_init(cfg))
    assert e.value.code == P.STAGE_EINVAL
