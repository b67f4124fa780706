"""Forward and backward with fewer kept columns of X than a 16-byte load holds, extracted, and a few output columns behind a panel of
256 x 256 tiles, on the GPU, against the definition in 64 bits."""
import numpy as np
import pytest

import act_util as au
from test_gpu_act import layer

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M,N", [(8192, 2064), (4096, 4112)])
@pytest.mark.parametrize("keep", [[95], [0, 3, 4, 50, 94], [1, 2, 3, 40, 41, 42, 95], [0, 1, 2, 3, 4, 5, 6, 95]])
def test_few_kept_columns_and_columns_behind_a_panel(M, N, keep):
    layer(M, 96, N, "bf16", True, 0, True, au.SILU, True, True, 0.1, True, keep=np.array(keep))
