"""State for state_in and dstate_in for dstate, by the reverse scan that waves of two duties walk (fp16 rows of 128, fp32 rows of 64):
as apart, with more workgroups of segments than the chip has room for."""
import pytest

import test_gpu_delta_use as use
from test_gpu_delta_use import cottn   # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("G", [1, 2, 4])
@pytest.mark.parametrize("dk,dv,dtype", [(64, 64, "f32"), (64, 32, "f32"), (128, 32, "f16"), (128, 128, "f16")])
def test_states_in_place(cottn, G, dk, dv, dtype):   # noqa: F811
    use.test_states_in_place(cottn, G, dk, dv, dtype)
