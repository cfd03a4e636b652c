"""Sparse and shared generations over prefixes without a token."""
import pytest

from test_gpu_parts import log, torch_dev  # noqa: F401
from test_gpu_serving_step import Step

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kw", [dict(lens=(0, 0, 0), shared=0), dict(lens=(0, 0, 0)), dict(lens=(0, 0, 0), select=None), dict(lens=(1, 0, 0))],
                         ids=["selected", "selected_shared", "own", "one_token"])
def test_steps_over_empty_prefixes(torch_dev, kw):
    log(f"[case] empty {kw}")
    st = Step(torch_dev, "bf16", **kw)
    for i in range(2):
        st.new_inputs(20 + i)
        st.run()
        torch_dev.cuda.synchronize()
        st.check(f"step {i}")
        st.gen.advance()
