"""Replays the GPU tests of scales over the whole range of FP32 on the CPU execution model, as tests/test_host_model_replay_experts.py does
for the expert rows."""
import pytest

from test_host_model_replay_b128 import hostmodel_lib, test_gpu_tests_pass_on_the_host_model as _replay  # noqa: F401


@pytest.mark.parametrize("file,at_least", [("test_gpu_b128_scales.py", 51)])
def test_gpu_tests_of_scales_pass_on_the_host_model(hostmodel_lib, file, at_least):  # noqa: F811
    _replay(hostmodel_lib, file, at_least)
