"""A sample of the planted kernel mistakes (tests/host_model/mutation_check.py) in every run: all of them together take minutes, but
that the copies still build, pass without a mistake and fail with one must show without them."""
from test_mutation_checks import _run


def test_host_model_catches_a_sample_of_planted_kernel_mistakes():
    out = _run("tests/host_model/mutation_check.py", "(unmutated converters", "quantizer: MXFP4 blocks with a NaN", timeout=900)
    assert "2 of 2 as expected (1 planted mistakes)" in out
