"""Properties of the norm's, the output head's and the optimizer's host and device code that only their sources show."""

from test_lm_sources_cpu import sources


def function(file, name):
    """The body of the last function of a source file whose definition begins with this text."""
    (text,) = [t for f, t in sources() if f == file]
    at = text.rindex(name)
    return text[at:text.index("\n}\n", at)]


def test_a_plan_is_on_the_device_when_it_is_handed_out():
    """cudaMemcpy from pageable memory may return before the data has arrived, and streams that do not block do not wait for it."""
    body = function("lm_adam.cu", "cocodc_status cocodc_lm_adam_create(")
    last = body.rindex("cudaMemcpy(")
    assert "cudaStreamSynchronize(cudaStreamLegacy)" in body[last:body.index("*out = plan;")]
