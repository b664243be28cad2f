"""Properties of the norm's, the output head's and the optimizer's host and device code that only their sources show."""

import os
import re

from test_lm_sources_cpu import ROOT


def function(file, name):
    """The body of the last function of a source file whose definition begins with this text."""
    with open(os.path.join(ROOT, "paper_2504_17672_b200", "csrc", file)) as h:
        text = re.sub(r"//[^\n]*", "", h.read())
    at = text.rindex(name)
    return text[at:text.index("\n}\n", at)]


def test_a_plan_is_on_the_device_when_it_is_handed_out():
    """cudaMemcpy from pageable memory may return before the data has arrived, and streams that do not block do not wait for it."""
    body = function("lm_adam.cu", "cocodc_status cocodc_lm_adam_create(")
    last = body.rindex("cudaMemcpy(")
    assert "cudaStreamSynchronize(cudaStreamLegacy)" in body[last:body.index("*out = plan;")]


def test_a_handle_is_on_the_device_when_it_is_handed_out():
    """Nor do they wait for cudaMemset on the default stream, which need not be done when it returns."""
    for file, name, out in (("lm_api.cu", "cocodc_status cocodc_lm_create(", "*lm_out = lm;"), ("cocodc_api.cu", "cocodc_status cocodc_create(", "*ctx_out = c;")):
        body = function(file, name)
        last = max(body.rfind("cudaMemcpy("), body.rfind("cudaMemset("))
        assert "cudaStreamSynchronize(cudaStreamLegacy)" in body[last:body.index(out)], file


def test_the_norm_records_a_wait_that_gave_up_in_any_warp():
    """Warps of a row give up by themselves: the flag that all of them raise is looked at when the whole block has come to its end."""
    end = function("lm_norm.cu", "void ring_end(")
    assert re.search(r"__syncthreads\(\);\s*if \(threadIdx.x == 0 && \*ring.stop\) record\(status, COCODC_ERR_TIMEOUT\);", end)
    for kernel in ("k_norm(const", "k_norm_grad(const"):
        body = function("lm_norm.cu", kernel)
        assert re.search(r"^  if \(WIDE\) ring_end\(ring, r.t == 0, a.status\);$", body, re.M), kernel       # not in the rows' loop
        assert "COCODC_ERR_TIMEOUT" not in body and "return" not in body[:body.index("ring_end(")].replace("if (WIDE || t >= a.T) return;", "")


def test_no_memory_on_the_device_is_said_so():
    """As the header lists it, and as cocodc_create answers."""
    assert re.search(r"return e == cudaErrorMemoryAllocation \? COCODC_ERR_NOMEM : COCODC_ERR_CUDA;", function("lm_common.cuh", "inline cocodc_status allocate("))
    for file, name in (("lm_adam.cu", "cocodc_status cocodc_lm_adam_create("), ("lm_api.cu", "cocodc_status cocodc_lm_create(")):
        body = function(file, name)
        assert "cudaMalloc" not in body and re.search(r"got = [\w:]*allocate\([^;]*;\s*if \(got != COCODC_OK\) \{\s*delete \w+;\s*return got;", body), file


def test_long_rows_are_walked_without_a_step_past_31_bits():
    """A row may have 2^31 - 1 columns: the step behind the last one leaves an int, and what comes then is below the end again.
    So columns are counted from the row's end, up to 0."""
    for kernel in ("k_norm_long(const", "k_norm_grad_long(const"):
        body = function("lm_norm.cu", kernel)
        assert body.count("for (int c = (int)threadIdx.x - D; c < 0; c += kThreads)") >= 3 and not re.search(r"c < (a\.)?D\b", body), kernel


def test_ends_of_wide_rows_are_told_without_a_sum_past_31_bits():
    """x0 + 64 is past an int for the last columns of a row of almost 2^31; what is left of the row is not."""
    body = function("lm_head_tc.cuh", "void emit(")
    assert "cols - x >= 32" in body and "cols - x0 >= 64" in body and not re.search(r"x0? \+ (32|64) <=", body)
