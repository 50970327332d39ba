"""Kernels that share an SM's tensor memory with others: a CTA that holds columns must not wait for another CTA, which may itself
be waiting for columns (an allocation has no limit).  Two kernels of the library may lie on an SM only by linear_few_kernel;
the others take all columns and next to all of the shared memory.  Read off the source: a run that shows the fault does not end."""
import os
import re

from paper_2605_06665_b200 import build as builder


def source(name):
    return open(os.path.join(builder.CSRC, name)).read()


def test_few_token_kernel_returns_its_columns_before_it_waits_for_its_cluster():
    text = source("linear_tc.cu")
    body = text[text.index("linear_few_kernel(const __grid_constant__"):text.index("int launch_few(")]
    body = re.sub(r"//[^\n]*", "", body)
    alloc, free, wait = (body.index(w) for w in ("tc::tmem_alloc(", "tc::tmem_dealloc(", "tc::cluster_sync("))
    assert alloc < free < wait and body.count("tc::tmem_dealloc(") == 1


def test_no_more_few_token_ctas_on_an_sm_than_columns():
    text = source("linear_tc.cu")
    least = int(re.search(r"kFewSmemLeast = (\d+);", text).group(1))
    columns = int(re.search(r"kFewColumns = (\d+);", text).group(1))
    assert (512 // columns + 1) * (least + 1024) > 228 * 1024          # one more does not fit
    assert re.search(r"std::max\(2048 \+ bytes, kFewSmemLeast\)", text)
