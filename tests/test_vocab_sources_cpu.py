"""What the operators over vocabulary logits rest on beyond what a run shows, read
from their sources."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_34117_gb300", "csrc")


def _source(name):
    with open(os.path.join(CSRC, name)) as f:
        return f.read()


def test_arrays_of_a_kernel_that_runs_already_are_not_called_read_only():
    # a kernel that is launched programmatically starts while the one before it still writes: reads
    # of that one's arrays through __restrict__ const pointers need not be coherent
    source = _source("distill_loss.cu")
    parameters = re.search(r"loss_sum_kernel\((.*?)\) \{", source, re.S).group(1).split(",")
    row_loss = [p for p in parameters if "row_loss" in p]
    assert len(row_loss) == 1 and "__restrict__" not in row_loss[0]
