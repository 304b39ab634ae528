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


def _constant(source, name):
    return int(eval(re.search(rf"constexpr \w+ {name} = ([^;]+);", source).group(1)))


def test_nucleus_error_bound():
    # the relative difference between the scan's float mass of what it did not list and the whole
    # numbers' sum, in units of 2^-24, by the longest way that an element's share can take
    vocab, sample = _source("vocab.cuh"), _source("sample.cu")
    warps, unit = 256 // 32, _constant(vocab, "kUnit")
    room, listed = _constant(sample, "kSampleRoom"), _constant(sample, "kNucleus")
    units = -(-_constant(vocab, "kVocabMax") * 4 // 16 // warps // unit)   # of a warp, at the most
    cuts = units // (room - 32 - listed)                                  # from more than room - 32 to `listed`
    steps, refreshes, at = -(-units // 32), 1, 1                           # after the 2nd, 8th, ... and the last
    while at < steps:
        refreshes, at = refreshes + 1, 4 * at + 3
    ex2, expf, product, bits = 4, 4, 1, 40
    exponent = bits * 0.6931472 * ((1 + 1 + 1.23) + (1 + 1))  # z - ref, times c, c's own; z - m, times 1 / T
    raises = (refreshes + cuts + 3 + 3) * (ex2 + product)     # + most_of_many's, + the join's and its own selection
    drops = (ex2 + product) + (room + 31) // 32 * (refreshes + cuts + 1)   # additions to a lane's sum
    selection = unit + unit + 8 + 8 + 8                       # most_of_many, emit and merge: windows, elements, keys
    end = room * unit // 32 + room * 8 // 32 + 1 + 3          # candidates: windows and elements of a lane
    sums = 6 + 2 + 2 * (5 + warps - 1)                        # a unit, the compensated sum, block_reduce twice
    total = exponent + ex2 + expf + raises + drops + selection + end + sums + (ex2 + product)
    assert total * 2.0 ** -24 <= 1.0 / _constant(sample, "kMassError"), (total, cuts, refreshes)
