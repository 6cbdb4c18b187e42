"""GPU: the options of a layer of PagedSequences mean the same over a cache of 16 bits and one of 8."""
import pytest
import torch

from helpers import cuda
from paper_2608_08721_gb300 import binding as lr
from paper_2608_08721_gb300 import prefill

pytestmark = pytest.mark.gpu


def layer(block, **options):
    """Two chunks of two sequences; returns the second's output and whether the device found fault."""
    Hq, Hkv, d = 4, 2, 64
    g = torch.Generator().manual_seed(1)
    seqs = prefill.PagedSequences(1, 2, 128, Hq, Hkv, d, lr.RopeFreqs(d), 120, page_size=32, block=block)
    for n, opts in (([60, 50], {}), ([30, 1], options)):
        step = seqs.begin(n)
        x = torch.randn((sum(n), Hq + 2 * Hkv, d), generator=g).to(torch.bfloat16).to(cuda())
        O = seqs.layer(0, x, step, **opts)
        seqs.end(step)
    seqs.check()
    return O


@pytest.mark.parametrize("block", [0, 16])
def test_options_that_are_none_are_not_given(block):
    none = dict(softcap=None, slopes=None, first_key=None, prefix_len=None, softmax_scale=None)
    for given in (dict(), dict(window=20), dict(window=20, sinks=3)):
        want = layer(block, **given)
        assert torch.equal(layer(block, **given, **none), want)
        assert torch.equal(layer(block, **{"window": None, "sinks": None, **given}), want)


@pytest.mark.parametrize("block", [0, 16])
def test_sinks_without_a_window_hide_and_show_nothing(block):
    assert torch.equal(layer(block, sinks=7), layer(block))


@pytest.mark.parametrize("block", [0, 16])
def test_sinks_that_no_call_takes_are_refused(block):
    first = torch.zeros(31, dtype=torch.int32, device=cuda())
    for opts in (dict(window=20), dict()):
        with pytest.raises(ValueError, match="exclude each other"):
            layer(block, sinks=3, first_key=first, **opts)
        with pytest.raises(lr.LibraspecError):
            layer(block, sinks=-1, **opts)
        assert layer(block, sinks=0, first_key=first, **opts).shape == (31, 4, 64)
