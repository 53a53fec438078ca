"""The fine-tuning example end to end: a decoder whose images carry no key is taught one, and the detector finds it."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("moment_bits", [8, 32])
def test_finetuned_decoder_writes_the_key(moment_bits):
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import finetune_decoder
    finally:
        sys.path.pop(0)
    history, results = finetune_decoder.main(steps=200, moment_bits=moment_bits, report=lambda s: print(s, flush=True))
    # a bit that says nothing costs log 2; half of them wrong and the penalty lie well above a decoder that has learnt most of them
    assert history[-1] < 0.2 * history[0]
    assert results["before"]["detected"] == 0 and abs(results["before"]["wrong"] - 24) < 8
    assert results["after"]["detected"] >= 12 and results["after"]["wrong"] < 6
