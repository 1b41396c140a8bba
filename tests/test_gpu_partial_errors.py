"""What the calls of a selection of pages record reaches its user, and the user of the steps that draft over it."""
import pytest
import torch

from paper_2604_26412_gb300 import kvshot
from paper_2604_26412_gb300.partial import PageSelection
from paper_2604_26412_gb300.step import DraftStep

from .test_gpu_partial_step import inputs

pytestmark = pytest.mark.gpu


def test_errors_of_a_selection_are_reported():
    inp = inputs(lens=(200, 0, 130, 1000))
    pages = PageSelection(inp, keep=5)
    step = DraftStep(inp, pages=pages)
    good = inp.page_table[0, 1].clone()
    inp.page_table[0, 1] = -5
    pages.update()
    inp.page_table[0, 1] = good
    step.run()  # (all of its own calls are right)
    torch.cuda.synchronize()
    assert step.error_code() == kvshot.KVSHOT_ERR_DEVICE_BOUNDS
    assert pages.error_code() == kvshot.KVSHOT_ERR_DEVICE_BOUNDS
    assert pages.error_code() == 0 and step.error_code() == 0
    quiet = DraftStep(inp, pages=pages, err_flag=False)
    quiet.run()
    assert quiet.error_code() == 0
