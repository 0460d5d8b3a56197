"""What the checks of a product's arguments cost the host: they run before every product, the smallest of which takes the GPU a few
microseconds."""
import sys

import pytest
import torch

from paper_2606_00539_gb300 import ExpertProducts
from paper_2606_00539_gb300 import products as module


@pytest.fixture(scope="module", autouse=True)
def loaded():
    if module.torch is None:
        module._load_torch()


def test_the_check_for_gradients_enters_no_frame_of_its_own():
    x, w = torch.zeros(2, 2), torch.zeros(2, 2)
    frames = []
    sys.setprofile(lambda frame, event, arg: frames.append(frame.f_code.co_name) if event == "call" else None)
    try:
        ExpertProducts._no_graph(x, w)
    finally:
        sys.setprofile(None)
    assert frames == ["_no_graph"]


def test_the_check_for_gradients():
    x, w = torch.zeros(2, 2), torch.zeros(2, 2)
    for operands in ((x, w), (x,)):
        ExpertProducts._no_graph(*operands)
    w.requires_grad_()
    for operands in ((x, w), (w, x), (w,)):
        with pytest.raises(ValueError, match="expert_linear or expert_gated"):
            ExpertProducts._no_graph(*operands)
        with torch.no_grad():
            ExpertProducts._no_graph(*operands)
