"""Scratch of the chunk calls is on the device of their tensors (host only)."""
import pytest
import torch

from paper_2609_13141_amd import sas


def test_scratch_of_another_device_is_refused():
    with pytest.raises(sas.SasError, match="scratch on cpu"):
        sas._scratch(sas.Workspace("cpu"), 64, torch.device("cuda", 0))
    buf = sas._scratch(sas.Workspace("cpu"), 64, torch.device("cpu"))
    assert buf.numel() >= 64
