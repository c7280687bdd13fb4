"""A given stream has to be of the device that the arrays are on (no GPU needed): a kernel
launched with that device's pointers on another device's stream would fault."""
import types

import pytest
import torch

import paper_2505_17826_amd as R


def test_a_stream_of_another_device_is_refused(monkeypatch):
    ran = []
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    fn = lambda *a: ran.append(a) or R.RFT_OK  # noqa: E731
    stream = lambda i: types.SimpleNamespace(  # noqa: E731
        cuda_stream=7, device=torch.device("cuda", i), device_index=i)
    with pytest.raises(RuntimeError, match="cuda:1"):
        R._call(fn, torch.device("cuda", 0), stream(1), 1)
    assert not ran
    R._call(fn, torch.device("cuda", 0), stream(0), 1)
    assert ran == [(1, 7)]
