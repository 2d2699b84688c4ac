"""The workspace argument of every call: memory of the GPU, or none, which the library refuses."""
import pytest
import torch

import paper_2606_10896_amd as gmm


@pytest.mark.parametrize("ws", [torch.empty(4096, dtype=torch.uint8), [0] * 4096, 4096])
def test_what_is_no_memory_of_the_gpu_is_refused(ws):
    with pytest.raises(TypeError):
        gmm._ws(ws)


def test_none_is_no_workspace():
    assert gmm._ws(None) == (0, 0)


def test_every_call_checks_it():
    """No call takes a workspace's address or size by itself."""
    for mod in (gmm, gmm.kv):
        with open(mod.__file__) as f:
            text = f.read()
        assert text.count("ws.data_ptr()") + text.count("ws.numel()") == (2 if mod is gmm else 0)
        assert "_ptr(ws)" not in text
