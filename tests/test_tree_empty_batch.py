"""A step without sequences: the calls that take a batch of none do nothing, whatever their tensors' addresses are."""
import pytest
import torch

from paper_2503_16257_amd import binding as vk

DEV = "cuda:0"


def step(dev):
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device=dev)  # noqa: E731
    masks = torch.zeros((0, 70, 2), dtype=torch.int64, device=dev)
    vk.tree_masks(i32(0, 70), masks)
    vk.tree_masks(None, masks, i32(0), i32(3, 0, 70), count=i32(0))
    rows = torch.zeros((0, 70, 99), device=dev)
    ws = torch.zeros(256, dtype=torch.uint8, device=dev)
    vk.tree_verify(rows, i32(0, 70), torch.zeros((0, 70), device=dev), i32(0, 70), i32(0), i32(0), ws)
    vk.tree_verify(rows, i32(0, 70), torch.zeros((0, 70), device=dev), i32(0, 70), i32(0), i32(0), ws, draft=rows, parents=i32(0, 70),
                   count=i32(0), distinct=True)
    # what does not fit is refused all the same
    with pytest.raises(ValueError):
        vk.tree_masks(i32(0, 69), masks)
    with pytest.raises(ValueError):
        vk.tree_masks(i32(0, 70), masks[:, :, :1])
    with pytest.raises(ValueError):
        vk.tree_masks(i32(0, 70), masks, i32(0), i32(3, 0, 69))


def test_the_marshalling_in_python(monkeypatch):
    """(Without a GPU: tensors on the host are taken for the device's; nothing is launched.)"""
    vk.lib()

    def arg(t, dtype, name, shape=None):
        if t is not None and shape is not None and tuple(t.shape) != shape:
            raise ValueError(name)
        return None if t is None else t.data_ptr()
    monkeypatch.setattr(vk, "_native", None)
    monkeypatch.setattr(vk, "_arg", arg)
    monkeypatch.setattr(vk, "_rows", lambda t, name, shape: None)
    monkeypatch.setattr(vk, "_stream", lambda s: None)
    step("cpu")


@pytest.mark.gpu
@pytest.mark.parametrize("native", [True, False])
def test_on_the_gpu(native, monkeypatch):
    vk.lib()
    if not native:
        monkeypatch.setattr(vk, "_native", None)
    step(DEV)
