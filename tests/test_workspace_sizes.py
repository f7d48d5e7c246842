"""The sizes of workspaces go by the SMs of the current device: the binding asks for them once for each
device, not once for all.  No GPU is needed: a library stands in whose sizes tell the device."""
import pytest
import torch

SIZES = {"sn_embed_bwd_workspace": (4, 32, 64), "sn_rmsnorm_bwd_workspace": (4, 64),
         "sn_blocknorm_bwd_workspace": (4, 64, 2), "sn_glu_bwd_workspace": (4, 64, 32)}


@pytest.fixture
def devices(monkeypatch):
    """(the binding, the present device in a list, the devices that sizes were asked on)."""
    from paper_2506_01260_gb300 import sn
    present, asked = [0], []

    class Library:
        def __getattr__(self, name):
            def size(*args):
                asked.append(present[0])
                args[-1]._obj.value = 1000 * (present[0] + 1)
                return 0
            return size

    monkeypatch.setattr(sn, "_lib", Library())
    monkeypatch.setattr(torch.cuda, "is_initialized", lambda: present[0] is not None)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: present[0])
    for name in SIZES:
        getattr(sn, name).cache_clear()
    yield sn, present, asked
    for name in SIZES:
        getattr(sn, name).cache_clear()


@pytest.mark.parametrize("name", sorted(SIZES))
def test_a_size_for_each_device(devices, name):
    sn, present, asked = devices
    size = getattr(sn, name)
    for turn in range(2):
        for present[0] in (0, 1):
            assert size(*SIZES[name]) == 1000 * (present[0] + 1)
    assert asked == [0, 1]


def test_arguments_by_name(devices):
    sn, present, asked = devices
    for present[0] in (0, 1, 0, 1):
        assert sn.sn_glu_bwd_workspace(T=4, d=64, f=32) == 1000 * (present[0] + 1)
    assert asked == [0, 1]


@pytest.mark.parametrize("name", sorted(SIZES))
def test_sizes_asked_for_before_a_device_is_in_use_are_not_kept(devices, name, monkeypatch):
    sn, present, asked = devices
    size = getattr(sn, name)
    monkeypatch.setattr(torch.cuda, "is_initialized", lambda: False)
    for present[0] in (0, 1, 0):
        assert size(*SIZES[name]) == 1000 * (present[0] + 1)
    assert asked == [0, 1, 0]
