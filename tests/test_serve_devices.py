"""The serving calls take tensors of the current device alone: refusals of the binding, before anything is launched."""
import pytest
import torch

import paper_2508_13337_amd as m


class On:
    """What the binding asks of a tensor, on a device that need not exist."""
    is_cuda = True

    def __init__(self, dev, shape, dtype=torch.bfloat16):
        self.dev, self.shape, self.dtype = dev, torch.Size(shape), dtype

    def get_device(self):
        return self.dev

    def is_contiguous(self):
        return True

    def numel(self):
        return self.shape.numel()

    def dim(self):
        return len(self.shape)

    def data_ptr(self):
        return 256


def calls(dev, other):
    """Every call with its tensors on dev, but for one on other."""
    f32, i32, i8, u8 = torch.float32, torch.int32, torch.int8, torch.uint8
    T, d, E, k, f = 2, 64, 4, 2, 64
    x, y = On(dev, (T, d)), On(dev, (T, d))
    one = lambda *a: On(dev, *a)
    yield lambda: m.xmoe_add_rmsnorm(x, None, On(other, (d,)), 1e-6, None, y=y)
    yield lambda: m.xmoe_add_rmsnorm_bwd(y, None, x, one((d,)), one((T,), f32), On(other, (T, d)), one((d,)), one((4096,), u8))
    yield lambda: m.xmoe_quantize_weights(one((E, d, f)), one((E, f, 128), i8), On(other, (E, f), f32))
    w = lambda: (one((E, f, 128), i8), one((E, f), f32))
    yield lambda: m.xmoe_expert_ffn_q8_fwd(one((T, 128), i8), one((T,), f32), On(other, (E + 1,), i32), *w(), *w(), *w(), y,
                                           one((4096,), u8))
    yield lambda: m.xmoe_layer_few_fwd(x, one((d, E)), None, one((E, d, f)), one((E, d, f)), one((E, f, d)), None,
                                       one((T, E), f32), one((T, k), i32), one((T, k), f32), y, On(other, (4096,), u8))


@pytest.mark.parametrize("which", range(5))
def test_tensors_of_two_devices(which, monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    with pytest.raises(ValueError, match="GPU of the other tensors, 0"):
        list(calls(0, 1))[which]()


@pytest.mark.parametrize("which", range(5))
def test_another_device_than_the_current_one(which, monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    with pytest.raises(ValueError, match="live on GPU 1, the current device is 0"):
        list(calls(1, 1))[which]()


def test_host_memory():
    x = torch.zeros(2, 64)
    with pytest.raises(ValueError, match="x must live on the GPU"):
        m.xmoe_add_rmsnorm(x, None, x[0], 1e-6, None, y=x)
