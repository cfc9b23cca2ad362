"""Arguments of the output head's Python classes that are refused before any call:
tensors on another GPU than the object's.  With stand-ins for tensors, so that it
needs neither a GPU nor two of them."""
import types

import pytest
import torch

from paper_2511_12500_amd import head, heap


class Tensor:
    """What the argument checks read of a contiguous device tensor."""
    is_cuda = True

    def __init__(self, shape, dtype, device):
        self.shape, self.dtype = torch.Size(shape), dtype
        self.device = torch.device("cuda", device)

    def dim(self):
        return len(self.shape)

    def stride(self, i=None):
        s = torch.empty(self.shape, device="meta").stride()
        return s if i is None else s[i]

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 1 << 20

    def get_device(self):
        return self.device.index


def bare(cls, **attributes):
    """An object without its constructor's GPU memory."""
    o = object.__new__(cls)
    o.__dict__.update(attributes)
    return o


def test_rows_of_another_gpu_are_refused():
    bf = torch.bfloat16
    op = bare(head.TokenLogprobs, rows=4, vocab=100, dtype=bf, device=0)
    here, there = Tensor((4, 100), bf, 0), Tensor((4, 100), bf, 1)
    assert op._matrices(here, here) == (100, 100)
    for logits, dlogits in ((there, None), (here, there)):
        with pytest.raises(ValueError, match="cuda:0"):
            op._matrices(logits, dlogits)
    one, other = Tensor((4,), torch.float32, 0), Tensor((4,), torch.float32, 1)
    assert op._grads(one, None, one) == [1 << 20, None, 1 << 20]
    with pytest.raises(ValueError, match="cuda:0"):
        op._grads(None, other, None)
    kd = bare(head.TopDistillation, rows=4, vocab=100, dtype=bf, device=1, k=3, mode=0)
    ids, values = Tensor((4, 3), torch.int64, 1), Tensor((4, 3), torch.float32, 1)
    kd._list(ids, values)
    for a, b in ((Tensor((4, 3), torch.int64, 0), values), (ids, Tensor((4, 3), torch.float32, 0))):
        with pytest.raises(ValueError, match="cuda:1"):
            kd._list(a, b)


def test_weights_and_tokens_of_another_gpu_are_refused():
    bf, u8 = torch.bfloat16, torch.uint8
    q, scales = Tensor((16, 32), u8, 1), Tensor((16, 2), bf, 1)
    weight = head.W4Weight(q, scales, None, 32)
    for bad in ((q, Tensor((16, 2), bf, 0), None), (q, scales, Tensor((16, 2), u8, 0))):
        with pytest.raises(ValueError, match="one GPU"):
            head.W4Weight(*bad, 32)
    for device, x, w in ((1, 0, weight), (0, 0, weight), (0, 1, weight)):
        out = bare(heap.GatheredOutput, heap=types.SimpleNamespace(device=device), dtype=bf, M=2,
                   N_local=16, tile_m=64, tile_n=16)
        with pytest.raises(ValueError, match=f"cuda:{device}"):
            out.run_w4(Tensor((2, 64), bf, x), w, 0)
