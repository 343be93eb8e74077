"""Tensors that the binding of the paged key/value cache refuses: on the host, on another
device than the pool, or with gaps.  Stand-ins for tensors and library; nothing is launched.
No GPU."""
import types

import pytest
import torch

from paper_2608_02474_gb300 import echocache as ec

BF16, I32 = torch.bfloat16, torch.int32


class Fake:
    """What the binding asks of a tensor; gpu -1 is the host."""

    def __init__(self, shape, dtype, gpu=0, stride=None):
        self.shape, self.dtype, self.gpu = torch.Size(shape), dtype, gpu
        packed = [1]
        for n in reversed(self.shape[1:]):
            packed.insert(0, packed[0] * n)
        self.strides = tuple(stride or packed)
        self.contiguous = self.strides == tuple(packed)
        self.is_cuda = gpu >= 0
        self.device = torch.device("cuda", gpu) if gpu >= 0 else torch.device("cpu")

    def stride(self):
        return self.strides

    def is_contiguous(self):
        return self.contiguous

    def get_device(self):
        return self.gpu

    def dim(self):
        return len(self.shape)

    def numel(self):
        return self.shape.numel()

    @property
    def nbytes(self):
        return self.numel() * self.dtype.itemsize

    def data_ptr(self):
        return 0x10000


@pytest.fixture
def calls(monkeypatch):
    """Names of the library's calls that were made."""
    made = []
    fake = types.SimpleNamespace(echo_kv_attention_workspace_size=lambda *a: 4096)
    for name in ("echo_kv_write", "echo_kv_read", "echo_kv_attention"):
        setattr(fake, name, lambda *a, name=name: made.append(name) or 0)
    monkeypatch.setattr(ec, "lib", lambda: fake)
    monkeypatch.setattr(ec, "_stream", lambda stream=None: None)
    return made


def pool(gpu=0):
    return ec.KVPool(Fake((4, 2, 2, 16, 64), BF16, gpu))


def batch(gpu=0, n=5):
    return ec.KVBatch(Fake((2, 3), I32, gpu), Fake((2,), I32, gpu), Fake((3,), I32, gpu), n)


def rows(gpu=0, dtype=BF16, stride=None):
    return Fake((5, 128), dtype, gpu, stride)


def attend(**change):
    a = dict(pool=pool(), batch=batch(), q=rows(), out=rows(), workspace=Fake((4096,), torch.uint8))
    a.update(change)
    return ec.echo_kv_attention(a.pop("pool"), a.pop("batch"), a.pop("q"), **a)


def test_calls_that_are_right(calls):
    attend()
    ec.echo_kv_write(pool(), batch(), rows(), rows())
    ec.echo_kv_read(pool(), batch(), k=rows(), v=rows())
    attend(pool=pool(1), batch=batch(1), q=rows(1), out=rows(1), workspace=Fake((1024,), torch.float32, 1))
    assert calls == ["echo_kv_attention", "echo_kv_write", "echo_kv_read", "echo_kv_attention"]


@pytest.mark.parametrize("gpu", [-1, 1])
def test_tensors_that_are_elsewhere(calls, gpu):
    for change in (dict(q=rows(gpu)), dict(out=rows(gpu)), dict(workspace=Fake((4096,), torch.uint8, gpu))):
        with pytest.raises(ValueError, match="CUDA"):
            attend(**change)
    for k, v in ((rows(gpu), rows()), (rows(), rows(gpu))):
        with pytest.raises(ValueError, match="CUDA"):
            ec.echo_kv_write(pool(), batch(), k, v)
        with pytest.raises(ValueError, match="CUDA"):
            ec.echo_kv_read(pool(), batch(), k=k, v=v)
    assert not calls


def test_a_workspace_with_gaps(calls):
    with pytest.raises(ValueError, match="workspace"):
        attend(workspace=Fake((64, 64), torch.uint8, stride=(128, 1)))
    assert not calls


def test_pool_and_batch_on_two_devices(calls):
    for p, b in ((pool(), batch(1)), (pool(1), batch())):
        with pytest.raises(ValueError, match="one device"):
            attend(pool=p, batch=b)
        with pytest.raises(ValueError, match="one device"):
            ec.echo_kv_write(p, b, rows(), rows())
    with pytest.raises(ValueError, match="one device"):
        ec.KVPool(Fake((4, 2, 2, 16, 64), torch.int8), Fake((4, 2, 2, 16), torch.float32, 1))
    for gpus in ((0, 1, 0), (0, 0, 1), (1, 0, 0)):
        with pytest.raises(ValueError, match="one device"):
            ec.KVBatch(Fake((2, 3), I32, gpus[0]), Fake((2,), I32, gpus[1]), Fake((3,), I32, gpus[2]), 5)
    assert not calls
