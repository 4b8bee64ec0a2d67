"""What the descriptors of the dropout, LayerNorm and 8-bit calls take from tensors and refuse.  No GPU needed."""
import pytest

from paper_2410_05985_amd import layup as LU

torch = pytest.importorskip("torch")


def test_offset_from_the_device_is_a_64_bit_integer():
    """The kernels read eight bytes there."""
    x = torch.zeros(4, 8)
    for t in (torch.int64, torch.uint64):
        assert LU.dropout_desc(x, x, p=0.5, offset_dev=torch.zeros(1, dtype=t)).drop.offset_dev
    assert LU.dropout_desc(x, x, p=0.5, offset_dev=0x1000).drop.offset_dev == 0x1000
    for bad in (torch.zeros(1, dtype=torch.int32), torch.zeros(1), torch.zeros(0, dtype=torch.int64)):
        with pytest.raises(ValueError):
            LU.dropout_desc(x, x, p=0.5, offset_dev=bad)
        with pytest.raises(ValueError):
            LU.layernorm_desc(x, x, p=0.5, offset_dev=bad)


def test_workspace_is_one_piece_of_memory():
    """Its bytes are counted from its elements: an expanded or strided one holds fewer, or others' between them."""
    x, v = torch.zeros(4, 8), torch.zeros(4)
    q = torch.zeros(4, 128, dtype=torch.uint8).view(torch.float8_e4m3fn)
    e = torch.zeros(4, 4, dtype=torch.uint8)
    room = torch.zeros(4096, dtype=torch.uint8)
    assert LU.layernorm_grad_desc(x, x, v, v, workspace=room).workspace_bytes == 4096
    assert LU.gemm_fp8_desc(q, e, 1, q, e, 1, torch.zeros(4, 4), 128, workspace=room).workspace_bytes == 4096
    assert not LU.layernorm_grad_desc(x, x, v, v).workspace
    for bad in (room[::2], torch.zeros(1).expand(1 << 20)):
        with pytest.raises(ValueError):
            LU.layernorm_grad_desc(x, x, v, v, workspace=bad)
        with pytest.raises(ValueError):
            LU.gemm_fp8_desc(q, e, 1, q, e, 1, torch.zeros(4, 4), 128, workspace=bad)


class Stream:
    cuda_stream = 0x1234

    def __init__(self, device):
        self.device_index = device


def descriptor_on(device):
    """A descriptor as of tensors on that GPU."""
    return LU._keep(LU.layup_dropout_desc(), Tensor(device))


class Tensor:
    def __init__(self, device):
        self.device = torch.device("cuda", device)


def test_a_stream_of_another_device_is_refused():
    calls = []
    f = lambda d, s: calls.append(s) or LU.LAYUP_OK  # noqa: E731
    with pytest.raises(ValueError):
        LU._call(f, descriptor_on(1), Stream(0))
    assert not calls
    LU._call(f, descriptor_on(1), Stream(1))
    LU._call(f, descriptor_on(1), 0x5678)  # a bare hipStream_t is the caller's word
    assert calls == [0x1234, 0x5678]


def test_no_stream_is_the_default_stream_of_the_tensors_device(monkeypatch):
    """NULL is the current device's default stream: that device has to be the tensors' during the call."""
    current, seen = [0], []

    class Device:
        def __init__(self, d):
            self.d = d

        def __enter__(self):
            self.old, current[0] = current[0], self.d

        def __exit__(self, *_):
            current[0] = self.old

    monkeypatch.setattr(torch.cuda, "current_device", lambda: current[0])
    monkeypatch.setattr(torch.cuda, "device", Device)
    for dev in (1, 0):
        LU._call(lambda d, s: seen.append((s, current[0])) or LU.LAYUP_OK, descriptor_on(dev), None)
    assert seen == [(None, 1), (None, 0)] and current == [0]
