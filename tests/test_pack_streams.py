"""Packing allocates its result: the call has to stand between what torch's current stream did before and what it does next, whichever
stream it runs on.  Without a GPU: who waits for whom, and when."""
import types

import pytest
import torch

from paper_2605_11186_amd import binding

EVENTS = []


class Stream:
    def __init__(self, handle, device_index=0):
        self.cuda_stream, self.device_index = handle, device_index

    def wait_stream(self, other):
        EVENTS.append(("wait", self.cuda_stream, other.cuda_stream))


class Matrix:
    """What the binding asks of a device tensor."""
    device = "cpu"

    def __init__(self, dtype):
        self.dtype, self.shape = dtype, (16, 256)

    def get_device(self):
        return 0

    def stride(self):
        return 256, 1

    def data_ptr(self):
        return 1 << 20


CURRENT, DEFAULT, OTHER = Stream(11), Stream(0), Stream(22)


@pytest.fixture
def calls(monkeypatch):
    del EVENTS[:]
    binding._load_types()
    monkeypatch.setattr(binding, "_current_device", lambda: 0)

    def pack(*args):
        EVENTS.append(("pack", args[-1] or 0))
        return 0

    library = types.SimpleNamespace(cats_pack_matrix=pack, cats_pack_quantized_matrix=pack, cats_packed_matrix_bytes=lambda r, c: 2 * r * c,
                                    cats_packed_quantized_bytes=lambda r, c: r * c)
    monkeypatch.setattr(binding, "library", lambda: library)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: CURRENT)
    monkeypatch.setattr(torch.cuda, "default_stream", lambda device=None: DEFAULT)
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle, device=None: Stream(handle))
    return EVENTS


@pytest.mark.parametrize("pack,dtype", [(binding.cats_pack_matrix, torch.bfloat16), (binding.cats_pack_quantized_matrix, torch.int8)])
def test_packing_stands_between_the_current_streams_work(calls, pack, dtype):
    for stream, handle in ((None, 0), (0, 0), (DEFAULT, 0), (OTHER, 22), (33, 33)):
        del calls[:]
        pack(Matrix(dtype), stream=stream)
        assert calls == [("wait", handle, 11), ("pack", handle), ("wait", 11, handle)]
    for stream in (CURRENT, 11):
        del calls[:]
        pack(Matrix(dtype), stream=stream)
        assert calls == [("pack", 11)]


def test_a_stream_of_another_device_is_refused(calls):
    with pytest.raises(binding.CatsError):
        binding.cats_pack_quantized_matrix(Matrix(torch.int8), stream=Stream(5, device_index=1))
    assert calls == []


@pytest.mark.gpu
@pytest.mark.parametrize("default", [True, False])
def test_weights_made_and_packed_on_a_side_stream(default):
    """Weights that a side stream is still at work on, packed on the default stream and on another one, and dropped at once."""
    import paper_2605_11186_amd as cats
    side, other = torch.cuda.Stream(), torch.cuda.Stream()
    gen = torch.Generator(device="cuda").manual_seed(1)
    w8 = torch.randint(-128, 128, (2048, 2048), dtype=torch.int8, device="cuda", generator=gen)
    w16 = torch.randn(2048, 2048, device="cuda", generator=gen).to(torch.bfloat16)
    want = cats.cats_pack_quantized_matrix(w8), cats.cats_pack_matrix(w16)
    torch.cuda.synchronize()
    on = None if default else other
    for _ in range(3):
        with torch.cuda.stream(side):
            for _ in range(20):
                torch.mm(w16, w16)   # the stream is busy
            a = w8.clone()
            b = w16.clone()
            pa, pb = cats.cats_pack_quantized_matrix(a, stream=on), cats.cats_pack_matrix(b, stream=on)
            del a, b
            for _ in range(3):   # takes the places of what was dropped
                torch.full((2048, 2048), 3, dtype=torch.int8, device="cuda"), torch.full_like(w16, 3)
            same = torch.equal(pa, want[0]), torch.equal(pb.view(torch.int16), want[1].view(torch.int16))
        assert same == (True, True)
