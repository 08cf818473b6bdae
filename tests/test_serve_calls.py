"""The served steps' Python calls without a GPU: what they do before the library
is called (torch's devices and streams are stood in for)."""
import contextlib
import ctypes as C

import pytest
import torch

from paper_2609_02109_amd import mf, serve


class Stream:
    def __init__(self, device, handle):
        self.device, self.cuda_stream = device, handle

    def __eq__(self, other):
        return self.device == other.device and self.cuda_stream == other.cuda_stream


class Rows:
    """As much of a tensor as a product asks of one."""
    requires_grad = False

    def __init__(self, *shape, device):
        self.shape, self.dtype, self.device = torch.Size(shape), torch.bfloat16, device

    def stride(self, d):
        return self.shape[1] if d == 0 else 1

    def data_ptr(self):
        return 4096

    def new_empty(self, shape):
        return Rows(*shape, device=self.device)


@pytest.fixture
def card(monkeypatch):
    """Two devices; -> what is current, and the (device, stream) of every launch."""
    now, launched = dict(device=0, stream={0: 0, 1: 0}), []

    @contextlib.contextmanager
    def device(d):
        before, now["device"] = now["device"], torch.device(d).index
        yield
        now["device"] = before

    @contextlib.contextmanager
    def stream(s):
        at, before = now["device"], now["stream"][s.device.index]
        now["device"], now["stream"][s.device.index] = s.device.index, s.cuda_stream
        yield
        now["device"], now["stream"][s.device.index] = at, before

    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(torch.cuda, "stream", stream)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda d=None: Stream(d, now["stream"][torch.device(d).index]))
    monkeypatch.setattr(serve, "_current_device", lambda: now["device"], raising=False)
    monkeypatch.setattr(serve, "_raw_stream", lambda i: now["stream"][i])

    class Lib:
        @staticmethod
        def mf_w4_matmul(args, ws, nbytes, stream):
            launched.append((now["device"], stream))
            return mf.MF_OK

        @staticmethod
        def mf_w4_workspace_size(args, nbytes):
            return mf.MF_OK

    monkeypatch.setattr(mf, "lib", Lib)
    return now, launched


def _weight(device):
    w = object.__new__(serve.W4Weight)
    w.n_out, w.n_in, w.group, w.dtype, w.device = 64, 128, 128, torch.bfloat16, device
    w.desc, w.packed, w._packed_ptr, w._ws_bytes = serve.W4Desc(64, 128, 128, mf.MF_BF16), None, 256, {}
    return w


def test_a_call_runs_on_its_tensors_device(card):
    now, launched = card
    here, there = torch.device("cuda", 0), torch.device("cuda", 1)
    for d in (here, there):
        y = _weight(d).matmul(Rows(2, 128, device=d))
        assert y.device == d and now["device"] == 0
        _weight(d).matmul(Rows(2, 128, device=d), stream=Stream(d, 77))
        assert now == dict(device=0, stream={0: 0, 1: 0})
    assert launched == [(0, 0), (0, 77), (1, 0), (1, 77)]


def test_a_stream_of_another_device_is_refused(card):
    d = torch.device("cuda", 1)
    with pytest.raises(ValueError):
        _weight(d).matmul(Rows(2, 128, device=d), stream=Stream(torch.device("cuda", 0), 77))
    assert card[1] == []


def test_a_batch_of_another_device_is_refused():
    cache, batch = object.__new__(serve.KV4Cache), object.__new__(serve.KV4Batch)
    cache.device, batch.device = torch.device("cuda", 0), torch.device("cuda", 1)
    for call in (lambda: cache.append(batch, None, None), lambda: cache.read(batch), lambda: cache.attention(batch, None)):
        with pytest.raises(ValueError):
            call()


@pytest.mark.parametrize("n,want", [(2 ** 27 - 16, mf.MF_OK), (2 ** 27 - 15, mf.MF_EUNSUPPORTED), (2 ** 31 - 16, mf.MF_EUNSUPPORTED)])
def test_w4_outputs_that_one_launch_takes(n, want):
    """Every call says so, the sizes' too."""
    d, nb = serve.W4Desc(n, 32, 32, mf.MF_BF16), C.c_size_t()
    a = serve.W4Args(d, 256, 1024, None, 4096, 0, 32, n)
    assert mf.lib.mf_w4_pack_bytes(C.byref(d), C.byref(nb)) == want
    assert mf.lib.mf_w4_workspace_size(C.byref(a), C.byref(nb)) == want
    assert mf.lib.mf_w4_matmul(C.byref(a), None, 0, None) == want
    if want:
        assert mf.lib.mf_w4_pack(C.byref(d), 1024, 2048, None, 4096, C.c_size_t(1 << 40), None) == want


@pytest.mark.parametrize("field", ["n_pages", "page_size", "n_kv_heads", "head_dim", "group"])
@pytest.mark.parametrize("past", [2 ** 32, -2 ** 32, 2 ** 64])
def test_sizes_past_32_bits_are_refused(field, past):
    """Not taken without their upper bits, as which they would be sizes that there are."""
    sizes = dict(n_pages=4, page_size=16, n_kv_heads=2, head_dim=64, group=32)
    with pytest.raises(ValueError):
        serve.KV4Cache(**{**sizes, field: sizes[field] + past})


class Ints:
    """As much of an int32 tensor as a batch asks of one."""
    dtype, is_cuda, device = torch.int32, True, torch.device("cuda", 0)

    def __init__(self, *shape):
        self.shape = torch.Size(shape)

    def dim(self):
        return len(self.shape)

    def is_contiguous(self):
        return True

    def stride(self, d):
        return self.shape[1] if d == 0 else 1

    def data_ptr(self):
        return 4096


@pytest.mark.parametrize("sizes", [dict(max_new=2 ** 32 + 1), dict(max_kv=2 ** 32 + 20), dict(rows=2 ** 64 + 1), dict(max_new=2 ** 31)])
def test_a_batch_past_32_bits_is_refused(monkeypatch, sizes):
    monkeypatch.setattr(serve, "isinstance", lambda t, kind: type(t) is Ints if kind is torch.Tensor else isinstance(t, kind), raising=False)
    good = dict(rows=1, max_new=1, max_kv=20)
    assert serve.KV4Batch(Ints(2), Ints(1), Ints(1, 4), **good).raw.max_kv == 20
    with pytest.raises(ValueError):
        serve.KV4Batch(Ints(2), Ints(1), Ints(1, 4), **{**good, **sizes})
