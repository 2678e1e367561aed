"""What the tensor layer of the stage operators does on the host: no GPU."""

import pytest
import torch


@pytest.fixture
def host(libssn, monkeypatch):
    """Tensors on the host pass for tensors of the current device: no call below reaches the library."""
    stage_ops = pytest.importorskip("paper_2607_13332_b200.stage_ops")
    monkeypatch.setattr(stage_ops, "_current_device", lambda: -1)
    monkeypatch.setattr(stage_ops, "_new", lambda shape, strides, dtype: torch.empty_strided(shape, strides, dtype=dtype))
    return stage_ops


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_gradient_lies_as_its_logits_do(host, monkeypatch, dtype):
    """Wherever the logits start, so that the kernel stores whole pieces."""
    monkeypatch.setattr(host, "_distill", lambda *args: None)
    buf = torch.zeros(4000, dtype=dtype)
    for logits in [buf[1:].view(31, 129)[i:] for i in range(9)] + [buf[i:i + 800].view(8, 100)[:, j:j + 90] for i in range(8) for j in (0, 3)] + [buf[5:105].view(1, 100)]:
        dlogits = host.distill_loss_grad(logits, None, None)[1]
        assert dlogits.shape == logits.shape and dlogits.stride(1) == 1
        assert all((dlogits[t].data_ptr() - logits[t].data_ptr()) % 16 == 0 for t in range(len(logits)))
        assert dlogits.untyped_storage().nbytes() <= len(logits) * (logits.shape[1] * dtype.itemsize + 16) + 16


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab", [1, 7, 96, 101])
def test_a_gradient_takes_no_more_room_than_its_rows(host, monkeypatch, dtype, vocab):
    monkeypatch.setattr(host, "_distill", lambda *args: None)
    whole = torch.zeros(5, 64, vocab, dtype=dtype)
    piece = 16 // dtype.itemsize
    for logits in (whole[:, -1], whole.flatten(0, 1)[::9], whole.flatten(0, 1), whole[:1, 3], torch.zeros(6, vocab + 13, dtype=dtype)[:, :vocab],
                   torch.zeros(6, 2, vocab, dtype=dtype)[:, 0], whole[:0, 0]):
        dlogits = host.distill_loss_grad(logits, None, None)[1]
        n, pitch = len(logits), dlogits.stride(0)
        assert dlogits.shape == logits.shape and dlogits.dtype == dtype and dlogits.stride(1) == 1
        assert vocab <= pitch < vocab + piece
        assert dlogits.untyped_storage().nbytes() <= n * (vocab + piece) * dtype.itemsize
        if n > 1:      # whole 16-byte pieces of the one are whole pieces of the other
            assert (logits.stride(0) - pitch) % piece == 0


def test_calls_without_a_status_word_share_the_librarys(host, monkeypatch):
    """What goes wrong on the device is on record whether it was asked for or not."""
    seen = []
    for name in ("_loss", "_matmul"):
        monkeypatch.setattr(host, name + "_args", lambda *args: args)
        monkeypatch.setattr(host, name, lambda args: seen.append(args[-2]) and 0)
    monkeypatch.setattr(host, "_raw_stream", lambda device: 0)
    monkeypatch.setattr(host, "_words", {-1: 0x7000})
    own = torch.zeros(1, dtype=torch.int32)
    x, s = torch.zeros(3, 16, dtype=torch.int8), torch.zeros(3)
    logits, ids, top = torch.zeros(3, 8), torch.zeros(3, 2, dtype=torch.int32), torch.zeros(3, 2)
    for word, want in ((None, 0x7000), (own, own.data_ptr())):
        del seen[:]
        host.int8_matmul(x, s, x, s, dev_status=word)
        host.distill_loss(logits, ids, top, dev_status=word)
        host.distill_loss_grad(logits, ids, top, dev_status=word)
        assert seen == [want] * 3


def test_without_the_private_names_of_torch(host, monkeypatch):
    """Another version of torch may not have them: the public ones do the same."""
    import importlib.util
    for name in ("_cuda_getDevice", "_cuda_getCurrentRawStream"):
        monkeypatch.delattr(torch._C, name)
    monkeypatch.delattr(torch._C._dynamo.guards, "_empty_strided_cuda")
    spec = importlib.util.spec_from_file_location("paper_2607_13332_b200.stage_ops_again", host.__file__)
    again = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(again)
    assert again._current_device is torch.cuda.current_device
    made = []
    monkeypatch.setattr(torch, "empty_strided", lambda *args, **kw: made.append((args, kw)))
    again._new((3, 8), (9, 1), torch.int8)
    assert made == [(((3, 8), (9, 1)), {"dtype": torch.int8, "device": "cuda"})]
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device: type("Stream", (), {"cuda_stream": 77 + device}))
    assert again._raw_stream(1) == 78


def test_without_a_gpu_there_is_no_status_word(libssn):
    if torch.cuda.is_available():
        pytest.skip("there is one here")
    assert libssn.library().stage_status_word() is None
