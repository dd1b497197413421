"""Where the recovery calls run: host memory never reaches a kernel, and a call goes to the device of its tensors."""
import contextlib

import pytest
import torch


@pytest.fixture(scope="module")
def P():
    import paper_2508_02322_b200 as pkg
    return pkg


def block(P, d=64, f=16):
    w = torch.zeros(f, d, dtype=torch.bfloat16)
    return P.Ffn(w, w, torch.zeros(d, f, dtype=torch.bfloat16))


def test_a_block_on_the_host_is_refused(P):
    ffn = block(P)                                            # sizes may be asked for
    assert P.camera_ffn_workspace_bytes(ffn, 4) > 0 and P.camera_ffn_saved_bytes(ffn, 4) > 0
    x = torch.zeros(4, 64, dtype=torch.bfloat16)
    ws = P.alloc_workspace(P.camera_ffn_workspace_bytes(ffn, 4, backward=True), "cpu")
    saved = P.alloc_workspace(P.camera_ffn_saved_bytes(ffn, 4), "cpu")
    with pytest.raises(ValueError):
        P.camera_ffn_forward(ffn, x, workspace=ws)
    with pytest.raises(ValueError):
        P.camera_ffn_backward(ffn, x, x, saved, workspace=ws)
    with pytest.raises(ValueError):
        P.camera_token_logprobs(torch.zeros(4, 10))


def test_buffers_are_checked(P):
    from paper_2508_02322_b200 import recovery
    ffn = block(P)
    n = P.camera_ffn_saved_bytes(ffn, 4)
    with pytest.raises(ValueError):
        recovery._saved(torch.zeros(1, dtype=torch.uint8).expand(n), ffn, 4)      # one byte of memory
    with pytest.raises(ValueError):
        recovery._workspace(torch.zeros(1, dtype=torch.uint8).expand(1 << 20), ffn, 4, False)
    ffn.device = torch.device("cuda", 0)
    with pytest.raises(ValueError):
        recovery._workspace(torch.zeros(1 << 20, dtype=torch.uint8), ffn, 4, False)
    with pytest.raises(ValueError):
        recovery._saved(torch.zeros(n, dtype=torch.uint8), ffn, 4)


class OnDevice:
    def __init__(self, index):
        self.index = index

    def get_device(self):
        return self.index


def test_calls_go_to_the_tensors_device(P, monkeypatch):
    from paper_2508_02322_b200 import recovery
    current = [0]

    @contextlib.contextmanager
    def device(index):
        before, current[0] = current[0], index
        yield
        current[0] = before

    monkeypatch.setattr(recovery, "_current_device", lambda: current[0])
    monkeypatch.setattr(recovery, "_raw_stream", lambda index: 100 + index)
    monkeypatch.setattr(torch.cuda, "device", device)
    seen = []

    def call(*args):
        seen.append((current[0],) + args)
        return 0

    recovery._enqueue(call, OnDevice(0), "a")
    recovery._enqueue(call, OnDevice(1), "b")
    assert seen == [(0, "a", 100), (1, "b", 101)] and current[0] == 0

    def camera_refused(*args):
        return -1
    with pytest.raises(P.CameraError, match="camera_refused"):
        recovery._enqueue(camera_refused, OnDevice(1))
    assert current[0] == 0


def test_the_gradients_room_follows_the_vocabulary_not_the_pitch(P):
    from paper_2508_02322_b200 import recovery
    z = torch.zeros(4, 50, 1000, dtype=torch.bfloat16)[:, -1]             # the last position of every sequence
    g, ld = recovery._gradient(z, None, z.stride(0))
    assert g.shape == z.shape and g.stride() == (ld, 1)
    assert g.untyped_storage().nbytes() <= 2 * 4 * 1008
    for vocab, pitch, dtype in ((1000, 1003, torch.bfloat16), (1001, 1001, torch.bfloat16), (999, 7777, torch.float32), (8, 8, torch.float32)):
        z = torch.zeros(3, pitch, dtype=dtype)[:, :vocab]
        g, ld = recovery._gradient(z, None, pitch)
        per = 16 // z.element_size()
        assert vocab <= ld < vocab + per and (ld - pitch) % per == 0     # rows aligned like those of the logits
