"""One workspace over calls of many sizes: what the largest call asked for is not refused to a smaller one."""
import ctypes as C

import pytest
import torch


@pytest.fixture(scope="module")
def P():
    import paper_2508_02322_b200 as pkg
    return pkg


@pytest.mark.skipif(torch.cuda.is_available(), reason="the addresses below are made up: the calls must not get to launch")
@pytest.mark.parametrize("d,f,most", [(3584, 2560, 2476), (2048, 1408, 1853), (4096, 14336, 4199), (512, 2048, 700)])
def test_the_workspace_of_the_largest_call_is_large_enough(P, d, f, most):
    from paper_2508_02322_b200.binding import camera_ffn_t
    lib = P.lib

    def ffn(width):
        return C.byref(camera_ffn_t(d, width, f, 4096, 4096, 4096))

    size = {b: lib.camera_ffn_workspace_bytes(ffn(f), most, b) for b in (0, 1)}
    asked = 0
    for n in sorted(set(range(1, most + 1, 61)) | {1, 64, 65, 203, 380, most - 1, most}):
        for width in (f, f * 7 // 8, f * 6 // 7, 77):
            asked += any(lib.camera_ffn_workspace_bytes(ffn(width), n, b) > size[b] for b in (0, 1))
            assert lib.camera_ffn_forward(ffn(width), 4096, n, 4096, None, 4096, size[0], None) != -3, (n, width)
            assert lib.camera_ffn_backward(ffn(width), 4096, 4096, n, 4096, 4096, 4096, 4096, 4096, 4096, size[1], None) != -3, (n, width)
    assert asked > 0                    # the query does name more for some smaller call: the case is there
