"""The block norm where a workgroup has several rows: the next row on its way while one is summed, gates that change between rows, the sums' two buffers in
turn, in every combination of types and with every kernel by width."""
import pytest

import test_gpu_training_ops as small

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
ah = small.ah


def rows_at_a_time(cols):
    """Workgroups of the forward pass: 2048 threads for each of 256 compute units."""
    threads = min(1024, -(-(-(-cols // 8)) // 64) * 64)
    return 256 * (2048 // threads)


FORWARD = [  # rows, columns, gate, x and s in fp32, y and h in fp32, columns that the rows have beyond
    (1100, 8192, None, False, False, 0), (1100, 8192, "vector", True, False, 0), (1100, 8192, 700, True, True, 0), (1100, 8192, 1, False, True, 0),
    (600, 8200, "vector", False, False, 0), (1100, 8200, 3, True, False, 1), (600, 16384, 1, True, True, 0), (600, 8200, 250, False, True, 3),
    (2100, 4091, None, True, True, 3), (2100, 4091, 3, False, False, 0), (2100, 4091, 700, False, True, 0), (1100, 4091, 1, True, False, 1),
    (2300, 2048, 3, False, False, 0), (9000, 64, 700, True, False, 0), (9000, 100, 1, False, False, 0),
]


@pytest.mark.parametrize("rows,cols,gate,s32,y32,pad", FORWARD)
def test_forward(ah, rows, cols, gate, s32, y32, pad):
    assert rows > rows_at_a_time(cols)
    small.test_block_norm(ah, rows, cols, gate, s32, y32, pad)
    # in the residual stream's own place: rows ahead are read before this one is written
    v, rows_per, _ = small.norm_inputs(rows, cols, gate, rows + cols)
    x, y = small.up(v["x"], s32, pad), small.up(v["y"], y32, pad)
    more = dict(w_post=small.up(v["w_post"]), w_pre=small.up(v["w_pre"], True), gate=small.up(v["gate"], y32), gate_rows=rows_per, keep="ckpt8")
    want = ah.adahop_block_norm(x, y, **more)
    got = ah.adahop_block_norm(x, y, s=x, **more)
    assert torch.equal(x, want["s"])
    for name in ("h", "rstd_post", "rstd_pre"):
        assert torch.equal(got[name], want[name]), name
    for name in ("ckpt_y", "ckpt_s"):
        assert all(torch.equal(a, b) for a, b in zip(got[name], want[name])), name


BACKWARD = [  # rows, columns, gate, from checkpoints, stream in fp32, block's side in fp32, columns beyond
    (777, 4091, 1, False, True, False, 0), (777, 4091, 1, True, False, False, 0), (777, 4091, "vector", True, True, False, 3), (777, 4091, 3, False, False, True, 1),
    (777, 4091, None, False, True, True, 0), (1100, 4091, 2, True, True, True, 0),
    (1100, 8192, "vector", True, False, False, 0), (1100, 8192, "vector", True, True, False, 0), (1100, 8192, "vector", False, True, False, 0),
    (1100, 8192, None, False, False, False, 0), (1100, 8192, 1, True, False, False, 0), (1100, 8192, 2, False, False, True, 0), (1100, 8192, 3, True, True, True, 0),
    (1100, 8192, 1, False, True, True, 0), (1100, 8192, 700, True, False, True, 0),
    (1300, 4096, "vector", False, True, True, 0), (1300, 4096, 1, True, True, False, 0),
    (2100, 1032, 1, False, True, False, 0), (2100, 1031, 3, True, True, False, 1), (2100, 1024, "vector", False, False, True, 0), (2100, 1024, 1, True, True, True, 0),
    (2100, 1024, 700, False, True, True, 0), (5000, 100, 1, False, True, False, 3), (2405, 2048, None, True, True, False, 0),
    (600, 8200, 1, False, True, False, 0), (600, 16384, "vector", False, True, True, 0), (600, 8200, 3, True, False, True, 1), (600, 8264, 250, False, False, True, 0),
]


@pytest.mark.parametrize("rows,cols,gate,kept,s32,y32,pad", BACKWARD)
def test_backward(ah, rows, cols, gate, kept, s32, y32, pad):
    """(In place too, and twice for the same bits.)"""
    small.test_block_norm_backward(ah, rows, cols, gate, kept, s32, y32, pad)
