"""The training operators where sums leave fp32, codes mean no number, and sizes end what can be numbered."""
import numpy as np
import pytest

import test_gpu_training_ops as small
from oracle import training as orc

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
ah = small.ah


def rest_of(cols):
    """What 1 / cols in fp32 leaves of the true quotient: the kernel adds it, and an infinite sum must not meet it."""
    over = np.float32(1) / np.float32(cols)
    return 1.0 - float(over) * cols


@pytest.mark.parametrize("cols,sign", [(64, 0), (8192, 0), (1000, -1), (4091, -1), (8200, -1), (3000, 1), (1023, 1), (12000, 1)])
@pytest.mark.parametrize("f32", [False, True])
def test_rows_with_an_infinite_sum_of_squares(ah, cols, sign, f32):
    """Whatever the width: the factor of such a row is 0, so that its finite elements count as 0 under that norm and its infinities as NaN."""
    assert np.sign(rest_of(cols)) == sign
    rng = np.random.default_rng(cols)
    rows, at, alpha = 7, cols // 3, 0.5
    x, y = rng.normal(size=(rows, cols)), rng.normal(size=(rows, cols))
    y[5] = 0
    clean_x, clean_y = small.up(x, f32), small.up(y, f32)
    clean_y[1], clean_y[2] = 0, 0                   # what rows 1 and 2 come to where their y counts as nothing
    bad_x, bad_y = small.up(x, f32), small.up(y, f32)
    bad_y[1, at], bad_y[2, at] = 3e38, float("inf")
    bad_x[3, at], bad_x[4, at] = 3e38, float("-inf")
    bad_y[5, at] = float("nan")
    more = dict(residual_scale=alpha, keep="ckpt8")
    small.say("infinite sums of squares", cols, f32)
    want = ah.adahop_block_norm(clean_x, clean_y, **more)
    got = ah.adahop_block_norm(bad_x, bad_y, **more)
    others = [c for c in range(cols) if c != at]
    for row in (0, 6):
        for name in ("s", "h", "rstd_post", "rstd_pre"):
            assert torch.equal(got[name][row], want[name][row]), name
    # y's squares pass fp32: its norm is 0, the residual alone is left
    assert float(got["rstd_post"][1]) == 0 and torch.equal(got["s"][1], want["s"][1]) and torch.equal(got["h"][1], want["h"][1])
    assert bool(torch.all(got["ckpt_y"][0][1] & 127 == 0)) and torch.equal(got["ckpt_s"][0][1], want["ckpt_s"][0][1])
    # an infinity in y: NaN in its own place, and by way of it under the second norm
    assert float(got["rstd_post"][2]) == 0 and torch.equal(got["s"][2][others], want["s"][2][others]) and bool(got["s"][2, at].isnan())
    assert bool(got["rstd_pre"][2].isnan()) and bool(got["h"][2].isnan().all())
    codes = got["ckpt_y"][0][2] & 127
    assert int(codes[at]) == 127 and bool(torch.all(codes[others] == 0)) and bool(torch.all(got["ckpt_s"][0][2] & 127 == 127))
    # s's squares pass fp32, and an infinity in s
    for row in (3, 4):
        assert float(got["rstd_post"][row]) == float(want["rstd_post"][row]) and float(got["rstd_pre"][row]) == 0
        assert torch.equal(got["s"][row][others], want["s"][row][others]) and bool(torch.all(got["h"][row][others] == 0))
        assert bool(torch.all(got["ckpt_s"][0][row][others] & 127 == 0))
    assert float(got["h"][3, at]) == 0 and bool(got["h"][4, at].isnan()) and float(got["s"][4, at]) == float("-inf")
    # NaN stays NaN
    assert all(bool(got[n][5].isnan().all()) for n in ("rstd_post", "rstd_pre", "s", "h"))


@pytest.mark.parametrize("cols", [96, 8192, 8200])
def test_weights_of_absent_parts(ah, cols):
    """The weight of a branch or of a norm that is not there takes no part, whatever it holds."""
    rows = 5
    gen = torch.Generator(device="cuda").manual_seed(cols)
    x, y, d = (torch.randn(rows, cols, generator=gen, device="cuda").to(torch.bfloat16) for _ in range(3))
    w = torch.ones(cols, device="cuda")
    bad = w.clone()
    bad[3], bad[cols - 1] = float("inf"), float("nan")
    small.say("weights of absent parts", cols)
    want, got = ah.adahop_block_norm(x, w_pre=w, residual_scale=0.5), ah.adahop_block_norm(x, w_pre=w, w_post=bad, residual_scale=0.5)
    assert torch.equal(got["s"], want["s"]) and torch.equal(got["h"], want["h"])
    want, got = ah.adahop_block_norm(x, y, pre_norm=False), ah.adahop_block_norm(x, y, w_pre=bad, pre_norm=False)
    assert torch.equal(got["s"], want["s"])
    f = ah.adahop_block_norm(x, y, keep="ckpt8")
    back = lambda w_pre: ah.adahop_block_norm_backward(d, None, None, f["ckpt_y"], None, f["rstd_post"], w_pre=w_pre)  # noqa: E731
    want, got = back(w), back(bad)
    assert torch.equal(got["d_x"], want["d_x"]) and torch.equal(got["d_y"], want["d_y"]) and bool(got["d_x"].isfinite().all())


def test_backward_without_a_branch_but_with_its_weight(ah):
    """As the forward pass takes it: the same as without, and no gradient of it."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    x, d = (torch.randn(5, 96, generator=gen, device="cuda").to(torch.bfloat16) for _ in range(2))
    w = torch.randn(96, generator=gen, device="cuda")
    f = ah.adahop_block_norm(x, w_post=w, w_pre=w, keep="stats")
    small.say("backward without a branch")
    back = lambda **more: ah.adahop_block_norm_backward(d, d, f["s"], None, f["rstd_pre"], f["rstd_post"], w_pre=w, **more)  # noqa: E731
    want, got = back(), back(w_post=w)
    assert torch.equal(got["d_x"], want["d_x"]) and torch.equal(got["d_w_pre"], want["d_w_pre"])
    assert got["d_y"] is None and got["d_w_post"] is None


def test_type_of_the_residual_streams_gradient(ah):
    """From d_h and checkpoints alone it is of d_h's type unless d_x is given; in float32 it is what bfloat16 is the rounding of."""
    gen = torch.Generator(device="cuda").manual_seed(4)
    x, y = (torch.randn(9, 200, generator=gen, device="cuda") for _ in range(2))
    d = torch.randn(9, 200, generator=gen, device="cuda").to(torch.bfloat16)
    f = ah.adahop_block_norm(x, y.to(torch.bfloat16), keep="ckpt8")
    assert f["s"].dtype == torch.float32
    small.say("type of d_x")
    back = lambda s, d_s=None, **more: ah.adahop_block_norm_backward(d_s, d, s, f["ckpt_y"] if isinstance(s, tuple) else y.to(torch.bfloat16),  # noqa: E731
                                                                     f["rstd_pre"], f["rstd_post"], **more)["d_x"]
    rounded, whole = back(f["ckpt_s"]), back(f["ckpt_s"], d_x=torch.empty_like(x))
    assert rounded.dtype == torch.bfloat16 and whole.dtype == torch.float32 and torch.equal(whole.to(torch.bfloat16), rounded)
    assert not torch.equal(whole, rounded.float())
    assert back(f["s"]).dtype == back(f["ckpt_s"], torch.zeros_like(x)).dtype == torch.float32


@pytest.mark.parametrize("tokens,d_out,d_in", [(256, 96, 160), (96, 512, 320)])
def test_unpacked_checkpoint_as_an_operand(ah, tokens, d_out, d_in):
    """The weight gradient as an MXFP4 product of the unpacked checkpoint: the bits of the product of the values that the checkpoint stands for."""
    gen = torch.Generator(device="cuda").manual_seed(tokens)
    x = torch.randn(tokens, d_in, generator=gen, device="cuda")
    G = torch.randn(tokens, d_out, generator=gen, device="cuda").to(torch.bfloat16)
    x8 = ah.adahop_ckpt8_pack(x)
    value = orc.ckpt8_unpack(*small.stored8(x8))
    bits = torch.from_numpy(value).to(torch.bfloat16)
    assert np.array_equal(bits.double().numpy(), value)                 # bfloat16 holds them all
    small.say("unpacked checkpoint as an operand", tokens, d_out, d_in)
    product = lambda v: ah.adahop_gemm(ah.Operand(G, False), ah.Operand(v, False), ah.ADAHOP_IHT, 32)["C"]  # noqa: E731
    got, want = product(ah.adahop_ckpt8_unpack(x8)), product(bits.cuda())
    assert torch.equal(got, want)
    # of the same gradient as the product in bf16, to what MXFP4 leaves (an eighth and less of either operand)
    exact = ah.adahop_ckpt8_wgrad(G, x8)
    assert ((got - exact).norm() / exact.norm()).item() < 0.25


def test_a_scale_that_is_no_number(ah):
    """E8M0's 255 is NaN: so is whatever it scales, in every reader of a checkpoint, and nothing beside it."""
    rows, cols = 40, 256
    codes = torch.arange(256, dtype=torch.uint8, device="cuda").repeat(rows, 1)
    codes[:, 127], codes[:, 255] = 0, 0             # the codes that are NaN by themselves
    scales = torch.full((rows, 8), 120, dtype=torch.uint8, device="cuda")
    clean = (codes, scales.clone())
    scales[3, 2] = 255
    there = torch.zeros(rows, cols, dtype=torch.bool, device="cuda")
    there[3, 64:96] = True
    value = codes.view(torch.float8_e4m3fn).float() * scales.view(torch.float8_e8m0fnu).float().repeat_interleave(32, dim=1)
    assert torch.equal(value.isnan(), there)        # torch's reading of the two types
    assert np.array_equal(orc.ckpt8_unpack(codes.cpu().numpy(), scales.cpu().numpy()), value.double().cpu().numpy(), equal_nan=True)
    small.say("a scale of 255")
    for dtype in (torch.float32, torch.bfloat16):
        got = ah.adahop_ckpt8_unpack((codes, scales), dtype=dtype)
        assert torch.equal(got.isnan(), there) and torch.equal(got[~there], value.to(dtype)[~there])
    G = torch.randn(rows, 64, device="cuda").to(torch.bfloat16)
    got, want = ah.adahop_ckpt8_wgrad(G, (codes, scales)), ah.adahop_ckpt8_wgrad(G, clean)
    assert torch.equal(got.isnan(), there[3].expand(64, cols)) and torch.equal(got[:, ~there[3]], want[:, ~there[3]])
    d_a = torch.randn(rows, cols, device="cuda").to(torch.bfloat16)
    got, want = ah.adahop_swiglu_backward(clean, (codes, scales), d_a), ah.adahop_swiglu_backward(clean, clean, d_a)
    assert torch.equal(got["d_g"].isnan(), there) and torch.equal(got["d_g"][~there], want["d_g"][~there]) and torch.equal(got["d_u"], want["d_u"])
    one = torch.ones(rows, device="cuda")
    back = lambda s: ah.adahop_block_norm_backward(d_a, d_a, s, clean, one, one, w_pre=d_a[0])  # noqa: E731
    got, want = back((codes, scales)), back(clean)
    rest = [r for r in range(rows) if r != 3]
    assert torch.equal(got["d_x"][rest], want["d_x"][rest]) and bool(got["d_x"][3, 64:96].isnan().all())
    assert torch.equal(got["d_w_pre"].isnan(), there[3])


def test_more_pieces_than_32_bits_number(ah):
    """Just below 2^35 elements with a nearly empty last block in every row: 2^30 blocks of 32 columns and 2 031 488 more, above 2^32 pieces of 8. 173 GB."""
    rows, cols = 2097024, 16385
    assert rows * cols < 2 ** 35 and 4 * rows * -(-cols // 32) > 2 ** 32
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 185e9:
        pytest.skip("185 GB of free memory wanted")
    gen = torch.Generator(device="cuda").manual_seed(8)
    wrap = 2 ** 30 // 513                           # the row in which block 2^30 lies
    at = torch.tensor([0, 1, 2, 1234567, wrap - 1, wrap, wrap + 1, rows - 2, rows - 1], device="cuda")
    few = torch.randn(len(at), cols, generator=gen, device="cuda").to(torch.bfloat16)

    def only_there(t):
        """Zero but in the rows `at`, which are left zero too."""
        t[at] = 0
        return not any(bool(t[a:a + 2 ** 17].any()) for a in range(0, rows, 2 ** 17))
    x, out = (torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    x[at] = few
    codes, scales = ah.adahop_ckpt8_empty(rows, cols)
    codes.fill_(0x55), scales.fill_(0x55)
    small.say("most blocks: pack", rows, cols)
    ah.adahop_ckpt8_pack(x, out=(codes, scales))
    want = ah.adahop_ckpt8_pack(few)
    assert torch.equal(codes[at], want[0]) and torch.equal(scales[at], want[1])
    assert only_there(codes) and only_there(scales)
    codes[at], scales[at] = want
    out.fill_(7.0)
    small.say("most blocks: unpack")
    ah.adahop_ckpt8_unpack((codes, scales), out=out)
    few = ah.adahop_ckpt8_unpack(want)
    assert torch.equal(out[at], few) and only_there(out)
    del codes, scales
    x[at] = few
    out.fill_(7.0)
    small.say("most blocks: gated activation")
    ah.adahop_swiglu(x, x, a=out)
    assert torch.equal(out[at], ah.adahop_swiglu(few, few)["a"]) and only_there(out)
    out[at] = few
    want = ah.adahop_swiglu_backward(few, few, few)
    small.say("most blocks: gated activation, backward")
    ah.adahop_swiglu_backward(x, x, out, d_g=x, d_u=out)       # in the place of g and of a's gradient
    assert torch.equal(x[at], want["d_g"]) and torch.equal(out[at], want["d_u"]) and only_there(x) and only_there(out)
    del x, out
    torch.cuda.empty_cache()
