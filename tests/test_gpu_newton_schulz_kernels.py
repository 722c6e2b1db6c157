"""Each kernel of the updates by Newton-Schulz products against the same iteration in 64 bits on the GPU: A, its polynomial and the step from either side, in tiles of 256, 192, 128 (one and two
workgroups on a compute unit) and 64, whole and in slices of the contraction, the iterate held as one number and as two; at sizes whose tiles and slabs end anywhere.

Bounds: of the result's norm 3e-3, as derived in test_gpu_newton_schulz_spectra.py, and of every row's and column's four times that (roundings are of the same size all over, a single element
that is missing or another's is a few hundredths of its row); bf16 half a step more."""
import pytest

import test_gpu_newton_schulz as common

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
ah = common.ah

U32, BF16, MOST = 2.0 ** -24, 2.0 ** -8, 3e-3
A, B, C = 3.4445, -4.7750, 2.0315

# rows, cols; of A, the polynomial and the step: the tile (128 alone: negative) and whether some tiles are cut into slices
SIZES = [
    (2051, 1003, (-128, 0), (64, 0), (-128, 0)), (16401, 131, (-128, 1), (64, 0), (128, 0)), (3101, 2899, (192, 0), (192, 0), (256, 0)), (16003, 1299, (192, 1), (64, 0), (192, 0)),
    (5301, 4999, (256, 0), (256, 0), (192, 0)), (7003, 2901, (256, 1), (192, 0), (192, 1)), (1501, 1507, (-128, 0), (-128, 0), (-128, 0)), (1003, 5003, (-128, 1), (64, 0), (192, 0)),
    (2899, 2905, (192, 0), (192, 0), (192, 0)), (1301, 16005, (192, 1), (64, 0), (192, 0)), (4999, 5005, (256, 0), (256, 0), (192, 0)), (2901, 7003, (256, 1), (192, 0), (192, 1)),
    (4301, 4307, (192, 1), (192, 1), (192, 1)), (8190, 8195, (256, 1), (256, 1), (256, 1)), (16403, 1003, (-128, 1), (64, 0), (256, 1)), (131, 16403, (64, 1), (64, 0), (128, 0)),
    (131, 50003, (64, 1), (64, 0), (256, 0)), (50003, 131, (-128, 1), (64, 0), (256, 0)), (4096, 4096, (192, 0), (192, 0), (256, 0)), (2048, 2048, (-128, 0), (-128, 0), (-128, 0)),
    (8192, 2048, (-128, 0), (-128, 0), (256, 0)), (257, 300, (64, 0), (64, 0), (64, 0)),
    (143, 132, (64, 0), (64, 0), (64, 0)), (1757, 132, (64, 1), (64, 0), (64, 0)),
    # the iterate as two numbers
    (32779, 3, (-128, 1), (64, 0), (128, 0)), (40001, 100, (-128, 1), (64, 0), (128, 0)), (65536, 128, (-128, 1), (64, 0), (128, 0)), (16403, 67, (-128, 1), (64, 0), (-128, 0)),
    (67, 16403, (64, 1), (64, 0), (-128, 0)), (3, 32779, (64, 1), (64, 0), (128, 0)), (100, 40001, (64, 1), (64, 0), (128, 0)), (128, 65535, (64, 1), (64, 0), (128, 0)), (600, 1, (64, 1), (64, 0), (64, 0)),
    (1, 1, (64, 0), (64, 0), (64, 0)), (121, 127, (64, 0), (64, 0), (64, 0)), (130, 65, (64, 0), (64, 0), (64, 0)),
]


def check_plan(ah, m, n, wanted):
    got = [ah.adahop_debug_newton_schulz_plan(m, n, i) for i in range(3)]
    assert [(-t if alone else t, int(slices > 1)) for t, alone, slices in got] == list(wanted), f"other kernels than this test is of: {got}"


def matrix(m, n):
    gen = torch.Generator(device="cuda").manual_seed(3 * m + n)
    r = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    return r(m, n).addmm_(r(m, 4), r(4, n), alpha=2.0)


def exact(u, steps):
    x = u / (torch.linalg.vector_norm(u) + 1e-7)
    for _ in range(steps):
        g = x @ x.t().contiguous() if x.shape[0] <= x.shape[1] else x.t().contiguous() @ x
        p = B * g + C * (g @ g)
        x = A * x + (p @ x if x.shape[0] <= x.shape[1] else x @ p)
    return x


def check(got, want, more=0.0):
    off, size = (got.double() - want), torch.linalg.vector_norm(want).item()
    assert torch.linalg.vector_norm(off).item() <= (MOST + more) * size, torch.linalg.vector_norm(off).item() / size
    for d, number in ((1, want.shape[0]), (0, want.shape[1])):
        over = off.norm(dim=d) / want.norm(dim=d).clamp(min=size / number ** 0.5)
        assert over.max().item() <= 4 * (MOST + more), (d, over.argmax().item(), over.max().item())


@pytest.mark.parametrize("m,n,gram,poly,step", SIZES)
def test_against_64_bits(ah, m, n, gram, poly, step):
    check_plan(ah, m, n, (gram, poly, step))
    g = matrix(m, n)
    for steps, dtype, pad in ((5, torch.float32, 3), (2, torch.bfloat16, 0)):
        common.say("orthogonalize kernels", m, n, steps)
        room = torch.full((m + 1, n + pad), 7.0, dtype=dtype, device="cuda")
        want = exact(g.double(), steps)
        space = torch.full((ah.lib().adahop_newton_schulz_workspace_bytes(m, n),), 255, dtype=torch.uint8, device="cuda")  # NaN wherever nothing has been written
        out = ah.adahop_orthogonalize(g, out=room[:m, :n], steps=steps, workspace=space)
        check(out, want, 0.0 if dtype == torch.float32 else BF16)
        for _ in range(3):
            assert torch.equal(out, ah.adahop_orthogonalize(g, dtype=dtype, steps=steps)), "other bits in another call"
        assert bool((room[m:] == 7).all()) and bool((room[:, n:] == 7).all())
    common.say("update kernels", m, n)
    w, mom = torch.randn(m, n, device="cuda").mul_(0.02), matrix(n, m).t().contiguous()
    was, u = w.double(), g.double() + 0.95 * (0.95 * mom.double() + g.double())
    copy = torch.empty(m, n, dtype=torch.bfloat16, device="cuda")
    want = exact(u, 2)
    ah.adahop_muon_update(w, g, mom, 1.0, weight_decay=0.1, scale=1.0, steps=2, w_bf16=copy, workspace=space)
    assert torch.equal(copy, w.to(torch.bfloat16))
    moved = 0.9 * was - w.double()
    # the step out of a weight that is rounded to fp32 (0.9 to 2^-25, two products and their difference to 2^-24 each)
    lost = 4 * U32 * torch.linalg.vector_norm(was).item() / torch.linalg.vector_norm(want).item()
    check(moved, want, lost + 4 * U32)
