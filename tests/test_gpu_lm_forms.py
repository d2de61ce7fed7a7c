"""The language-model operators' kernels for large inputs, each at the smallest sizes that reach it, against the 64-bit
references (needs an MI355X)."""
import pytest

import lm_reference as ref
from test_gpu_lm import DEV, IDS, TYPES, check_xent, inputs, logits, run_and_check

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
gs = pytest.importorskip("paper_2108_06004_amd")
from paper_2108_06004_amd import lm  # noqa: E402


# Time unsplit, several blocks a workgroup. Strips of all sequences decide the groups: 140 give sixteen forward (blocks of 128
# steps) and eight backward (64), 300 eight and eight, 330 and more eight and four (32). Rows of 64 channels fill their
# 128-byte lines, rows of 34 and 130 do not; 130 channels of 16 bits go two to a lane. No number of sequences is a multiple
# of the eight XCDs.
@pytest.mark.parametrize("B,T,C", [(140, 420, 64), (140, 420, 34), (300, 150, 64), (300, 150, 34), (330, 150, 64),
                                   (330, 150, 34), (170, 150, 130)])
@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
def test_recurrence_of_many_sequences(B, T, C, dtype):
    lengths = torch.tensor([T - (37 * b) % (T // 2) for b in range(B)], dtype=torch.int32, device=DEV)
    lengths[B // 2] = 0
    lengths[1], lengths[B - 1] = 128, 1
    i = inputs(B + C, B, T, C, dtype, gate=C != 130, packed=C == 34)
    run_and_check(i, lengths, "ragged")
    whole = {k: v[:, :T - 22].contiguous() if v is not None and v.dim() == 3 else v for k, v in i.items()}
    run_and_check(whole, what="whole")


# (2,048, 4,096] pieces of 16 bytes: 512 threads; (8,192, 16,384] and more rows than are split: 1,024 threads of sixteen
# pieces, through the caches or, rows of whole 128-byte lines, past them; more pieces: split, first read past the caches
# from 65 rows on; from 257 rows on the divisor shares the scratch with the parts
@pytest.mark.parametrize("N,V", [(5, 30_000), (65, 70_001), (65, 70_016), (65, 131_201)])
@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
def test_cross_entropy_of_long_rows(N, V, dtype):
    V = V // 2 if dtype == torch.float32 else V
    z, t = logits(N + V, N, V, dtype)
    t[::7] = -100
    grad = check_xent(z, t, what=f"{N}x{V}")
    out = torch.full((N, V + 1), 9.0, dtype=dtype, device=DEV)  # rows of another alignment than the logits'
    lm.cross_entropy_forward(z, t, grad=out[:, 1:])
    assert torch.equal(out[:, 1:], grad) and (out[:, 0] == 9.0).all()


def test_cross_entropy_of_many_split_rows():
    z, t = logits(5, 260, 65_601, torch.float32)
    t[::3] = -100
    check_xent(z, t, what="260 split rows")


def test_forms_are_the_ones_named():
    # the rules are the library's own: scratch is needed exactly where time or rows are split
    lib = gs.load_library()
    for B, T, C in ((140, 420, 64), (140, 420, 34), (300, 150, 64), (330, 150, 34), (170, 150, 130)):
        for dtype in (gs.GS_F32, gs.GS_BF16, gs.GS_F16):
            assert lib.gs_recurrence_work(B, T, C, dtype) == 0
    assert lib.gs_cross_entropy_work(65, 70_001, gs.GS_BF16) == lib.gs_cross_entropy_work(65, 35_008, gs.GS_F32) == 0
    assert lib.gs_cross_entropy_work(65, 131_201, gs.GS_BF16) > 0 and lib.gs_cross_entropy_work(260, 65_601, gs.GS_F32) > 0
