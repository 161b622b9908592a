"""GPU: dgamma and dbeta to the bit.  With mean 0, rstd 1 and small whole numbers in s and dy every product and every partial sum is a
whole number below 2^24, which fp32 holds exactly in whatever order it is added: a row left out, or taken twice, shows."""
import pytest
import torch

import norm_util as M

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def api():
    from paper_1810_01993_amd import api as _api
    assert torch.cuda.is_available()
    return _api


# Per channel count the rows that a workgroup has side by side, and the workgroups there are at most (16-bit types; fp32 has other
# borders, which the channel counts twice as large fall on): rows on either side of one row, of the borders between workgroups, of
# four turns of one workgroup, of one turn of all of them and of two.
BORDERS = {3: (64, 768), 8: (256, 768), 16: (128, 768), 33: (32, 768), 64: (32, 768), 77: (16, 768), 128: (16, 768), 256: (16, 256),
           304: (16, 256), 512: (8, 256), 771: (8, 256), 1024: (4, 256), 1025: (4, 256), 1544: (1, 512), 2048: (1, 512), 2057: (1, 512),
           4104: (1, 256), 8192: (1, 256), 12295: (1, 256)}
ROWS = {C: sorted({k for b in (1, per, 4 * per, 5 * per, per * most, 2 * per * most) for k in (b - 1, b, b + 1) if 0 < k * C < 1 << 26})
        for C, (per, most) in BORDERS.items()}
# beyond the registers: slabs of 64 rows, 512 of them at most
ROWS[20001] = [1, 63, 64, 65, 127, 129, 700]
MANY = [(20011, 8), (30011, 24), (100003, 3), (25013, 40), (65537, 64), (20001, 128), (9001, 304), (40007, 256), (3001, 1024),
        (1025, 2048), (2051, 771), (600, 4104), (300, 8192), (77, 20000), (300001, 16), (110592, 304), (208297, 77), (33000, 16400)]


def _check(api, n, C, dtype, joined):
    print(f"[case] parameter gradients n={n} C={C} {dtype} joined={joined}", flush=True)
    g = torch.Generator(device="cuda").manual_seed(n + C)
    s, dy = (torch.randint(-3, 4, (n, C), generator=g, device="cuda", dtype=torch.int8) for _ in range(2))
    dy[-1] = 3                                          # the last row shows in every channel
    want_g, want_b = torch.zeros(C, dtype=torch.int64, device="cuda"), torch.zeros(C, dtype=torch.int64, device="cuda")
    for a in range(0, n, 1 << 14):                      # sums of an integer type stay exact
        part = slice(a, a + (1 << 14))
        want_g += (s[part].short() * dy[part].short()).sum(0, dtype=torch.int64)
        want_b += dy[part].sum(0, dtype=torch.int64)
    assert n * 9 < 1 << 24
    s, dy = s.to(M.DT[dtype]), dy.to(M.DT[dtype])
    m, r = torch.zeros(n, device="cuda"), torch.ones(n, device="cuda")
    gamma = torch.linspace(0.5, 1.5, C, device="cuda")
    if joined:
        _, _, dg, db = api.dropout_add_layer_norm_bwd(dy, dy, s, api.DropoutDesc(0.3, n), gamma, m, r)
    else:
        _, dg, db = api.layer_norm_bwd(dy, s, gamma, m, r)
    assert torch.equal(dg.double(), want_g.double()) and torch.equal(db.double(), want_b.double())


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("C", list(ROWS))
def test_either_side_of_every_border(api, C, dtype):
    for n in ROWS[C]:
        _check(api, n, C, dtype, n % 2 == 0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,C", MANY, ids=[f"{n}x{C}" for n, C in MANY])
def test_many_rows(api, n, C, dtype):
    for joined in (False, True):
        _check(api, n, C, dtype, joined)
