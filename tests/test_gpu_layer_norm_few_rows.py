"""GPU: backward calls of a few rows: the row gradients have the same bits whether the parameters' gradients are asked for (then one
workgroup may have all rows) or not, and the parameters' gradients are those of the formula."""
import pytest
import torch

import norm_util as M

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("C", [5, 64, 77, 256, 1024, 1537, 2048, 4099, 8192, 16384])
def test_with_and_without_parameter_gradients(C, dtype):
    from paper_1810_01993_amd import api
    g = torch.Generator(device="cuda").manual_seed(C)
    gamma, beta = 1 + 0.3 * torch.randn(C, generator=g, device="cuda"), torch.zeros(C, device="cuda")
    d = api.DropoutDesc(0.25, 3)
    for n in (1, 2, 3, 4, 5, 8, 16, 17, 64, 65):
        print(f"[case] few rows n={n} C={C} {dtype}", flush=True)
        x, dy, ds = (torch.randn((n, C), generator=g, device="cuda").to(M.DT[dtype]) for _ in range(3))
        _, m, r = api.layer_norm_fwd(x, gamma, beta)
        dx, dg, db = api.layer_norm_bwd(dy, x, gamma, m, r)
        M.check_backward(dy, x, gamma, m, r, dx, dg, db, dtype)
        assert torch.equal(dx, api.layer_norm_bwd(dy, x, gamma, m, r, want_params=False)[0])
        dres, dx, dg2, db2 = api.dropout_add_layer_norm_bwd(dy, ds, x, d, gamma, m, r)
        assert torch.equal(dg, dg2) and torch.equal(db, db2)
        alone = api.dropout_add_layer_norm_bwd(dy, ds, x, d, gamma, m, r, want_params=False)
        assert torch.equal(dres, alone[0]) and torch.equal(dx, alone[1])
