"""What a product leaves when a wait inside it runs out with copies and MMAs under way."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")


@pytest.mark.parametrize("m", [1, 30, 64, 65, 300])
def test_8bit_product_that_gives_up_under_way(m):
    """The MMA issuers give up after their first tile and the other roles find out: what was finished is right, the rest NaN, nothing beside it is
    touched, a report once, and the next products as if nothing had been."""
    from paper_2607_07388_b200 import binding as tfe, engine
    rng = torch.Generator(device=DEV).manual_seed(m)
    w, x = torch.randn((70_000, 1024), generator=rng, device=DEV), torch.randn((m, 1024), generator=rng, device=DEV)
    head = engine.QuantizedHead(w.bfloat16())
    want = head.logits(x.bfloat16())
    assert engine.matmul_fp8_status() == 0
    store = torch.full((m, 70_016), 5.0, dtype=want.dtype, device=DEV)
    out = store[:, 8:70_008]
    tfe.tfe_matmul_fp8_give_up(2)
    try:
        for _ in range(2):
            head.logits(x.bfloat16(), out=out)
            assert engine.matmul_fp8_status() != 0 and engine.matmul_fp8_status() == 0
    finally:
        tfe.tfe_matmul_fp8_give_up(0)
    gone = torch.isnan(out)
    assert gone.any() and bool((gone | (out == want)).all())
    assert (store[:, :8] == 5.0).all() and (store[:, 70_008:] == 5.0).all()
    for _ in range(2):
        assert torch.equal(head.logits(x.bfloat16()), want)
    assert engine.matmul_fp8_status() == 0
