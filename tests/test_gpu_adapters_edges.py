"""Adapters at the edges of what a call is given: scales that no row uses, gradients of no rows."""
import pytest

pytestmark = pytest.mark.gpu


def test_scale_of_an_adapter_without_rows_is_not_used():
    import torch
    import paper_2405_13954_amd as P
    g = torch.Generator().manual_seed(1)
    x, dy = torch.randn(40, 16, generator=g).cuda(), torch.randn(40, 24, generator=g).cuda()
    a, b, u = torch.randn(4, 3, 16, generator=g).cuda(), torch.randn(4, 3, 24, generator=g).cuda(), torch.randn(40, 3, generator=g).cuda()
    ids = torch.randint(0, 2, (40,), generator=g, dtype=torch.int32).cuda()
    plan = P.logra_adapter_plan(ids, 4)
    scale = torch.tensor([0.5, 2.0, float("nan"), float("inf")], device="cuda")
    da, db = torch.full_like(a, 7.0), torch.full_like(b, 7.0)
    P.logra_adapter_backward(x, dy, a, b, plan, u, da, db, scale=scale)
    assert bool((da[2:] == 0).all()) and bool((db[2:] == 0).all())
    assert bool(torch.isfinite(da).all()) and bool(torch.isfinite(db).all())
    first = [da.clone(), db.clone()]
    da.fill_(7.0), db.fill_(7.0)
    P.logra_adapter_backward(x, dy, a, b, plan, u, da, db, scale=scale, accumulate=True)
    assert bool((da[2:] == 7).all()) and bool((db[2:] == 7).all())
    assert torch.allclose(da[:2], first[0][:2] + 7) and torch.allclose(db[:2], first[1][:2] + 7)


def test_no_rows_clear_gradients_of_any_size():
    # 1,023 adapters of rank 128 at 131,328 columns: 69 GB of dA, more 16-byte stores than one grid axis holds threads
    import torch
    import paper_2405_13954_amd as P
    n, rank, n_in = 1023, 128, 131328
    torch.cuda.empty_cache()
    da = torch.empty(n * rank * n_in + 1024, device="cuda").fill_(5.0)
    db = torch.ones(n * rank * 8, device="cuda")
    P._check(P.lib().logra_adapter_backward(None, n_in, None, 8, P.F32, 0, n_in, 8, rank, n, None, 0, None, None, None, None,
                                            None, 0, None, 0, da.data_ptr(), db.data_ptr(), 0, 0.0, 0, 0, None, 0,
                                            torch.cuda.current_stream().cuda_stream))
    assert bool((da[-1024:] == 5.0).all()), "a store behind dA"
    for at in range(0, n * rank * n_in, 1 << 30):
        assert not bool(da[at:min(at + (1 << 30), n * rank * n_in)].any())
    assert not bool(db.any())
    del da
    torch.cuda.empty_cache()
