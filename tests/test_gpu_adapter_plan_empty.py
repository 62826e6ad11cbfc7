"""A step that no request has rows in, planned on a plan that the step before filled."""
import pytest

torch = pytest.importorskip("torch")
import paper_2306_03078_amd.block_binding as K  # noqa: E402

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(300)]


def test_a_plan_of_no_requests():
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    plan = K.SpQRAdapterPlan(130, 3)
    K.spqr_adapter_plan(plan, ints([0, 2]), ints([0, 100, 130]))
    assert plan.count.item() == 3
    K.spqr_adapter_plan(plan, ints([]), ints([0]))
    assert plan.count.item() == 0 and (plan.row == -1).all() and (plan.tile == ints([-1, 0])).all()
    bank = K.SpQRAdapters([torch.ones(3, 4, 64, dtype=torch.float16, device="cuda")], [torch.ones(3, 32, 4, dtype=torch.float16, device="cuda")], rows=130)
    out = torch.full((130, 32), 5.0, device="cuda")
    K.spqr_adapters(bank, plan, torch.ones(130, 64, dtype=torch.float16, device="cuda"), [out], [out])
    assert (out == 5.0).all()


def test_a_plan_of_requests_without_rows():
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    plan = K.spqr_adapter_plan(K.SpQRAdapterPlan(70, 2), ints([1] * 70))
    assert plan.count.item() == 2
    K.spqr_adapter_plan(plan, ints([0, 1, -1]), ints([0, 0, 0, 0]))
    assert plan.count.item() == 0 and (plan.row == -1).all() and (plan.tile == ints([-1, 0])).all()
