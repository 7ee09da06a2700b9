"""The binding of the paged calls: what is not plain goes the way of Python, with the same results."""
import pytest
import torch

import paper_2503_02236_amd as vq
from test_paged import Case

gpu = pytest.mark.gpu


@gpu
def test_paged_calls_under_a_mode_are_left_to_python(gpu_device):
    """A mode that intercepts calls sees what Python does with the tensors; subclasses of tensors, caches and plans likewise."""
    from paper_2503_02236_amd import binding
    from torch.overrides import TorchFunctionMode
    vq.lib()                       # (which loads the native part)
    native = binding._marshal
    assert native is not None, "the native part of the binding is not built"
    case = Case([(40, 3), (20, 1)], seed=1)
    kv, q, table, cu, seq, _ = case.dev(gpu_device)
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device=gpu_device)  # noqa: E731
    slots = i32([3, -1, 70, 9])

    class Mode(TorchFunctionMode):
        seen = 0

        def __torch_function__(self, func, types, args=(), kwargs=None):
            Mode.seen += 1
            return func(*args, **(kwargs or {}))

    class Sub(torch.Tensor):
        pass

    class SubCache(vq.VQKVPagesDev):
        pass

    class SubPlan(vq.VQPagePlan):
        pass

    def step(plan):
        return (i32([5, -1]), i32([3, 40]), i32([[5, -1, -1], [1, 2, 3]]), i32([0, 4, -9, -9, -9, -9]), i32([2]), 16, plan, None)

    plan = vq.VQPagePlan(2, 30, gpu_device)
    calls = [(native.attn_paged, (kv, q, 0.1, table, cu, seq, None, None, 0, 0.0, None, None)), (native.kv_quantize_paged, (kv, q, q, slots)),
             (native.kv_pages_assign, step(plan))]
    for call, args in calls:
        assert call(*args) is not NotImplemented
        with Mode():
            assert call(*args) is NotImplemented, call
    want = vq.vq_attn_paged(kv, q, 0.1, table, cu, seq)
    for public, args in ((vq.vq_attn_paged, (kv, q, 0.1, table, cu, seq)), (vq.vq_kv_quantize_paged, (kv, q, q, slots)), (vq.vq_kv_pages_assign, step(plan)[:6] + (None, plan))):
        Mode.seen = 0
        with Mode():
            public(*args)
        assert Mode.seen > 0, public
    sub = SubCache(**{f: getattr(kv, f) for f in kv.__dataclass_fields__})
    assert native.attn_paged(sub, *calls[0][1][1:]) is NotImplemented and native.kv_quantize_paged(sub, q, q, slots) is NotImplemented
    assert native.attn_paged(kv, q.as_subclass(Sub), *calls[0][1][2:]) is NotImplemented
    assert native.kv_pages_assign(*step(SubPlan(2, 30, gpu_device))) is NotImplemented
    torch.cuda.synchronize()
    assert torch.equal(vq.vq_attn_paged(sub, q, 0.1, table, cu, seq), vq.vq_attn_paged(kv, q, 0.1, table, cu, seq)) and want.shape == q.shape
