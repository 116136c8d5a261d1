"""More of what the binding of the float-side calls refuses, and what it hands to the library (CPU: the library is replaced by one
that records calls)."""
import pytest
import torch

from test_float_calls_checks import _ran, _refused, niti            # noqa: F401  (the fixture)

BF = torch.bfloat16


def test_parts_of_the_backward_call(niti):                          # noqa: F811
    a, w, s = torch.zeros(3, 16, dtype=torch.int8), torch.zeros(5, 16, dtype=torch.int8), torch.zeros(1, dtype=torch.int32)
    d = torch.zeros(3, 5, dtype=BF)
    for x in (False, True):
        for y in (False, True):
            for b in (False, True):
                got = niti.linear_act_bwd(a, s, w, s, d, need_dx=x, need_dw=y, need_dbias=b)
                args = _ran(niti, "niti_linear_act_bwd")[-1]
                assert [g is not None for g in got] == [p is not None for p in args[8:11]] == [x, y, b]
    from paper_2009_13108_b200 import NitiError
    for kw in (dict(dx=torch.zeros(3, 16, dtype=BF), need_dx=False), dict(dw=torch.zeros(5, 16), need_dw=False), dict(dbias=torch.zeros(5), need_dbias=False)):
        with pytest.raises(NitiError):
            niti.linear_act_bwd(a, s, w, s, d, **kw)


def test_scalars_without_an_element_are_refused(niti):             # noqa: F811
    """The pointer of an empty tensor is null, which the library takes for no gradient scale at all."""
    p, g = torch.zeros(300), torch.zeros(300)
    step, none = torch.ones(1, dtype=torch.int32), torch.empty(0, dtype=torch.int32)
    plan = niti.adamw_tensors([p], [g], [p + 1], [p + 2])
    w8 = torch.zeros(300, dtype=torch.int8)
    _refused(niti, lambda: niti.adamw(plan, step, 1e-3, grad_scale=torch.empty(0)), lambda: niti.adamw(plan, none, 1e-3),
             lambda: niti.adamw_tensors([p], [g], [p + 1], [p + 2], w8=[w8], s_w=[none]))
    niti.adamw(plan, step, 1e-3, grad_scale=torch.ones(()))
    assert len(_ran(niti, "niti_adamw")) == 1


def test_weights_of_no_matrix_are_refused(niti):                    # noqa: F811
    a, s = torch.zeros(3, 16, dtype=torch.int8), torch.zeros(1, dtype=torch.int32)
    _refused(niti, lambda: niti.linear_act_fwd(a, s, torch.zeros((), dtype=torch.int8), s))


def test_parameters_that_share_memory_are_refused(niti):            # noqa: F811
    """A list that holds a parameter twice would update it twice at once."""
    p, g, w = torch.zeros(600), torch.zeros(600), torch.zeros(600, dtype=torch.int8)
    sw = torch.zeros(1, dtype=torch.int32)
    state = lambda n: [torch.zeros(n) for _ in range(2)]                                       # noqa: E731
    m, v = state(300), state(300)
    t = niti.adamw_tensors
    _refused(niti, lambda: t([p, p], [g, g], state(600), state(600)), lambda: t([p[:300], p[299:599]], [g[:300]] * 2, m, v),
             lambda: t([p[:300], p[300:]], [g[:300]] * 2, m, v, w8=[w[:300], w[100:400]], s_w=[sw, sw]))
    # neighbours in one buffer, shared gradients and empty tensors are in order
    t([p[:300], p[300:], p[:0]], [g[:300], g[:300], g[:0]], m + [p[:0]], v + [p[:0]], w8=[w[:300], w[300:], w[:0]], s_w=[sw] * 3)


def test_gradients_of_a_list_can_be_replaced(niti):                 # noqa: F811
    from paper_2009_13108_b200 import NitiError
    p, q = torch.zeros(300), torch.zeros(2, 5)
    old = [torch.zeros(300), torch.zeros(2, 5)]
    plan = niti.adamw_tensors([p, q], old, [p + 1, q + 1], [p + 2, q + 2])
    new = [torch.zeros(300, dtype=BF), torch.zeros(2, 5)]
    plan.set_grads(new)
    assert [plan.array[i].g for i in (0, 1)] == [t.data_ptr() for t in new]
    assert plan.array[0].g_type == 1 and plan.array[1].g_type == 0 and plan.tensors[1][0] is new[0]
    for bad in ([new[0]], [new[0], torch.zeros(5, 2)], [new[0], torch.zeros(2, 5, dtype=torch.int32)], [new[0], torch.zeros(5, 2).t()],
                [torch.zeros(300), torch.zeros(2, 5, device="meta")], [new[0], None]):
        with pytest.raises(NitiError):
            plan.set_grads(bad)
        assert plan.array[0].g == new[0].data_ptr() and plan.tensors[1][1] is new[1]
    niti.adamw(plan, torch.ones(1, dtype=torch.int32), 1e-3)


def test_another_current_device_is_refused(monkeypatch):
    """A default stream belongs to the current device: a call there would run on one GPU with another's memory."""
    from paper_2009_13108_b200 import Niti, NitiError
    n = Niti.__new__(Niti)
    n._gpu, n.device = 1, torch.device("cuda", 1)
    current = [0]
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: current[0], raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda d: 100 + d, raising=False)
    with pytest.raises(NitiError, match="current device"):
        n._stream()
    current[0] = 1
    assert n._stream() == 101


def test_an_allocator_that_answers_otherwise_is_not_used():
    from paper_2009_13108_b200 import api
    right = lambda shape, strides, dtype: torch.empty_strided(shape, strides, dtype=dtype)    # noqa: E731

    def fails(*args):
        raise TypeError("other arguments")

    assert api._allocates(right, -1)
    for wrong in (None, fails, lambda s, t, d: None, lambda s, t, d: right(s, t, torch.float32), lambda s, t, d: right(t, s, d),
                  lambda s, t, d: right(s, (1, s[0]), d)):
        assert not api._allocates(wrong, -1)
    assert not api._allocates(right, 0)                                # (on another device)
