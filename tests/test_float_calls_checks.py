"""What the binding of the float-side calls refuses before the library sees a pointer, and what the library is handed
(CPU: the library is replaced by one that records calls)."""
import types

import pytest
import torch


class _Library:
    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append((name, args))
            return 1 << 20 if name == "niti_workspace_bytes" else 0
        return call


@pytest.fixture()
def niti(monkeypatch):
    from paper_2009_13108_b200 import Niti
    n = Niti.__new__(Niti)
    n.lib, n.h, n._gpu, n._ws_need = _Library(), None, -1, {}          # (a CPU tensor's device number)
    n.device = torch.device("cpu")
    n._ws = n._owned_ws = torch.empty(1 << 20, dtype=torch.uint8)
    monkeypatch.setattr(Niti, "_stream", lambda self: 0)
    from paper_2009_13108_b200 import api
    monkeypatch.setattr(api, "_empty_on_current", None)
    return n


def _ran(niti, name):
    return [args for called, args in niti.lib.calls if called == name]


def _refused(niti, *calls):
    from paper_2009_13108_b200 import NitiError
    for call in calls:
        with pytest.raises(NitiError):
            call()
    assert not [c for c, _ in niti.lib.calls if c != "niti_workspace_bytes"]


F = torch.float32
BF = torch.bfloat16


def test_norm_refusals(niti):
    x, g, r = torch.zeros(4, 8, dtype=BF), torch.ones(8), torch.ones(4)
    _refused(niti, lambda: niti.rmsnorm_fwd(x.double(), g), lambda: niti.rmsnorm_fwd(x[0], g), lambda: niti.rmsnorm_fwd(x.t(), g[:4]),
             lambda: niti.rmsnorm_fwd(x, g[:4]), lambda: niti.rmsnorm_fwd(x, g.to(BF)), lambda: niti.rmsnorm_fwd(x, g, residual=x[:2]),
             lambda: niti.rmsnorm_fwd(x, g, residual=x.float()), lambda: niti.rmsnorm_fwd(x, g, h=x), lambda: niti.rmsnorm_fwd(x, g, y=x),
             lambda: niti.rmsnorm_fwd(x, g, s_y=torch.zeros(1, dtype=torch.int32)), lambda: niti.rmsnorm_fwd(x, g, rstd=torch.ones(5)),
             lambda: niti.rmsnorm_fwd(types.SimpleNamespace(dtype=BF, dim=lambda: 2, shape=(4, 8), get_device=lambda: 3, is_contiguous=lambda: True, device="cuda:3"), g),
             lambda: niti.rmsnorm_bwd(x, x[:2], g, r), lambda: niti.rmsnorm_bwd(x, x, g, r.to(BF)), lambda: niti.rmsnorm_bwd(x, x, g, r, dh=x.float()),
             lambda: niti.quantize(x[:, ::2]), lambda: niti.quantize(x.int()))


def test_dequantize_refusals(niti):
    q, s = torch.zeros(4, 8, dtype=torch.int8), torch.zeros(4, dtype=torch.int32)
    _refused(niti, lambda: niti.dequantize(q, s[:3]), lambda: niti.dequantize(q, s.float()), lambda: niti.dequantize(q.int(), s),
             lambda: niti.dequantize(q, s, dtype=torch.float64), lambda: niti.dequantize(q, s, block=0), lambda: niti.dequantize(q, s, block=16),
             lambda: niti.dequantize(q.t(), s), lambda: niti.dequantize(q, s, out=torch.zeros(8, 4)))


def test_dequantize_counts_a_short_last_block(niti):
    q = torch.zeros(1000, dtype=torch.uint8)
    niti.dequantize(q, torch.zeros(4, dtype=torch.int8), block=256)
    niti.dequantize(q.view(4, 250), torch.zeros(4, dtype=torch.int8))
    niti.dequantize(q.view(4, 250), torch.zeros(1, dtype=torch.int8))
    assert [a[-1] for a in _ran(niti, "niti_dequantize")] == [256, 250, 0]
    assert all(a[5] == 1 and a[6] == 1 for a in _ran(niti, "niti_dequantize"))          # codes, int8 exponents


def test_linear_refusals(niti):
    a, w, s = torch.zeros(3, 16, dtype=torch.int8), torch.zeros(5, 16, dtype=torch.int8), torch.zeros(1, dtype=torch.int32)
    o = torch.zeros(3, 5, dtype=BF)
    f, b = niti.linear_act_fwd, niti.linear_act_bwd
    _refused(niti, lambda: f(a.int(), s, w, s), lambda: f(a[0], s, w, s), lambda: f(a, s, w[:, :8], s), lambda: f(a, s, w.t(), s),
             lambda: f(a, s.long(), w, s), lambda: f(a, torch.zeros(2, dtype=torch.int32), w, s), lambda: f(a, s, w, torch.zeros(5, dtype=torch.int32)),
             lambda: f(a, s, w, s, bias=torch.zeros(5, dtype=BF)), lambda: f(a, s, w, s, residual=o.float()), lambda: f(a, s, w, s, act="swish"),
             lambda: f(a, s, w, s, dtype=torch.int8), lambda: f(a, s, w, s, out=o.float()), lambda: f(a, s, w, s, z=o[:2]),
             lambda: b(a, torch.zeros(3, dtype=torch.int32), w, s, o), lambda: b(a, s, w, s, o[:2]), lambda: b(a, s, w, s, o, z=o.float()),
             lambda: b(a, s, w, s, o, dw_dtype=torch.int8), lambda: b(a, s, w, s, o, dx=torch.zeros(3, 16)), lambda: b(a[:, :8], s, w, s, o),
             lambda: b(a, s, w, s, o, dbias=torch.zeros(5, dtype=BF)), lambda: b(a, s, w, s, o, act="tanh"))


def test_linear_hands_over_rows_of_exponents(niti):
    a, w, s = torch.zeros(3, 16, dtype=torch.int8), torch.zeros(5, 16, dtype=torch.int8), torch.zeros(1, dtype=torch.int32)
    niti.linear_act_fwd(a, s, w, s)
    niti.linear_act_fwd(a, torch.zeros(3, dtype=torch.int32), w, s, keep_z=True)
    one, rows = _ran(niti, "niti_linear_act_fwd")
    assert one[4] == 0 and rows[4] == 1 and one[10] is None and rows[10] is not None


def test_adamw_refusals(niti):
    p, g = torch.zeros(300), torch.zeros(300, dtype=BF)
    c, e = torch.zeros(300, dtype=torch.uint8), torch.zeros(2, dtype=torch.int8)
    w, sw = torch.zeros(300, dtype=torch.int8), torch.zeros(1, dtype=torch.int32)
    t = niti.adamw_tensors
    _refused(niti, lambda: t([p], [g], [p], [p, p]), lambda: t([p.to(BF)], [g], [p], [p]), lambda: t([p], [g.int()], [p], [p]),
             lambda: t([p], [g[:9]], [p], [p]), lambda: t([p], [g], [c], [c]), lambda: t([p], [g], [c], [c], s_m=[e]),
             lambda: t([p], [g], [c], [c], s_m=[e[:1]], s_v=[e]), lambda: t([p], [g], [p], [p], s_m=[e], s_v=[e]),
             lambda: t([p], [g], [p], [p], w8=[w]), lambda: t([p], [g], [p], [p], w8=[p], s_w=[sw]), lambda: t([p], [g], [p], [p], weight_decay=[0.1, 0.2]),
             lambda: t([p[::2]], [g[::2]], [p[::2]], [p[::2]]),
             lambda: niti.adamw(t([p], [g], [p], [p]), torch.zeros(1), 1e-3), lambda: niti.adamw(t([p], [g], [p], [p]), sw, 1e-3, grad_scale=sw))


def test_adamw_list(niti):
    import ctypes
    from paper_2009_13108_b200.api import _AdamwTensor
    assert ctypes.sizeof(_AdamwTensor) == 80                        # niti_adamw_tensor on a 64-bit host
    p, g = torch.zeros(300), torch.zeros(300, dtype=torch.float16)
    m, v, sm, sv = niti.adamw_state(p)
    assert m.dtype == torch.uint8 and sm.shape == (2,) and not m.any()
    plan = niti.adamw_tensors([p, p + 1], [g, g], [m, m], [v, v], s_m=[sm, sm], s_v=[sv, sv], weight_decay=[0.0, 0.5])
    assert len(plan) == 2 and plan.state_bits == 8 and plan.array[1].weight_decay == 0.5
    assert plan.array[0].p == p.data_ptr() and plan.array[0].g_type == 2 and plan.array[0].w8 is None and plan.array[0].n == 300
    niti.adamw(plan, torch.ones(1, dtype=torch.int32), 1e-3)
    args = _ran(niti, "niti_adamw")[0]
    assert args[3:5] == (2, 8) and args[6:10] == (1e-3, 0.9, 0.999, 1e-8) and args[10] is None


def test_workspace_queries():
    import ctypes
    from paper_2009_13108_b200 import build
    lib = ctypes.CDLL(build.build())
    lib.niti_workspace_bytes.restype = ctypes.c_size_t
    query = lambda op, *d: lib.niti_workspace_bytes(op, (ctypes.c_int64 * len(d))(*d), len(d))       # noqa: E731
    header, slabs = 256 * 1024, 160 * 128 * 256 * 4
    up = lambda v: (v + 255) // 256 * 256                                                             # noqa: E731
    assert query(8, 1000, 64) == header + up(4000) and query(8, 0, 64) == header and query(8, 5, 0) == 0 and query(8, 5) == 0
    assert query(9, 1000, 64) == header + 320 * 4 * 64
    # operands with rows that are no multiple of 16 bytes are copied
    assert query(11, 100, 50, 64) == header + slabs and query(11, 100, 50, 60) == header + slabs + up(100 * 64) + up(50 * 64)
    blocks = 25                                        # four rows each
    assert query(12, 100, 50, 64) == header + slabs + 256 + up(blocks * 50 * 4) + up(100 * 64)
    assert query(11, -1, 50, 64) == 0 and query(12, 10, 0, 64) == 0
