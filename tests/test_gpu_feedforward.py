"""The float-side calls as a transformer's feed-forward block strings them together: norm with residual into int8, up projection
with GELU, rounding, down projection onto the residual stream; backwards through the same; an AdamW step that refreshes the
int8 weights.  The calls share one workspace and are ordered by the stream alone."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
M, C, F = 260, 192, 448
S_W = -10


@pytest.fixture(scope="module")
def niti():
    from paper_2009_13108_b200 import Niti
    n = Niti(0)
    yield n
    n.close()


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


class Block:
    def __init__(self, niti, bits=8):
        self.n = niti
        r = lambda *s: torch.randn(s, device="cuda", generator=_gen(sum(s)))                  # noqa: E731
        self.x, self.res, self.dout = r(M, C).to(torch.bfloat16), r(M, C).flip(0).contiguous().to(torch.bfloat16), (1e-2 * r(M, C).flip(1).contiguous()).to(torch.bfloat16)
        self.s_w = [niti.scalar(S_W), niti.scalar(S_W)]
        # masters on the grid of the int8 weights, so that payloads stand for them exactly
        self.w8 = [torch.randint(-100, 101, s, device="cuda", generator=_gen(s[0]), dtype=torch.int32).to(torch.int8) for s in ((F, C), (C, F))]
        self.w = [w.float() * 2.0 ** S_W for w in self.w8]
        self.gain, self.bias = 1 + 0.1 * r(C), 0.1 * r(F)
        self.params = self.w + [self.gain, self.bias]
        self.grads = [torch.zeros_like(p) for p in self.params]
        states = [niti.adamw_state(p, bits) for p in self.params]
        m, v, sm, sv = zip(*states)
        self.states = [s for s in m + v + sm + sv if s is not None]
        spare = [torch.zeros_like(p, dtype=torch.int8) for p in (self.gain, self.bias)]       # (only weights are read as payloads)
        self.plan = niti.adamw_tensors(self.params, self.grads, m, v, s_m=sm if bits == 8 else None, s_v=sv if bits == 8 else None,
                                       w8=self.w8 + spare, s_w=self.s_w + [niti.scalar(-6), niti.scalar(-6)], weight_decay=[0.1, 0.1, 0.0, 0.0])
        self.step_no = torch.zeros(1, dtype=torch.int32, device="cuda")

    def step(self, between=lambda: None):
        n = self.n
        y, s_y, h, rstd = n.rmsnorm_fwd(self.x, self.gain, residual=self.res, rows=False)
        between()
        u, z = n.linear_act_fwd(y, s_y, self.w8[0], self.s_w[0], bias=self.bias, act="gelu", keep_z=True)
        between()
        q, s_q = n.quantize(u, rows=False)
        between()
        out, _ = n.linear_act_fwd(q, s_q, self.w8[1], self.s_w[1], residual=h)
        between()
        du, _, _ = n.linear_act_bwd(q, s_q, self.w8[1], self.s_w[1], self.dout, dw=self.grads[1])
        between()
        dy, _, _ = n.linear_act_bwd(y, s_y, self.w8[0], self.s_w[0], du, z=z, act="gelu", dw=self.grads[0], dbias=self.grads[3], round_mode=0)
        between()
        dx, _ = n.rmsnorm_bwd(dy, h, self.gain, rstd, dh=self.dout, dgain=self.grads[2])
        between()
        grads = [g.clone() for g in self.grads]
        self.step_no += 1
        n.adamw(self.plan, self.step_no, lr=1e-2)
        between()
        return [out, dx, y, q] + grads + [p.clone() for p in self.params] + [w.clone() for w in self.w8] + [s.clone() for s in self.states]


def _same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("bits", [8, 32])
def test_a_run_is_the_same_however_it_is_enqueued(niti, bits):
    one = Block(niti, bits)
    want = [one.step(torch.cuda.synchronize) for _ in range(3)]
    two = Block(niti, bits)
    assert all(_same(two.step(), w) for w in want)                          # back to back
    three = Block(niti, bits)                                               # with the step's headers cleared in one go
    for w in want:
        niti.begin_step()
        got = three.step()
        niti.end_step()
        assert _same(got, w)
    four = Block(niti, bits)                                                # in a graph
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        got = four.step()
    torch.cuda.current_stream().wait_stream(side)
    keep = niti.buffers()
    for w in want:
        graph.replay()
        assert _same(got, w)
    del keep
    five = Block(niti, bits)                                                # on another stream than the tensors were made on
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = [five.step() for _ in want]
    side.synchronize()
    assert all(_same(g, w) for g, w in zip(got, want))
    assert niti.check() == 0


def test_two_contexts_take_turns(niti):
    from paper_2009_13108_b200 import Niti
    other = Niti(0)
    a, b, c = Block(niti), Block(other), Block(niti)
    want = [c.step() for _ in range(2)]
    for w in want:
        assert _same(a.step(), w) and _same(b.step(), w)
    other.close()


def test_integer_calls_in_between_keep_their_results(niti):
    """The headers of the workspace change hands between integer calls and these."""
    rng = np.random.default_rng(3)
    a = torch.from_numpy(rng.integers(-127, 128, (300, 256), dtype=np.int8)).cuda()
    w = torch.from_numpy(rng.integers(-127, 128, (512, 256), dtype=np.int8)).cuda()
    s = niti.scalar(-7)
    want = niti.linear_fwd(a, s, w, s, relu=True)[0].clone()
    blk, ref = Block(niti), Block(niti)
    first = ref.step()
    for k in range(4):
        got = niti.linear_fwd(a, s, w, s, relu=True)[0]
        assert torch.equal(got, want)
        if k == 0:
            assert _same(blk.step(), first)
        else:
            blk.step()
    assert torch.equal(niti.linear_fwd(a, s, w, s, relu=True)[0], want)


def test_gradients_of_the_block(niti):
    """Against the 64-bit gradients of the block without any rounding.  An operand rounded to payloads is off by half a step an
    element at most, 0.5 / rms(payload) of its norm; the errors and activations here have payloads of 12 and more (checked), so
    each of the at most three rounded factors on the way to a gradient adds less than 0.042 to its relative error, and the
    bfloat16 tensors in between 2^-8 each."""
    blk = Block(niti)
    out, dx, y, q, dw1, dw2, dgain, dbias = blk.step()[:8]
    for payload in (y, q):
        assert payload.float().square().mean().sqrt() > 12
    X = (blk.x.float() + blk.res.float()).to(torch.bfloat16).double().requires_grad_()
    fresh = Block(niti)                                        # (the weights as they were before the step)
    W1, W2, G, B = [p.double().requires_grad_() for p in fresh.params]
    H = X
    Y = H * torch.rsqrt(H.square().mean(1, keepdim=True) + 1e-6) * G
    O = H + torch.nn.functional.gelu(Y @ W1.t() + B) @ W2.t()
    O.backward(blk.dout.double())
    rel = lambda a, b: float((a.double() - b).norm() / b.norm())                          # noqa: E731
    assert rel(out, O.detach()) < 0.1
    for got, want in ((dw1, W1.grad), (dw2, W2.grad), (dgain, G.grad), (dbias, B.grad), (dx, X.grad)):
        assert rel(got, want) < 3 * 0.042 + 4 * 2.0 ** -8
