"""Global gradient norm, clipping and the update on clipped gradients, through the C ABI.

Tolerances (e = 2^-24): the sum of squares is 64-bit, so the norm and the factor are off by their rounding to fp32 (e each); a clipped
element is off by the factor's rounding and the product's: 2 e.  The update's own roundings are those of et_update_masked, which it has to
agree with bit for bit on the same (clipped) gradients.
"""
import numpy as np
import pytest
import torch

import paper_2312_14227_b200 as et
from oracle import token_oracle as tok

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
E = 2.0 ** -24


def _layers(d, blocks):
    return [(d, d, 0, 1, -1, et.ET_LAYER_NORM, 1e-5), (d, 3 * d + 8, 0, 1, -1), (3 * d + 8, d, 0, 1, -1)] * blocks


class Net:
    def __init__(self, layers, dtype=et.ET_F32, seed=0, mask=None, opt="sgd", master=False, offset=0, gscale=1e-2):
        g = torch.Generator(device=DEV)
        g.manual_seed(seed)
        self.layers, self.dtype = layers, dtype
        et.et_debug_guard_regions(True)
        self.s = et.et_stack_create(layers, 8, dtype)
        et.et_debug_guard_regions(False)
        tdt = torch.bfloat16 if dtype == et.ET_BF16 else torch.float32
        shapes = []
        for ly in layers:
            kind = ly[5] if len(ly) > 5 else 0
            shapes += [(ly[1],) if kind == et.ET_LAYER_NORM else (ly[0], ly[1]), (ly[1],)]
        self.params = [torch.randn(s, generator=g, device=DEV).mul_(0.02).to(tdt) for s in shapes]
        self.ws = torch.empty(et.et_stack_workspace_bytes(self.s), dtype=torch.uint8, device=DEV)
        et.et_stack_bind(self.s, self.params[0::2], self.params[1::2], self.ws)
        n = len(shapes)
        self.mask = np.ones(n, dtype=np.uint8) if mask is None else np.asarray(mask, dtype=np.uint8)
        # `offset` floats in front: gradients that start off the 16-byte boundaries
        self.raw = [torch.randn(p.numel() + offset, generator=g, device=DEV) * gscale for p in self.params]
        self.grads = [r[offset:] for r in self.raw]
        self.master = [p.float() for p in self.params] if master else None
        if master:
            et.et_stack_bind_master(self.s, self.master[0::2], self.master[1::2])
        self.st = [[torch.rand(p.shape, generator=g, device=DEV) * v for p in self.params] for v in (1e-3, 1e-5)]
        if opt == "sgdw":
            et.et_stack_set_optimizer(self.s, et.ET_OPT_SGDW, self.st[0], momentum=0.9, weight_decay=1e-3)
        elif opt == "adam":
            et.et_stack_set_optimizer(self.s, et.ET_OPT_ADAM, self.st[0], self.st[1])
            et.et_stack_set_optimizer_step(self.s, 7)
        self.norm = torch.full((2,), float("nan"), device=DEV)

    def ptrs(self, ts):
        return [t if m else None for t, m in zip(ts, self.mask)]

    def oracle(self, max_norm):
        return tok.clip_factor([g.double().cpu().numpy() for g, m in zip(self.grads, self.mask) if m], max_norm)

    def check(self):
        torch.cuda.synchronize()
        st, bad = et.et_debug_check_guards(self.s)
        assert st == et.ET_OK, bad

    def state(self):
        return [x.clone() for x in self.params + (self.master or []) + self.st[0] + self.st[1]]


NETS = [([(3, 5, 0, 1, -1)], 0), ([(1, 1, 0, 1, -1)], 0), (_layers(136, 2), 0), (_layers(40, 3), 1), (_layers(8, 60), 0),
        (_layers(16, 180), 0), ([(1000, 4100, 0, 1, -1), (4100, 900, 0, 1, -1)], 3)]


@pytest.mark.parametrize("layers,offset", NETS)
def test_norm_and_clip(layers, offset):
    n = Net(layers, offset=offset, seed=len(layers))
    rng = np.random.default_rng(1)
    n.mask = (rng.random(len(n.params)) < 0.7).astype(np.uint8)
    n.mask[-1] = 1
    norm, _ = n.oracle(1.0)
    et.et_grad_norm(n.s, n.mask, n.ptrs(n.grads), n.norm)
    assert abs(float(n.norm[0]) - norm) <= 2 * E * norm and float(n.norm[1]) == 1.0
    for max_norm in (float(np.float32(0.3 * norm)), float(np.float32(2 * norm)), float("inf")):
        outs = [torch.full((p.numel() + 2,), 7.0, device=DEV) for p in n.params]
        views = [o[1:-1] for o in outs]                       # misaligned, with a word in front and behind
        before = [g.clone() for g in n.grads]
        et.et_clip_grads(n.s, n.mask, n.ptrs(n.grads), n.ptrs(views), max_norm, n.norm)
        n.check()
        _, f = n.oracle(max_norm)
        got = n.norm.cpu().numpy().astype(np.float64)
        assert abs(got[0] - norm) <= 2 * E * norm and abs(got[1] - f) <= 2 * E * f
        for g, b, v, o, m in zip(n.grads, before, views, outs, n.mask):
            assert torch.equal(g, b)
            assert float(o[0]) == 7.0 and float(o[-1]) == 7.0
            if not m:
                assert (o == 7.0).all()
                continue
            err = (v.double() - g.double() * f).abs()
            assert (err <= 3 * E * g.double().abs() * f).all()
            if f == 1.0:
                assert torch.equal(v, g)


def test_clip_in_place():
    n = Net(_layers(72, 2), seed=3)
    norm, _ = n.oracle(1.0)
    before = [g.clone() for g in n.grads]
    et.et_clip_grads(n.s, n.mask, n.grads, n.grads, 2 * norm)                 # nothing to clip, no report asked for
    n.check()
    assert all(torch.equal(a, b) for a, b in zip(before, n.grads))
    outs = [torch.empty_like(g) for g in n.grads]
    et.et_clip_grads(n.s, n.mask, n.grads, outs, 0.25 * norm)
    et.et_clip_grads(n.s, n.mask, n.grads, n.grads, 0.25 * norm, n.norm)
    n.check()
    assert all(torch.equal(a, b) for a, b in zip(outs, n.grads))


def test_nothing_selected():
    n = Net(_layers(16, 1))
    n.mask[:] = 0
    none = [None] * len(n.params)
    for call in (lambda: et.et_grad_norm(n.s, n.mask, none, n.norm), lambda: et.et_clip_grads(n.s, n.mask, none, none, 1.0, n.norm),
                 lambda: et.et_update_clipped(n.s, n.mask, none, 0.1, 1.0, n.norm)):
        n.norm.fill_(float("nan"))
        before = n.state()
        call()
        n.check()
        assert n.norm.tolist() == [0.0, 1.0]
        assert all(torch.equal(a, b) for a, b in zip(before, n.state()))
    et.et_clip_grads(n.s, n.mask, none, none, 1.0)
    et.et_update_clipped(n.s, n.mask, none, 0.1, 1.0)


@pytest.mark.parametrize("scale", [1e20, 1e30, 1e-25, 1e-30])
def test_squares_outside_the_range_of_fp32(scale):
    n = Net(_layers(40, 1), gscale=scale)
    norm, f = n.oracle(scale)
    outs = [torch.empty_like(g) for g in n.grads]
    et.et_clip_grads(n.s, n.mask, n.grads, outs, scale, n.norm)
    n.check()
    assert abs(float(n.norm[0]) - norm) <= 2 * E * norm and abs(float(n.norm[1]) - f) <= 2 * E * f


def test_zero_gradients():
    n = Net(_layers(40, 1), gscale=0.0)
    outs = [torch.full_like(g, 3.0) for g in n.grads]
    et.et_clip_grads(n.s, n.mask, n.grads, outs, 1.0, n.norm)
    n.check()
    assert n.norm.tolist() == [0.0, 1.0] and all((o == 0).all() for o in outs)


@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("opt", ["sgd", "sgdw", "adam"])
def test_a_norm_that_is_not_finite_leaves_the_step_out(bad, opt):
    n = Net(_layers(40, 2), dtype=et.ET_BF16, master=True, opt=opt)
    n.grads[4][17] = bad
    before = n.state()
    et.et_update_clipped(n.s, n.mask, n.grads, 0.1, 1.0, n.norm)
    n.check()
    assert not np.isfinite(float(n.norm[0])) and float(n.norm[1]) == 0.0
    assert all(torch.equal(a, b) for a, b in zip(before, n.state()))
    et.et_grad_norm(n.s, n.mask, n.grads, n.norm)
    assert float(n.norm[1]) == 0.0
    outs = [torch.full_like(g, 3.0) for g in n.grads]
    et.et_clip_grads(n.s, n.mask, n.grads, outs, 1.0, n.norm)
    n.check()
    assert all((o == 0).all() for o in outs)


@pytest.mark.parametrize("opt", ["sgd", "sgdw", "adam"])
@pytest.mark.parametrize("dtype,master", [(et.ET_F32, False), (et.ET_BF16, False), (et.ET_BF16, True)])
@pytest.mark.parametrize("layers", [_layers(136, 2), _layers(16, 180)])
def test_update_agrees_with_clip_then_update(opt, dtype, master, layers):
    mask = (np.random.default_rng(5).random(2 * len(layers)) < 0.6).astype(np.uint8)
    for clip in (0.3, 3.0):
        a, b = (Net(layers, dtype, seed=9, mask=mask, opt=opt, master=master) for _ in range(2))
        norm, _ = a.oracle(1.0)
        et.et_update_clipped(a.s, a.mask, a.ptrs(a.grads), 0.05, clip * norm, a.norm)
        outs = [torch.empty_like(g) for g in b.grads]
        et.et_clip_grads(b.s, b.mask, b.ptrs(b.grads), b.ptrs(outs), clip * norm, b.norm)
        et.et_update_masked(b.s, b.mask, b.ptrs(outs), 0.05)
        a.check()
        b.check()
        assert torch.equal(a.norm, b.norm)
        for x, y in zip(a.state(), b.state()):
            assert torch.equal(x, y)


def test_update_against_the_formula():
    n = Net(_layers(72, 2), opt="adam", seed=11)
    norm, f = n.oracle(1.0)
    max_norm = float(np.float32(0.2 * norm))
    _, f = n.oracle(max_norm)
    w, m, v = ([x.double() for x in xs] for xs in (n.params, n.st[0], n.st[1]))
    et.et_update_clipped(n.s, n.mask, n.grads, 0.01, max_norm)
    n.check()
    b1, b2, eps = (float(np.float32(x)) for x in (0.9, 0.999, 1e-8))
    lr = float(np.float32(0.01))
    for i, g in enumerate(n.grads):
        g = (g.double() * f).reshape(w[i].shape)
        m1, v1 = b1 * m[i] + (1 - b1) * g, b2 * v[i] + (1 - b2) * g * g
        step = lr * (m1 / (1 - b1 ** 7)) / ((v1 / (1 - b2 ** 7)).sqrt() + eps)
        # m, v: g is off by 3 e, each product and sum rounds (4 e of the parts); 1 - b1 and 1 - b2 are formed in fp32: e / (1 - b) relative.
        # step: m's and half of v's relative error and about six roundings; the weight rounds once
        assert ((n.st[0][i].double() - m1).abs() <= 8 * E * (b1 * m[i].abs() + (1 - b1) * g.abs())).all()
        tv = (8 + 1 / (1 - b2)) * E * (b2 * v[i] + (1 - b2) * g * g)
        assert ((n.st[1][i].double() - v1).abs() <= tv).all()
        rel = (0.5 * tv / v1 + 16 * E)
        tm = lr * 16 * E * (b1 * m[i].abs() + (1 - b1) * g.abs()) / (1 - b1 ** 7) / ((v1 / (1 - b2 ** 7)).sqrt() + eps)
        assert ((n.params[i].double() - (w[i] - step)).abs() <= step.abs() * rel + tm + 2 * E * (w[i].abs() + step.abs())).all()


def test_same_inputs_same_bits_and_replay():
    n = Net(_layers(136, 3), seed=13)
    outs = [torch.empty_like(g) for g in n.grads]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    et.et_clip_grads(n.s, n.mask, n.grads, outs, 0.1, n.norm, stream=side)
    torch.cuda.synchronize()
    first = [o.clone() for o in outs] + [n.norm.clone()]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        et.et_clip_grads(n.s, n.mask, n.grads, outs, 0.1, n.norm, stream=side)
    for o in outs:
        o.fill_(float("nan"))
    g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, outs + [n.norm]))
    for x in n.grads:
        x.mul_(2.0)                                           # doubled gradients: the same clipped ones (powers of two are exact)
    g.replay()
    n.check()
    assert all(torch.equal(a, b) for a, b in zip(first[:-1], outs)) and float(n.norm[0]) == 2 * float(first[-1][0])
    del g


def test_a_tensor_beyond_32_bit_offsets():
    k = 47000                                            # 2.2e9 elements
    s = et.et_stack_create([(k, k, 0, 1, -1)], 1, et.ET_F32)
    W, b = torch.zeros(k * k, device=DEV), torch.zeros(k, device=DEV)
    ws = torch.empty(et.et_stack_workspace_bytes(s), dtype=torch.uint8, device=DEV)
    et.et_stack_bind(s, [W], [b], ws)
    g = torch.zeros(k * k, device=DEV)
    g[-1], g[0], g[2 ** 31] = 3.0, 4.0, 12.0
    norm = torch.empty(2, device=DEV)
    et.et_update_clipped(s, [1, 0], [g, None], 1.0, 6.5, norm)
    torch.cuda.synchronize()
    assert norm.tolist() == [13.0, 0.5]
    assert float(W[-1]) == -1.5 and float(W[0]) == -2.0 and float(W[2 ** 31]) == -6.0 and int((W != 0).sum()) == 3
    et.et_clip_grads(s, [1, 0], [g, None], [g, None], 6.5, norm)
    torch.cuda.synchronize()
    assert float(g[-1]) == 1.5 and float(g[0]) == 2.0 and float(g[2 ** 31]) == 6.0 and int((g != 0).sum()) == 3
