"""Rotary, gated and dropout layers against the float64 oracle, through the C ABI.

Tolerances: rotary: cosine and sine off by 2^-22 (half a unit of a 24-bit half turn, pi 2^-25, and two steps of sincospi), three fp32
roundings and the store; gated: the oracle's own bounds; dropout: one product and one sum in fp32 and the store, dropped elements
exactly 0 (or the residual)."""
import numpy as np
import pytest
import torch

import paper_2312_14227_b200 as et
from oracle import block_oracle as blk

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F, B = et.ET_F32, et.ET_BF16
TDT = {F: torch.float32, B: torch.bfloat16}
STEP = {F: blk.E, B: blk.U}


def dev(a, dtype):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(TDT[dtype]).to(DEV)


def f64(t):
    return t.double().cpu().numpy()


def desc(kind, i, o, **k):
    return et.et_layer_desc(**{"in_features": i, "out_features": o, "fold": 1, "residual_src": -1, "kind": kind, **k})


class Run:
    """A stack with its input, output gradient and the gradient of its input; guard words round the workspace, guard rows behind outputs."""

    def __init__(self, layers, M, dtype, W=None, b=None, seed=0, x=None):
        rng = np.random.default_rng(seed)
        self.M, self.layers = M, layers
        et.et_debug_guard_regions(True)
        self.s = et.et_stack_create(layers, M, dtype)
        et.et_debug_guard_regions(False)
        self.ws = torch.empty(et.et_stack_workspace_bytes(self.s), dtype=torch.uint8, device=DEV)
        self.ws.fill_(0xFF)
        self.W, self.b = W or [None] * len(layers), b or [None] * len(layers)
        et.et_stack_bind(self.s, self.W, self.b, self.ws)
        out = layers[-1].out_features // layers[-1].fold
        self.x = dev(rng.normal(size=(M, layers[0].in_features)), dtype) if x is None else x
        self.dY = dev(rng.normal(size=(M, out)), dtype)
        self.y = torch.full((M + 1, out), 7.0, dtype=TDT[dtype], device=DEV)
        self.dX = torch.full((M + 1, layers[0].in_features), 7.0, dtype=TDT[dtype], device=DEV)
        et.et_stack_set_input_gradient(self.s, self.dX)

    def __call__(self, mask=None, grads=None, **k):
        et.et_forward_stack(self.s, self.x, self.y)
        et.et_backward_elastic(self.s, self.dY, mask or [0] * (2 * len(self.layers)), grads, **k)
        assert et.et_device_status(self.s) == et.ET_OK
        st, bad = et.et_debug_check_guards(self.s)
        assert st == et.ET_OK, bad
        assert bool((self.y[self.M] == 7).all()) and bool((self.dX[self.M] == 7).all())
        return self.y[:self.M], self.dX[:self.M]


def within(name, a, want, err):
    a = f64(a)
    assert np.isfinite(a).all(), name
    off = np.abs(a - want) - err
    assert off.max() <= 1e-37, (name, np.unravel_index(off.argmax(), off.shape), float(off.max()))


# ------------------------------------------------------------------------------------------ rotary
def rotary(M, heads, kv, dim, sections, dtype, positions=None, seq_len=0, theta=10000.0, adjacent=False, own=False, seed=0):
    w = (heads + 2 * kv) * dim
    d = desc(et.ET_LAYER_ROTARY, w, w, heads=heads, kv_heads=kv, head_dim=dim, axes=len(sections), sections=tuple(sections) + (0,) * (3 - len(sections)),
             pairing=int(adjacent), spectrum=int(own), theta=theta, seq_len=seq_len)
    r = Run([d], M, dtype, seed=seed)
    if positions is not None:
        et.et_stack_set_positions(r.s, torch.tensor(np.asarray(positions), dtype=torch.int32, device=DEV))
    else:
        positions = [np.arange(M) % (seq_len or M)]
    y, dX = r()
    for name, a, v, back in (("y", y, r.x, False), ("dX", dX, r.dY, True)):
        want, size = blk.rotary(f64(v), heads, kv, dim, sections, positions, float(np.float32(theta)), adjacent, own, back)
        within(name, a, want, size * (2.0 ** -22 + 3 * blk.E) + np.where(size > 0, STEP[dtype], 0.0) * np.abs(want))
    return r


@pytest.mark.parametrize("dtype", [F, B])
@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("M,heads,kv,dim,sections", [(1, 1, 1, 8, (4,)), (37, 4, 2, 64, (32,)), (130, 3, 1, 80, (20, 12)), (33, 2, 2, 128, (22, 21, 21)),
                                                     (50, 2, 1, 24, (1, 1, 1)), (7, 1, 1, 16, (5,)), (300, 2, 2, 96, (16, 16))])
def test_rotary(M, heads, kv, dim, sections, adjacent, dtype):
    rng = np.random.default_rng(M)
    pos = rng.integers(0, 5000, (len(sections), M))
    for own in (False, True):
        rotary(M, heads, kv, dim, sections, dtype, pos, adjacent=adjacent, own=own, seed=M)


@pytest.mark.parametrize("dtype", [F, B])
def test_rotary_positions_far_negative_and_not_given(dtype):
    rng = np.random.default_rng(0)
    far = np.concatenate([rng.integers(2 ** 30, 2 ** 31 - 1, 20), [2 ** 31 - 1, -2 ** 31, -1, 0, 1], -rng.integers(1, 2 ** 20, 20)])
    rotary(45, 2, 1, 64, (32,), dtype, [far], theta=500000.0)
    rotary(45, 2, 1, 64, (16, 16), dtype, [far, far[::-1].copy()], theta=100.0, own=True)
    rotary(45, 2, 1, 64, (16,), dtype)
    rotary(45, 2, 1, 64, (32,), dtype, seq_len=9)
    rotary(45, 2, 1, 64, (32,), dtype, [far], theta=0.5)              # frequencies above 1


def test_rotary_of_odd_widths_in_fp32():
    rotary(11, 2, 1, 6, (1, 2), F, np.arange(22).reshape(2, 11))
    rotary(11, 3, 2, 7, (3,), F, [np.arange(11)], adjacent=True)


def test_rotary_of_several_axes_needs_positions():
    d = desc(et.ET_LAYER_ROTARY, 24, 24, heads=1, kv_heads=1, head_dim=8, axes=2, sections=(2, 2, 0), theta=10.0)
    r = Run([d], 4, F)
    with pytest.raises(et.EtError) as e:
        r()
    assert e.value.status == et.ET_ERR_STATE


# ------------------------------------------------------------------------------------------ gated
def gated(M, K, h, act, dtype, seed=0, mask=(1, 1)):
    rng = np.random.default_rng(seed)
    W, b = dev(rng.normal(size=(K, 2 * h)) / np.sqrt(K), dtype), dev(rng.normal(size=2 * h) * 0.3, dtype)
    r = Run([desc(et.ET_LAYER_GATED, K, 2 * h, fold=2, act=act)], M, dtype, [W], [b], seed=seed + 1)
    grads = [torch.full((K, 2 * h), float("nan"), device=DEV) if mask[0] else None, torch.full((2 * h,), float("nan"), device=DEV) if mask[1] else None]
    y, dX = r(list(mask), grads)
    o = blk.gated(f64(r.x), f64(W), f64(b), act, f64(r.dY), STEP[dtype])
    within("y", y, *o["y"])
    within("dX", dX, *o["dx"])
    for name, g in zip(("dW", "db"), grads):
        if g is not None:
            within(name, g, *o[name])
    return r


@pytest.mark.parametrize("act", [et.ET_ACT_GELU_TANH, et.ET_ACT_RELU, et.ET_ACT_SILU])
@pytest.mark.parametrize("dtype", [F, B])
@pytest.mark.parametrize("M,K,h", [(1, 8, 8), (5, 16, 24), (100, 136, 344), (129, 72, 64), (257, 64, 136), (300, 200, 128), (513, 64, 72)])
def test_gated(M, K, h, act, dtype):
    gated(M, K, h, act, dtype, seed=M)


def block_pair(M, K, h, N, act, residual=False, dropout=False, seed=0):
    """Gated layer with a dense layer above: dZ comes out of that layer's error-gradient product (not where something lies between)."""
    rng = np.random.default_rng(seed)
    W = [dev(rng.normal(size=(K, 2 * h)) / np.sqrt(K), B), dev(rng.normal(size=(h, N)) / np.sqrt(h), B)]
    b = [dev(rng.normal(size=2 * h) * 0.3, B), dev(rng.normal(size=N) * 0.3, B)]
    layers = [desc(et.ET_LAYER_GATED, K, 2 * h, fold=2, act=act), desc(et.ET_LAYER_DENSE, h, N, residual_src=1 if residual else -1)]
    r = Run(layers, M, B, W, b, seed=seed + 1)
    grads = [torch.full(p.shape, float("nan"), device=DEV) for q in zip(W, b) for p in q]
    y, dX = r([1, 1, 1, 1], grads)
    g = f64(r.dY) @ f64(W[1]).T
    gerr = blk.E * (N + 2) * (np.abs(f64(r.dY)) @ np.abs(f64(W[1])).T)
    if residual:
        g = g + f64(r.dY)
        gerr = gerr + (blk.U + blk.E) * np.abs(g)        # the gradient of the gated layer's output is stored
    o = blk.gated(f64(r.x), f64(W[0]), f64(b[0]), act, g, blk.U, dy_err=gerr)
    within("dX", dX, *o["dx"])
    within("dW", grads[0], *o["dW"])
    within("db", grads[1], *o["db"])
    a, aerr = o["y"]
    out = a @ f64(W[1]) + f64(b[1]) + (a if residual else 0)
    size = np.abs(a) @ np.abs(f64(W[1])) + np.abs(f64(b[1]))
    within("y", y, out, (aerr @ np.abs(f64(W[1]))) + blk.E * (h + 3) * size + (aerr if residual else 0) + blk.U * np.abs(out))
    within("dW2", grads[2], a.T @ f64(r.dY), (aerr + blk.E * (M + 2) * np.abs(a)).T @ np.abs(f64(r.dY)))
    return r


@pytest.mark.parametrize("act", [et.ET_ACT_GELU_TANH, et.ET_ACT_RELU, et.ET_ACT_SILU])
@pytest.mark.parametrize("M,K,h,N", [(1, 8, 8, 8), (37, 24, 72, 40), (300, 136, 344, 136), (257, 64, 128, 64), (850, 40, 4808, 24)])
def test_gated_below_a_dense_layer(M, K, h, N, act):
    block_pair(M, K, h, N, act, seed=M)


def test_gated_whose_output_joins_a_residual():
    block_pair(200, 64, 96, 96, et.ET_ACT_SILU, residual=True)


def test_gated_below_a_gated_layer_and_two_streams():
    rng = np.random.default_rng(7)
    W = [dev(rng.normal(size=(40, 112)) / 6, B), dev(rng.normal(size=(56, 144)) / 7, B), dev(rng.normal(size=(72, 40)) / 8, B)]
    b = [dev(rng.normal(size=n) * 0.2, B) for n in (112, 144, 40)]
    layers = [desc(et.ET_LAYER_GATED, 40, 112, fold=2, act=3), desc(et.ET_LAYER_GATED, 56, 144, fold=2, act=1), desc(et.ET_LAYER_DENSE, 72, 40)]
    for streams in (0, 1):
        r = Run(layers, 333, B, W, b)
        et.et_stack_set_option(r.s, et.ET_OPTION_TWO_STREAMS, streams)
        grads = [torch.full(p.shape, float("nan"), device=DEV) for q in zip(W, b) for p in q]
        y, dX = r([1] * 6, grads)
        leaf = [p.double().requires_grad_() for q in zip(W, b) for p in q]
        x = r.x.double().requires_grad_()
        z = x @ leaf[0] + leaf[1]
        z = torch.nn.functional.silu(z[:, :56]) * z[:, 56:] @ leaf[2] + leaf[3]
        out = torch.nn.functional.gelu(z[:, :72], approximate="tanh") * z[:, 72:] @ leaf[4] + leaf[5]
        want = torch.autograd.grad(out, [x] + leaf, r.dY.double())
        for a, w in zip([dX] + grads, want):
            assert (a.double() - w).abs().max() <= 2e-2 * w.abs().max()


def test_gates_beyond_what_z_is_kept_in():
    """Z is kept at most 65504: the output is formed from all of it, gradients are those of a gate or factor of 65504."""
    W, b = torch.eye(8, 16, device=DEV).to(torch.bfloat16), dev([0] * 16, B)
    W[:, 8:] = torch.eye(8, device=DEV)
    x = dev([[1e6, -1e6, 2e5, 1, 70000, 65536, 0, 3]] * 2, B)
    r = Run([desc(et.ET_LAYER_GATED, 8, 16, fold=2, act=et.ET_ACT_RELU)], 2, B, [W], [b], x=x)
    y, dX = r()
    z = f64(x)
    assert np.abs(f64(y) - np.maximum(z, 0) * z).max() <= blk.U * 1e12
    held = np.clip(z, -65504, 65504)
    want = f64(r.dY) * (held * (held > 0) + np.maximum(held, 0))
    assert np.abs(f64(dX) - want).max() <= 4 * blk.U * np.abs(want).max()


def test_gated_in_wide_tiles_and_long_contractions():
    gated(2600, 24, 1928, et.ET_ACT_SILU, B)                          # enough tiles for the 128-column form, a ragged last one
    gated(300, 2056, 136, et.ET_ACT_GELU_TANH, B)
    gated(40, 40, 33, et.ET_ACT_SILU, F)                              # odd widths


@pytest.mark.parametrize("mask", [(1, 0), (0, 1), (0, 0)])
def test_gated_masks(mask):
    gated(130, 64, 72, et.ET_ACT_SILU, B, mask=mask)


def test_gated_saturates():
    """Gates far out: SiLU and GELU of large values are the value or 0, their slopes 1 or 0; nothing overflows."""
    for dtype in (F, B):
        for act in (1, 2, 3):
            W, b = torch.eye(8, 16, device=DEV).to(TDT[dtype]), dev([0] * 8 + [1] * 8, dtype)
            x = dev([[-3e4, -200, -20, 20, 200, 3e4, 0, 1]] * 3, dtype)
            r = Run([desc(et.ET_LAYER_GATED, 8, 16, fold=2, act=act)], 3, dtype, [W], [b], x=x)
            y, dX = r()
            z = f64(x)[:, :6]
            assert np.abs(f64(y)[:, :6] - np.maximum(z, 0)).max() <= 1e-3
            assert np.abs(f64(dX)[:, :6] - f64(r.dY)[:, :6] * (z > 0)).max() <= 1e-3


# ------------------------------------------------------------------------------------------ dropout
SEEDS = [(0, 0), (12345678901234567890, 7), (2 ** 64 - 1, 2 ** 32 + 5)]


def seed_of(seed, step):
    return torch.tensor([seed - 2 ** 64 if seed >= 2 ** 63 else seed, step], dtype=torch.int64, device=DEV)


@pytest.mark.parametrize("dtype,M,width", [(F, 1, 1), (F, 50, 197), (F, 3, 2), (B, 1, 8), (B, 40, 72), (B, 129, 256)])
@pytest.mark.parametrize("p", [0.1, 0.5, 0.97])
@pytest.mark.parametrize("residual", [False, True])
def test_dropout(dtype, M, width, p, residual):
    p = float(np.float32(p))
    r = Run([desc(et.ET_LAYER_DROPOUT, width, width, drop=p, residual_src=0 if residual else -1)], M, dtype)
    for seed, step in SEEDS:
        et.et_stack_set_dropout_seed(r.s, seed_of(seed, step))
        y, dX = r()
        keep = blk.kept(0, M * width, p, seed, step, 0).reshape(M, width)
        scale = 1 / (1 - round(p * 2 ** 32) / 2 ** 32)
        for a, v in ((y, f64(r.x)), (dX, f64(r.dY))):
            part = np.where(keep, v * scale, 0.0)
            want = part + v if residual else part
            within("dropout", a, want, 2 * blk.E * np.abs(part) + (blk.E if residual else 0) * np.abs(want) + STEP[dtype] * np.abs(want))
            if not residual:
                assert not f64(a)[~keep].any()


def test_dropout_without_a_seed_and_of_nothing():
    r = Run([desc(et.ET_LAYER_DROPOUT, 40, 40, drop=0.5)], 9, B)
    y, dX = r()
    assert torch.equal(y, r.x) and torch.equal(dX, r.dY)
    et.et_stack_set_dropout_seed(r.s, seed_of(1, 1))
    assert not torch.equal(r()[0], r.x)
    et.et_stack_set_dropout_seed(r.s, None)
    assert torch.equal(r()[0], r.x)
    r = Run([desc(et.ET_LAYER_DROPOUT, 40, 40, drop=0.0)], 9, F)
    et.et_stack_set_dropout_seed(r.s, seed_of(1, 1))
    assert torch.equal(r()[0], r.x)


def test_dropped_elements_are_not_looked_at():
    r = Run([desc(et.ET_LAYER_DROPOUT, 64, 64, drop=0.5)], 20, B)
    et.et_stack_set_dropout_seed(r.s, seed_of(3, 1))
    keep = torch.from_numpy(blk.kept(0, 1280, 0.5, 3, 1, 0).reshape(20, 64)).to(DEV)
    r.x[~keep] = float("nan")
    assert bool(torch.isfinite(r()[0]).all())


def test_dropout_layers_draw_apart_and_a_replay_follows_the_step_in_memory():
    layers = [desc(et.ET_LAYER_DROPOUT, 64, 64, drop=0.5), desc(et.ET_LAYER_DROPOUT, 64, 64, drop=0.5)]
    ones = torch.ones(30, 64, device=DEV)
    r = Run(layers, 30, F, x=ones)
    seed = seed_of(9, 4)
    et.et_stack_set_dropout_seed(r.s, seed)
    r()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        et.et_forward_stack(r.s, r.x, r.y, stream=side)
        et.et_backward_elastic(r.s, r.dY, [0] * 4, stream=side)
    for step in (4, 5, 6):
        seed[1] = step
        graph.replay()
        torch.cuda.synchronize()
        keep = blk.kept(0, 1920, 0.5, 9, step, 0) & blk.kept(0, 1920, 0.5, 9, step, 1)
        assert np.array_equal(f64(r.y[:30]).ravel(), 4.0 * keep)
        assert torch.equal(r.dX[:30] != 0, torch.from_numpy(keep.reshape(30, 64)).to(DEV) & (r.dY != 0))


@pytest.mark.parametrize("act", [1, 2])
def test_dropout_above_an_activation(act):
    """The gradient goes on through the activation below, and joins a skip connection."""
    rng = np.random.default_rng(act)
    dense = desc(et.ET_LAYER_DENSE, 16, 24, act=act)
    top = desc(et.ET_LAYER_DENSE, 24, 24, residual_src=1)
    W, b = [dev(rng.normal(size=(16, 24)) / 4, F), None, dev(rng.normal(size=(24, 24)) / 5, F)], [dev(rng.normal(size=24), F), None, dev(np.zeros(24), F)]
    r = Run([dense, desc(et.ET_LAYER_DROPOUT, 24, 24, drop=0.25), top], 10, F, W, b)
    et.et_stack_set_dropout_seed(r.s, seed_of(5, 6))
    y, dX = r()
    keep = blk.kept(0, 240, 0.25, 5, 6, 1).reshape(10, 24)
    z = f64(r.x) @ f64(W[0]) + f64(b[0])
    f, slope, _ = blk.act(z, act)
    want = np.where(keep, f / 0.75, 0) @ f64(W[2]) + f
    assert np.abs(f64(y) - want).max() <= 2e-5
    g = np.where(keep, f64(r.dY) @ f64(W[2]).T / 0.75, 0) + f64(r.dY)
    assert np.abs(f64(dX) - (g * slope) @ f64(W[0]).T).max() <= 2e-5


def test_dropout_offsets_beyond_32_bits():
    M, width = 1_050_000, 4096
    assert M * width > 2 ** 32
    d = desc(et.ET_LAYER_DROPOUT, width, width, drop=0.5)
    s = et.et_stack_create([d], M, B)
    ws = torch.empty(et.et_stack_workspace_bytes(s), dtype=torch.uint8, device=DEV)
    et.et_stack_bind(s, [None], [None], ws)
    x = torch.ones(M, width, dtype=torch.bfloat16, device=DEV)
    y = torch.zeros_like(x)
    seed = seed_of(77, 3)
    et.et_stack_set_dropout_seed(s, seed)
    et.et_forward_stack(s, x, y)
    torch.cuda.synchronize()
    for row in (0, 2 ** 20 - 1, 2 ** 20, M - 1):
        assert np.array_equal(f64(y[row]), 2.0 * blk.kept(row * width, width, 0.5, 77, 3, 0)), row


# ------------------------------------------------------------------------------------------ gradient of the input
@pytest.mark.parametrize("dtype,tol", [(F, 1e-4), (B, 2e-2)])
@pytest.mark.parametrize("mask", [0, 3, 15, 4])
def test_input_gradient_of_dense_and_norm_stacks(dtype, tol, mask):
    """Against the gradient that the same stack behind an identity layer (whose bias gradient sums it) and float64 autograd give."""
    rng = np.random.default_rng(4)
    M, d = 70, 64
    layers = [desc(et.ET_LAYER_NORM, d, d, eps=1e-5), desc(et.ET_LAYER_DENSE, d, 128, act=1), desc(et.ET_LAYER_DENSE, 128, d, residual_src=0)]
    W = [dev(1 + 0.1 * rng.normal(size=d), dtype), dev(rng.normal(size=(d, 128)) / 8, dtype), dev(rng.normal(size=(128, d)) / 11, dtype)]
    b = [dev(0.1 * rng.normal(size=n), dtype) for n in (d, 128, d)]
    r = Run(layers, M, dtype, W, b)
    bits = [mask >> i & 1 for i in range(6)]
    grads = [torch.zeros(t.shape, device=DEV) if m else None for t, m in zip([t for p in zip(W, b) for t in p], bits)]
    y, dX = r(bits, grads)
    x = r.x.double().requires_grad_()
    n = torch.nn.functional.layer_norm(x, (d,), W[0].double(), b[0].double(), 1e-5)
    out = torch.nn.functional.gelu(n @ W[1].double() + b[1].double(), approximate="tanh") @ W[2].double() + b[2].double() + x
    g, = torch.autograd.grad(out, x, r.dY.double())
    assert (y.double() - out).abs().max() <= tol * out.abs().max()
    assert (dX.double() - g).abs().max() <= tol * g.abs().max()


def test_input_gradient_of_dense_layers_alone_and_detached():
    rng = np.random.default_rng(6)
    layers = [desc(et.ET_LAYER_DENSE, 64, 128, act=2), desc(et.ET_LAYER_DENSE, 128, 64)]
    W, b = [dev(rng.normal(size=(64, 128)) / 8, B), dev(rng.normal(size=(128, 64)) / 11, B)], [dev(np.zeros(128), B), dev(np.zeros(64), B)]
    r = Run(layers, 300, B, W, b)
    g = [torch.zeros(64, 128, device=DEV), None, None, None]
    r([1, 0, 0, 0], g)
    rep = et.Report(2)
    et.et_backward_elastic(r.s, r.dY, [0, 0, 1, 0], [None, None, torch.zeros(128, 64, device=DEV), None], report=rep)
    assert rep.dgrad.tolist() == [1, 1] and rep.deepest == 1
    x, w0, w1 = r.x.double(), W[0].double(), W[1].double()
    want = ((r.dY.double() @ w1.T) * ((x @ w0) > 0)) @ w0.T
    assert (r.dX[:300].double() - want).abs().max() <= 2e-2 * want.abs().max()
    et.et_stack_set_input_gradient(r.s, None)
    r.dX.fill_(7)
    again = torch.zeros_like(g[0])
    r([1, 0, 0, 0], [again, None, None, None])                        # the one-launch path
    assert bool((r.dX == 7).all())
    assert (again - g[0]).abs().max() <= 2e-2 * g[0].abs().max()
