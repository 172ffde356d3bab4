"""The embedding layer against the float64 oracle, through the C ABI: lookup, gradient by sorted tokens, importance, updates, and a
whole fine-tuning step (embedding, dense layers, policy loss, backward, clipped update).

Tolerances (e = 2^-24): a looked-up value is one product, rounded to fp32 and to the storage type.  A gradient element of an id with k
rows is k - 1 fp32 additions and one product: e (k + 2) of scale * sum |g|.  An update adds one product and one rounding.
"""
import numpy as np
import pytest
import torch

import paper_2312_14227_b200 as et
import workloads as wl
from oracle import elastic_oracle as orc
from oracle import token_oracle as tok

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
E = 2.0 ** -24
F, B = et.ET_F32, et.ET_BF16


def _ids(rng, M, V, kind):
    if kind == "zipf":
        r = np.exp(rng.random(M) * np.log(V + 1.0)).astype(np.int64) - 1
        return rng.permutation(V)[np.clip(r, 0, V - 1)].astype(np.int32)
    if kind == "one":
        return np.full(M, V // 2, dtype=np.int32)
    if kind == "some-out":
        ids = rng.integers(0, V, M)
        ids[::3] = -1
        ids[1::7] = V
        ids[2::11] = 2 ** 31 - 1
        return ids.astype(np.int32)
    if kind == "all-out":
        return np.full(M, -1, dtype=np.int32)
    if kind == "ends":
        return rng.choice([0, V - 1], M).astype(np.int32)
    if kind == "ordered":
        return np.sort(rng.integers(0, V, M)).astype(np.int32)
    return rng.integers(0, V, M).astype(np.int32)


class Emb:
    def __init__(self, M, V, d, dtype, kind="uniform", scale=1.5, seed=0, master=False):
        rng = np.random.default_rng(seed)
        self.M, self.V, self.d, self.dtype, self.scale = M, V, d, dtype, scale
        self.tdt = torch.bfloat16 if dtype == B else torch.float32
        et.et_debug_guard_regions(True)
        self.s = et.et_stack_create([(V, d, 0, 1, -1, et.ET_LAYER_EMBEDDING)], M, dtype)
        et.et_debug_guard_regions(False)
        self.T = torch.from_numpy(rng.normal(size=(V, d)).astype(np.float32)).to(self.tdt).to(DEV)
        self.ids = _ids(rng, M, V, kind)
        self.x = torch.from_numpy(self.ids).to(DEV)
        self.dY = torch.from_numpy(rng.normal(size=(M, d)).astype(np.float32)).to(self.tdt).to(DEV)
        self.ws = torch.empty(et.et_stack_workspace_bytes(self.s), dtype=torch.uint8, device=DEV)
        et.et_stack_bind(self.s, [self.T], [None], self.ws)
        self.T32 = self.T.float() if master else None
        if master:
            et.et_stack_bind_master(self.s, [self.T32], [None])
        et.et_stack_set_embedding_scale(self.s, scale)
        self.y = torch.full((M, d), float("nan"), dtype=self.tdt, device=DEV)

    def check(self):
        torch.cuda.synchronize()
        st, bad = et.et_debug_check_guards(self.s)
        assert st == et.ET_OK, bad

    def forward(self):
        et.et_forward_stack(self.s, self.x, self.y)
        self.check()

    def oracle(self):
        """The gradient, the sum of absolute terms and the rows of each id, float64."""
        ok = (self.ids >= 0) & (self.ids < self.V)
        g, a, k = np.zeros((self.V, self.d)), np.zeros((self.V, self.d)), np.zeros(self.V)
        dY = self.dY.double().cpu().numpy()
        np.add.at(g, self.ids[ok], self.scale * dY[ok])
        np.add.at(a, self.ids[ok], abs(self.scale) * np.abs(dY[ok]))
        np.add.at(k, self.ids[ok], 1)
        return g, a, k

    def grad_tol(self):
        g, a, k = self.oracle()
        return g, E * (k[:, None] + 2) * a


SHAPES = [(1, 1, 8, F, "uniform"), (1, 1000, 8, B, "uniform"), (300, 50, 7, F, "uniform"), (300, 50, 200, F, "zipf"),
          (257, 1000, 264, B, "zipf"), (1000, 65536, 72, B, "uniform"), (5000, 700, 136, B, "zipf"), (4096, 511, 64, F, "ordered"),
          (4099, 512, 64, F, "some-out"), (2500, 130000, 40, B, "some-out"), (3000, 17, 8, B, "one"), (33, 3, 2056, B, "ends"),
          (64, 40, 4104, B, "zipf"), (70, 30, 2051, F, "zipf"), (100, 10, 16, F, "all-out"), (20000, 300000, 24, F, "zipf"),
          (9000, 4, 40, F, "ends")]


@pytest.mark.parametrize("M,V,d,dtype,kind", SHAPES)
def test_lookup(M, V, d, dtype, kind):
    c = Emb(M, V, d, dtype, kind, seed=M)
    c.forward()
    ok = (c.ids >= 0) & (c.ids < V)
    want = c.scale * c.T.double().cpu().numpy()[np.where(ok, c.ids, 0)] * ok[:, None]
    half = torch.finfo(c.tdt).eps / 2
    assert (np.abs(c.y.double().cpu().numpy() - want) <= np.abs(want) * (half + 2 * E)).all()


@pytest.mark.parametrize("M,V,d,dtype,kind", SHAPES)
def test_exported_gradient(M, V, d, dtype, kind):
    c = Emb(M, V, d, dtype, kind, seed=M + 1, scale=-0.75)
    c.forward()
    grad = torch.full((V, d), float("nan"), device=DEV)
    before = c.T.clone()
    rep = et.Report(1)
    et.et_backward_elastic(c.s, c.dY, [1, 0], [grad, None], report=rep)
    c.check()
    g, tol = c.grad_tol()
    assert (np.abs(grad.double().cpu().numpy() - g) <= tol).all()
    assert torch.equal(before, c.T)
    assert rep.deepest == 0 and rep.wgrad[0] == 1 and rep.bgrad[0] == 0 and rep.launches > 0


@pytest.mark.parametrize("master", [False, True])
@pytest.mark.parametrize("M,V,d,dtype,kind", [(300, 50, 200, F, "zipf"), (2500, 1300, 40, B, "some-out"), (700, 90, 2056, B, "zipf")])
def test_fused_sgd_touches_named_rows_only(M, V, d, dtype, kind, master):
    if master and dtype == F:
        pytest.skip("masters are for bf16 stacks")
    c = Emb(M, V, d, dtype, kind, seed=7, master=master)
    c.forward()
    named = np.unique(c.ids[(c.ids >= 0) & (c.ids < V)])
    rest = np.setdiff1d(np.arange(V), named)
    before = c.T.clone()
    lr = float(np.float32(0.05))
    et.et_backward_elastic(c.s, c.dY, [1, 0], flags=et.ET_FLAG_FUSE_SGD, lr=lr)
    c.check()
    g, tol = c.grad_tol()
    w = before.double().cpu().numpy()
    want = w - lr * g
    half = torch.finfo(c.tdt).eps / 2
    bound = lr * tol + 2 * E * (np.abs(lr * g) + np.abs(want))
    if master:
        assert (np.abs(c.T32.double().cpu().numpy() - want) <= bound).all()
        assert torch.equal(c.T32.to(torch.bfloat16), c.T)
    assert (np.abs(c.T.double().cpu().numpy() - want) <= bound + half * (np.abs(want) + bound)).all()
    assert torch.equal(c.T[rest], before[rest])


@pytest.mark.parametrize("dtype", [F, B])
@pytest.mark.parametrize("opt", ["sgdw", "adam"])
def test_optimisers_move_every_row(dtype, opt):
    """Momentum, decay and second moments act on rows without a token too: the fused step is the exported gradient's step."""
    a, b = (Emb(500, 90, 136, dtype, "zipf", seed=8) for _ in range(2))
    states = []
    for c in (a, b):
        st = [torch.full((90, 136), v, device=DEV) for v in (1e-2, 1e-4)]
        if opt == "sgdw":
            et.et_stack_set_optimizer(c.s, et.ET_OPT_SGDW, [st[0], None], momentum=0.9, weight_decay=1e-2)
        else:
            et.et_stack_set_optimizer(c.s, et.ET_OPT_ADAM, [st[0], None], [st[1], None])
        states.append(st)
        c.forward()
    et.et_backward_elastic(a.s, a.dY, [1, 0], flags=et.ET_FLAG_FUSE_SGD, lr=0.01)
    grad = torch.empty(90, 136, device=DEV)
    et.et_backward_elastic(b.s, b.dY, [1, 0], [grad, None])
    et.et_update_masked(b.s, [1, 0], [grad, None], 0.01)
    a.check()
    b.check()
    assert torch.equal(a.T, b.T) and all(torch.equal(x, y) for x, y in zip(*states))
    assert (states[0][0] != 1e-2).all()


@pytest.mark.parametrize("dtype,master", [(F, False), (B, False), (B, True)])
@pytest.mark.parametrize("snapshot", [False, True])
@pytest.mark.parametrize("M,V,d", [(500, 90, 136), (40, 3000, 264), (4000, 20, 8)])
def test_importance(dtype, master, snapshot, M, V, d):
    c = Emb(M, V, d, dtype, "zipf", seed=9, master=master)
    c.forward()
    rng = np.random.default_rng(10)
    dw = torch.from_numpy(rng.normal(size=(V, d)).astype(np.float32) * 1e-2).to(DEV)
    cur = c.T32 if master else c.T
    if snapshot:
        delta = (cur.float() - dw).to(cur.dtype)
        step = cur.double() - delta.double()
    else:
        delta = dw.to(c.tdt)
        step = delta.double()
    imp = torch.full((2,), float("nan"), device=DEV)
    grad = torch.empty(V, d, device=DEV)
    flags = et.ET_FLAG_DELTA_IS_SNAPSHOT if snapshot else 0
    et.et_backward_elastic(c.s, c.dY, [1, 0], [grad, None], [delta, None], imp, flags)
    c.check()
    g, tol = c.grad_tol()
    step = step.cpu().numpy()
    # each product and each addition of the sum rounds: at most (8 in a thread + 40 levels) e of the absolute sum; the step of a snapshot rounds once
    bound = (tol * np.abs(step)).sum() + 64 * E * np.abs(g * step).sum() + 64 * E * (np.abs(g) * np.abs(step)).sum()
    want = (g * step).sum()
    assert abs(float(imp[0]) - want) <= bound and float(imp[1]) == 0.0
    if not snapshot:
        et.et_importance(c.s, [1, 0], [grad, None], [delta, None], imp)
        assert abs(float(imp[0]) - want) <= bound and float(imp[1]) == 0.0
        et.et_tensor_metric(c.s, [1, 0], et.ET_METRIC_GRADIENT_MAGNITUDE, [grad, None], imp)
        assert abs(float(imp[0]) - np.abs(g).sum()) <= tol.sum() + 128 * E * np.abs(g).sum()


def test_same_inputs_same_bits_and_replay():
    c = Emb(6000, 5000, 264, B, "zipf", seed=12)
    grad = torch.empty(5000, 264, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())

    def step(st):
        et.et_forward_stack(c.s, c.x, c.y, stream=st)
        et.et_backward_elastic(c.s, c.dY, [1, 0], [grad, None], stream=st)

    step(side)
    torch.cuda.synchronize()
    first = grad.clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        step(side)
    for seed in (1, 2):
        c.x.copy_(torch.from_numpy(_ids(np.random.default_rng(seed), 6000, 5000, "some-out")).to(DEV))
        grad.fill_(float("nan"))
        g.replay()
        torch.cuda.synchronize()
        got, y = grad.clone(), c.y.clone()
        step(None)
        torch.cuda.synchronize()
        assert torch.equal(got, grad) and torch.equal(y, c.y)
    c.x.copy_(torch.from_numpy(c.ids).to(DEV))
    g.replay()
    c.check()
    assert torch.equal(first, grad)
    del g


# ---- in a stack -------------------------------------------------------------------------------------
def _token_stack(dtype, V=67, d=72, hid=136, out=104):
    return [wl.embedding_layer(V, d, 2.0), wl.norm_layer(d), wl.Layer(d, hid, act=wl.ACT_GELU_TANH), wl.Layer(hid, d, residual_src=1),
            wl.norm_layer(d), wl.Layer(d, out)]


class TokenNet:
    def __init__(self, dtype, M=150, seed=0, layers=None):
        rng = np.random.default_rng(seed)
        self.layers = layers or _token_stack(dtype)
        self.L, self.M, self.dtype = len(self.layers), M, dtype
        self.tdt = torch.bfloat16 if dtype == B else torch.float32
        et.et_debug_guard_regions(True)
        self.s = et.et_stack_create(self.layers, M, dtype)
        et.et_debug_guard_regions(False)
        self.params = []
        for ly in self.layers:
            if ly.kind == wl.KIND_EMBEDDING:
                pair = (rng.normal(size=(ly.in_features, ly.out_features)) * 0.3, np.zeros(0))
            elif ly.kind == wl.KIND_NORM:
                pair = (1 + 0.1 * rng.normal(size=ly.out_features), 0.1 * rng.normal(size=ly.out_features))
            else:
                pair = (rng.normal(size=(ly.in_features, ly.out_features)) / np.sqrt(ly.in_features), 0.1 * rng.normal(size=ly.out_features))
            self.params += [torch.from_numpy(p).to(self.tdt).to(DEV) for p in pair]
        self.ws = torch.empty(et.et_stack_workspace_bytes(self.s), dtype=torch.uint8, device=DEV)
        self.ids = rng.integers(0, self.layers[0].in_features, M).astype(np.int32)
        self.x = torch.from_numpy(self.ids).to(DEV)
        self.y = torch.empty(M, self.layers[-1].out_features, dtype=self.tdt, device=DEV)
        self.dY = torch.empty_like(self.y)
        self.targets = rng.integers(0, self.layers[-1].out_features, M).astype(np.int32)
        self.adv = rng.normal(size=M).astype(np.float32)
        self.bind()
        et.et_stack_set_embedding_scale(self.s, self.layers[0].scale)

    def bind(self):
        et.et_stack_bind(self.s, self.params[0::2], self.params[1::2], self.ws)

    def host(self, ts):
        return [t.double().cpu().numpy() for t in ts]

    def check(self):
        torch.cuda.synchronize()
        assert et.et_device_status(self.s) == et.ET_OK
        st, bad = et.et_debug_check_guards(self.s)
        assert st == et.ET_OK, bad


def _mask(L, sel=None):
    m = np.ones(2 * L, dtype=np.uint8)
    if sel is not None:
        m[:] = 0
        m[sel] = 1
    m[1] = 0
    return m


@pytest.mark.parametrize("dtype,tol", [(F, 1e-4), (B, 3e-2)])
@pytest.mark.parametrize("sel", [None, [0], [0, 4, 11], [2, 3], [10], [0, 2]])
@pytest.mark.parametrize("two_streams", [0, 1])
def test_fine_tuning_step(dtype, tol, sel, two_streams):
    """Lookup, dense layers, policy loss on the logits, masked backward, update on clipped gradients: as they are used together."""
    n = TokenNet(dtype, seed=3)
    et.et_stack_set_option(n.s, et.ET_OPTION_TWO_STREAMS, two_streams)
    mask = _mask(n.L, sel)
    before = [p.clone() for p in n.params]
    host = n.host(n.params)
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(DEV)  # noqa: E731
    loss, norm = torch.empty(4, device=DEV), torch.empty(2, device=DEV)
    grads = [torch.full(p.shape, float("nan"), device=DEV) if m else None for p, m in zip(n.params, mask)]
    et.et_forward_stack(n.s, n.x, n.y)
    et.et_loss_policy_grad(n.s, n.y, dev(n.targets), dev(n.adv), n.dY, loss_dev=loss, vocab=101)
    et.et_backward_elastic(n.s, n.dY, mask, grads)
    et.et_update_clipped(n.s, mask, grads, 0.1, 1e-3, norm)
    n.check()
    saved = orc.forward(n.layers, host[0::2], host[1::2], n.ids)
    rel = lambda a, o: np.abs(a - o).max() / max(np.abs(o).max(), 1e-30)  # noqa: E731
    assert rel(n.y.double().cpu().numpy(), saved.a[-1]) <= tol
    w = np.full(n.M, 1.0 / n.M)
    stats, _, dY, _ = tok.policy(saved.a[-1], n.targets, w, n.adv, None, None, 101, 1.0, 0.2, 0.2, 0.0)
    assert rel(n.dY.double().cpu().numpy(), dY) <= tol
    assert abs(float(loss[0]) - stats[0]) <= tol * np.abs(w * n.adv).sum()
    want, _ = orc.backward_masked(n.layers, host[0::2], saved, dY, mask)
    for t, m in enumerate(mask):
        if m:
            assert rel(grads[t].double().cpu().numpy(), want[t]) <= tol, t
    got_n, got_f = tok.clip_factor([g.double().cpu().numpy() for g in grads if g is not None], float(np.float32(1e-3)))
    assert abs(float(norm[0]) - got_n) <= 2 * E * got_n and abs(float(norm[1]) - got_f) <= 2 * E * got_f
    for p, b, g, m in zip(n.params, before, grads, mask):
        if not m:
            assert torch.equal(p, b)
        else:
            new = b.double() - 0.1 * got_f * g.double()
            half = torch.finfo(n.tdt).eps / 2
            assert ((p.double() - new).abs() <= (half + 2 * E) * new.abs() + 8 * E * (0.1 * got_f * g.double()).abs()).all()


@pytest.mark.parametrize("dtype", [F, B])
def test_stack_above_the_table_is_unchanged(dtype):
    """Layers above a lookup give what they give on the looked-up rows as an input."""
    n = TokenNet(dtype, seed=4)
    et.et_forward_stack(n.s, n.x, n.y)
    n.dY.normal_()
    mask = _mask(n.L, [4, 6, 7, 11])
    g1 = [torch.empty(p.shape, device=DEV) if m else None for p, m in zip(n.params, mask)]
    et.et_backward_elastic(n.s, n.dY, mask, g1)
    n.check()
    ok = torch.from_numpy(n.ids.astype(np.int64)).to(DEV)
    a1 = (n.params[0].float()[ok] * 2.0).to(n.tdt).contiguous()
    upper = [ly if ly.residual_src < 0 else wl.Layer(ly.in_features, ly.out_features, residual_src=ly.residual_src - 1) for ly in n.layers[1:]]
    s2 = et.et_stack_create(upper, n.M, dtype)
    ws = torch.empty(et.et_stack_workspace_bytes(s2), dtype=torch.uint8, device=DEV)
    et.et_stack_bind(s2, n.params[2::2], n.params[3::2], ws)
    y2 = torch.empty_like(n.y)
    et.et_forward_stack(s2, a1, y2)
    g2 = [torch.empty_like(g) if g is not None else None for g in g1[2:]]
    et.et_backward_elastic(s2, n.dY, mask[2:], g2)
    torch.cuda.synchronize()
    assert torch.equal(n.y, y2)
    assert all(torch.equal(a, b) for a, b in zip(g1[2:], g2) if a is not None)


@pytest.mark.parametrize("dtype", [F, B])
def test_profile_costs(dtype):
    n = TokenNet(dtype, seed=5)
    n.dY.zero_()
    before = [p.clone() for p in n.params]
    t_dw, t_dy, t_fwd = et.et_profile_costs(n.s, n.x, n.y, n.dY, 3)
    n.check()
    assert t_dw[0] > 0 and t_dw[1] == 0 and t_dy[0] == 0 and t_dy[1] == 0 and t_fwd > 0
    assert all(torch.equal(a, b) for a, b in zip(before, n.params))


@pytest.mark.parametrize("dtype,master", [(F, False), (B, False), (B, True)])
@pytest.mark.parametrize("opt", ["sgd", "sgdw", "adam"])
@pytest.mark.parametrize("M,V,d", [(4096, 700, 64), (4097, 700, 64), (9000, 5000, 40), (6000, 300, 1032)])
def test_fused_step_is_the_exported_gradients_step(dtype, master, opt, M, V, d):
    """Both ways of sorting, rows without a token filled beside either; with and without masters."""
    a, b = (Emb(M, V, d, dtype, "zipf", seed=21, master=master) for _ in range(2))
    states = []
    for c in (a, b):
        st = [torch.full((V, d), v, device=DEV) for v in (1e-2, 1e-4)]
        if opt == "sgdw":
            et.et_stack_set_optimizer(c.s, et.ET_OPT_SGDW, [st[0], None], momentum=0.9, weight_decay=1e-2)
        elif opt == "adam":
            et.et_stack_set_optimizer(c.s, et.ET_OPT_ADAM, [st[0], None], [st[1], None])
        states.append(st)
        c.forward()
    et.et_backward_elastic(a.s, a.dY, [1, 0], flags=et.ET_FLAG_FUSE_SGD, lr=0.01)
    grad = torch.full((V, d), float("nan"), device=DEV)
    et.et_backward_elastic(b.s, b.dY, [1, 0], [grad, None])
    et.et_update_masked(b.s, [1, 0], [grad, None], 0.01)
    a.check()
    b.check()
    assert torch.equal(a.T, b.T) and all(torch.equal(x, y) for x, y in zip(*states))
    if master:
        assert torch.equal(a.T32, b.T32)
    both = torch.full((V, d), float("nan"), device=DEV)             # exported and applied in one call
    c = Emb(M, V, d, dtype, "zipf", seed=21, master=master)
    c.forward()
    et.et_backward_elastic(c.s, c.dY, [1, 0], [both, None], flags=et.ET_FLAG_FUSE_SGD, lr=0.01)
    c.check()
    assert torch.equal(both, grad)


@pytest.mark.parametrize("dtype", [F, B])
def test_gradient_at_any_address(dtype):
    c = Emb(5000, 300, 64, dtype, "zipf", seed=22)
    c.forward()
    g, tol = c.grad_tol()
    raw = torch.full((300 * 64 + 8,), 7.0, device=DEV)
    for off in (1, 2, 3, 4):
        raw.fill_(7.0)
        view = raw[off:off + 300 * 64]
        et.et_backward_elastic(c.s, c.dY, [1, 0], [view, None])
        c.check()
        assert (np.abs(view.double().cpu().numpy().reshape(300, 64) - g) <= tol).all()
        assert (raw[:off] == 7).all() and (raw[off + 300 * 64:] == 7).all()


def test_host_resident_gradient():
    c = Emb(400, 90, 64, B, "zipf", seed=23)
    c.forward()
    grad, want = torch.empty(90, 64, device=DEV), torch.empty(90, 64, device=DEV)
    et.et_backward_elastic(c.s, c.dY, [1, 0], [want, None])
    host = c.dY.cpu().pin_memory()
    et.et_backward_elastic_host(c.s, host, [1, 0], [grad, None])
    c.check()
    assert torch.equal(grad, want)


@pytest.mark.parametrize("gemm_list", [0, 1])
@pytest.mark.parametrize("sel", [[2, 4, 7], [0, 2, 3, 4, 5, 6, 7], [0], [5]])
def test_dense_layers_above_a_table(gemm_list, sel):
    """Widths the one-launch backward takes: with it and without, the table selected or not, as on the looked-up rows."""
    layers = [wl.embedding_layer(300, 128, 0.5), wl.Layer(128, 256, act=wl.ACT_GELU_TANH), wl.Layer(256, 128, residual_src=1), wl.Layer(128, 320)]
    n = TokenNet(B, M=700, seed=6, layers=layers)
    et.et_stack_set_option(n.s, et.ET_OPTION_GEMM_LIST, gemm_list)
    et.et_forward_stack(n.s, n.x, n.y)
    n.dY.normal_()
    mask = _mask(n.L, sel)
    g1 = [torch.full(p.shape, float("nan"), device=DEV) if m else None for p, m in zip(n.params, mask)]
    et.et_backward_elastic(n.s, n.dY, mask, g1)
    n.check()
    host = n.host(n.params)
    saved = orc.forward(n.layers, host[0::2], host[1::2], n.ids)
    want, _ = orc.backward_masked(n.layers, host[0::2], saved, n.dY.double().cpu().numpy(), mask)
    for t in sel:
        got = g1[t].double().cpu().numpy()
        assert np.abs(got - want[t]).max() <= 3e-2 * np.abs(want[t]).max(), t


def test_tables_beyond_32_bit_offsets():
    V, d, M = 300000, 8200, 4200                       # 2.46e9 elements
    c_ids = np.random.default_rng(1).integers(0, V, M).astype(np.int32)
    c_ids[:3] = [V - 1, 0, V - 1]
    s = et.et_stack_create([(V, d, 0, 1, -1, et.ET_LAYER_EMBEDDING)], M, B)
    T = torch.zeros(V, d, dtype=torch.bfloat16, device=DEV)
    T[V - 1] = 3.0
    ws = torch.empty(et.et_stack_workspace_bytes(s), dtype=torch.uint8, device=DEV)
    et.et_stack_bind(s, [T], [None], ws)
    x = torch.from_numpy(c_ids).to(DEV)
    y = torch.empty(M, d, dtype=torch.bfloat16, device=DEV)
    et.et_forward_stack(s, x, y)
    assert (y[0] == 3).all() and (y[1] == 0).all() and (y[2] == 3).all()
    dY = torch.ones(M, d, dtype=torch.bfloat16, device=DEV)
    grad = torch.full((V, d), float("nan"), device=DEV)
    et.et_backward_elastic(s, dY, [1, 0], [grad, None])
    count = torch.zeros(V, device=DEV).index_add_(0, x.long(), torch.ones(M, device=DEV))
    assert torch.equal(grad.amax(1), count) and torch.equal(grad.amin(1), count)
    before = T[V - 1].clone()
    et.et_backward_elastic(s, dY, [1, 0], flags=et.ET_FLAG_FUSE_SGD, lr=0.5)
    torch.cuda.synchronize()
    k = float(count[V - 1])
    assert (T[V - 1].float() == before.float() - 0.5 * k).all() and (T[0].float() == -0.5 * float(count[0])).all()


def test_two_stacks_at_once():
    """Two stacks, each on a stream of its own, at the same time: what they give one after the other."""
    a, b = Emb(9000, 3000, 264, B, "zipf", seed=31), Emb(3000, 900, 520, F, "zipf", seed=32)
    out = {}
    for c in (a, b):
        c.grad = torch.empty(c.V, c.d, device=DEV)
        c.forward()
        et.et_backward_elastic(c.s, c.dY, [1, 0], [c.grad, None])
        c.check()
        out[c] = c.grad.clone()
        c.grad.fill_(float("nan"))
    streams = {c: torch.cuda.Stream() for c in (a, b)}
    torch.cuda.synchronize()
    for _ in range(10):
        for c in (a, b):
            et.et_forward_stack(c.s, c.x, c.y, stream=streams[c])
            et.et_backward_elastic(c.s, c.dY, [1, 0], [c.grad, None], stream=streams[c])
    torch.cuda.synchronize()
    for c in (a, b):
        c.check()
        assert torch.equal(out[c], c.grad)


@pytest.mark.parametrize("M", [200, 6000])
def test_reported_launches_and_timing(M):
    c = Emb(M, 900, 64, B, "zipf", seed=41)
    c.forward()
    grad = torch.empty(900, 64, device=DEV)
    before, rep = et.et_launch_count(), et.Report(1)
    et.et_backward_elastic(c.s, c.dY, [1, 0], [grad, None], report=rep)
    assert et.et_launch_count() - before == rep.launches > 0 and rep.flops_executed == 0.0
    want = grad.clone()
    et.et_timing_enable(c.s, True)
    et.et_forward_stack(c.s, c.x, c.y)
    et.et_backward_elastic(c.s, c.dY, [1, 0], [grad, None])
    t = et.et_timing_read(c.s)
    et.et_timing_enable(c.s, False)
    c.check()
    assert t["forward"][1] == 1 and t["wgrad"][1] >= 2 and t["wgrad_reduce"][1] == 1 and t["dgrad"][1] == 0
    assert all(ms > 0 for ms, n in t.values() if n) and torch.equal(want, grad)
