"""Token losses, clipping and the table's gradient at the ends of their ranges, through the C ABI.  Expected values are closed forms."""
import math

import numpy as np
import pytest
import torch

import paper_2312_14227_b200 as et

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
E = 2.0 ** -24
F, B = et.ET_F32, et.ET_BF16
INF = float("inf")


def _stack(M, width, dtype):
    s = et.et_stack_create([(8, width, 0, 1, -1)], M, dtype)
    tdt = torch.bfloat16 if dtype == B else torch.float32
    ws = torch.empty(et.et_stack_workspace_bytes(s), dtype=torch.uint8, device=DEV)
    et.et_stack_bind(s, [torch.zeros(8, width, dtype=tdt, device=DEV)], [torch.zeros(width, dtype=tdt, device=DEV)], ws)
    return s, tdt


def _dev(a, dt):
    return torch.tensor(a, dtype=dt, device=DEV)


# widths: rows held by one block, rows read twice
@pytest.mark.parametrize("dtype,width", [(F, 1024), (B, 1024), (B, 300000)])
def test_rejected_token_of_probability_zero(dtype, width):
    """x = inf: the pair's sigmoid loss and gradient are 0 and leave the batch's mean alone."""
    s, tdt = _stack(4, width, dtype)
    y = torch.zeros(4, width, dtype=tdt, device=DEV)     # every token's log probability is -log(width)
    y[1, 2] = -INF                                       # the rejected answer of pair 0
    t, begin = _dev([0, 2, 1, 1], torch.int32), _dev([0, 1, 2, 3, 4], torch.int32)
    for dY in (torch.full_like(y, float("nan")), None):
        stats, seq = torch.full((4,), float("nan"), device=DEV), torch.full((4,), float("nan"), device=DEV)
        et.et_loss_preference_grad(s, y, t, begin, dY, seq_logp=seq, loss_dev=stats, beta=0.5)
        torch.cuda.synchronize()
        # pair 1: x = 0, loss log 2; one rounding of the mean to 32 bits
        assert abs(float(stats[0]) - 0.5 * math.log(2)) <= 2 * E * math.log(2)
        assert float(stats[2]) == -INF and float(stats[3]) == 0.5 and float(seq[1]) == -INF
        if dY is not None:
            assert (dY[:2] == 0).all()
            # c = -1/2 beta / pairs = -1/8: -1/8 (1 - p) at the target; p itself and the product round, then the storage type
            want, half = -0.125 * (1 - 1 / width), torch.finfo(tdt).eps / 2
            assert abs(float(dY[2, 1]) - want) <= (half + 32 * E) * abs(want)
    stats = torch.empty(4, device=DEV)
    et.et_loss_preference_grad(s, y, t, begin, None, loss_dev=stats, beta=0.5, label_smoothing=0.1)
    assert float(stats[0]) == INF                        # with smoothing the loss of that pair is infinite


def _policy(s, y, t, adv, w, old=None, ref=None, **k):
    dY = torch.full_like(y, float("nan"))
    lp, stats = torch.full((len(y),), float("nan"), device=DEV), torch.full((4,), float("nan"), device=DEV)
    f = lambda a: None if a is None else _dev(a, torch.float32)  # noqa: E731
    et.et_loss_policy_grad(s, y, _dev(t, torch.int32), f(adv), dY, weights=f(w), logp_old=f(old), logp_ref=f(ref), logp=lp, loss_dev=stats, **k)
    torch.cuda.synchronize()
    return dY, lp, stats


@pytest.mark.parametrize("gap", [200.0, 1e4, INF])
@pytest.mark.parametrize("rows", [3, 700])               # the sums by the last block, or by a kernel of their own
@pytest.mark.parametrize("dtype,width", [(F, 1024), (B, 1024), (B, 300000)])
def test_divergence_that_is_reported_only(dtype, width, rows, gap):
    """kl_coef = 0: a reference far above the policy, or a taken token of probability 0, leaves loss and gradient alone."""
    if rows == 700 and width == 300000:
        rows = 1100                                      # rows read twice: 1024 and more take the kernel
    s, tdt = _stack(rows, width, dtype)
    y = torch.zeros(rows, width, dtype=tdt, device=DEV)
    y[0, 1] = -gap                                       # the taken token of row 0
    t, old = [1] * rows, [-math.log(width)] * rows
    w = [0.5, 0.5] + [0.0] * (rows - 2)
    for adv in ([1.0, 2.0] + [0.0] * (rows - 2), [-1.0, 2.0] + [0.0] * (rows - 2)):
        dY, lp, stats = _policy(s, y, t, adv, w, old, [-1.0] * rows, kl_coef=0.0)
        # row 0: r = 0; with A < 0 the clipped side counts, 0.8 A: surrogate -0.8 and no slope.  Row 1: r = 1 but for lp's roundings
        first = 0.5 * (0.0 if adv[0] > 0 else 0.8) - 1.0
        tol = 64 * E * (1 + math.log(width))
        assert abs(float(stats[0]) - first) <= tol and float(stats[0]) == float(stats[1])
        assert float(stats[2]) == INF and float(stats[3]) == (0.0 if adv[0] > 0 else 0.5)
        assert float(lp[0]) < -150 and (dY[0] == 0).all()
        want = -1.0 * (1 - 1 / width)
        assert abs(float(dY[1, 1]) - want) <= (torch.finfo(tdt).eps / 2 + tol) * abs(want) and torch.isfinite(dY[1]).all()


@pytest.mark.parametrize("clip_high", [0.2, INF])
@pytest.mark.parametrize("dtype,width", [(F, 1024), (B, 1024), (B, 300000)])
def test_no_advantage_and_a_ratio_beyond_fp32(dtype, width, clip_high):
    """A = 0 takes the row out of the loss, whatever the ratio; any other advantage keeps its row."""
    s, tdt = _stack(3, width, dtype)
    y = torch.zeros(3, width, dtype=tdt, device=DEV)
    lp0 = -math.log(width)
    dY, lp, stats = _policy(s, y, [1, 1, 1], [0.0, 2.0, 0.0], [0.5, 0.5, 0.5], [lp0 - 100, lp0, lp0 - 1e4], clip_high=clip_high)
    tol = 64 * E * (1 + math.log(width))
    assert (dY[0] == 0).all() and (dY[2] == 0).all() and abs(float(stats[0]) + 1.0) <= tol and float(stats[3]) == 0.0
    want = -1.0 * (1 - 1 / width)
    assert abs(float(dY[1, 1]) - want) <= (torch.finfo(tdt).eps / 2 + tol) * abs(want)
    y[0, 0] = float("nan")                               # a row with a NaN still gives NaN
    dY, _, stats = _policy(s, y, [1, 1, 1], [0.0, 2.0, 0.0], [0.5, 0.5, 0.5], [lp0 - 100, lp0, lp0 - 1e4], clip_high=clip_high)
    assert torch.isnan(dY[0]).any() and math.isnan(float(stats[0])) and (dY[2] == 0).all()


def test_elastic_loop_with_a_token_loss_handed_its_buffer():
    """loss_out goes straight to the call that writes four numbers; the losses are those of a buffer of its own."""
    from paper_2312_14227_b200.elastic_loop import ElasticLoop
    out = []
    for own in (False, True):
        s, _ = _stack(6, 64, F)
        g = torch.Generator(device=DEV)
        g.manual_seed(1)
        W, b = [torch.randn(8, 64, generator=g, device=DEV)], [torch.zeros(64, device=DEV)]
        ws = torch.empty(et.et_stack_workspace_bytes(s), dtype=torch.uint8, device=DEV)
        et.et_stack_bind(s, W, b, ws)
        t, adv, spare = _dev([1, 2, 3, 4, 5, 6], torch.int32), torch.randn(6, generator=g, device=DEV), torch.zeros(4, device=DEV)

        def loss(y, dY, loss_out, stream):
            et.et_loss_policy_grad(s, y, t, adv, dY, loss_dev=spare if own else loss_out, stream=stream)
            if own:
                loss_out[:1].copy_(spare[:1])

        x = torch.randn(6, 8, generator=g, device=DEV)
        loop = ElasticLoop(s, W, b, x, None, lr=0.5, period=4, window=2, rho=0.5, t_dw=np.ones(2), t_dy=np.ones(2), loss=loss)
        out.append(loop.run(5, elastic=False)["losses"])
    assert (out[0] == out[1]).all() and np.isfinite(out[0]).all() and (out[0] != 0).any()


@pytest.mark.parametrize("helper", [False, True])
def test_clipping_calls_refuse_gradients_they_would_misread(helper, monkeypatch):
    """A list of bf16 gradients of a bf16 stack is half of what would be read; with the helper module and without it."""
    from paper_2312_14227_b200 import binding
    monkeypatch.setattr(binding, "_helper", [binding._load_helper() if helper else None])
    layers = [(8, 8, 0, 1, -1, et.ET_LAYER_NORM, 1e-5), (8, 16, 0, 1, -1)]
    s = et.et_stack_create(layers, 4, B)
    shapes = [(8,), (8,), (8, 16), (16,)]
    params = [torch.zeros(n, dtype=torch.bfloat16, device=DEV) for n in shapes]
    ws = torch.empty(et.et_stack_workspace_bytes(s), dtype=torch.uint8, device=DEV)
    et.et_stack_bind(s, params[0::2], params[1::2], ws)
    g, norm = [torch.full(n, 2.0, device=DEV) for n in shapes], torch.zeros(2, device=DEV)
    bad = [(2, g[2].bfloat16(), et.ET_ERR_DTYPE), (2, torch.zeros(16, 8, device=DEV).t(), et.ET_ERR_INVALID_ARG),
           (3, torch.zeros(15, device=DEV), et.ET_ERR_INVALID_ARG), (1, torch.zeros(1, device=DEV).expand(8), et.ET_ERR_INVALID_ARG),
           (0, torch.zeros(8), et.ET_ERR_INVALID_ARG), (3, None, et.ET_ERR_INVALID_ARG)]
    for i, t, status in bad:
        lst = [t if i == j else u for j, u in enumerate(g)]
        for call in (lambda: et.et_grad_norm(s, [1] * 4, lst, norm), lambda: et.et_clip_grads(s, [1] * 4, g, lst, 1.0),
                     lambda: et.et_clip_grads(s, [1] * 4, lst, g, 1.0), lambda: et.et_update_clipped(s, [1] * 4, lst, 0.1, 1.0)):
            with pytest.raises(et.EtError) as e:
                call()
            assert e.value.status == status, (i, status)
        mask = [int(i != j) for j in range(4)]           # not selected: ignored, whatever it is
        et.et_grad_norm(s, mask, lst, norm)
        assert float(norm[0]) == np.float32(math.sqrt(4.0 * sum(math.prod(n) for n, m in zip(shapes, mask) if m)))
    et.et_clip_grads(s, [1] * 4, g, g, 1.0, norm)
    n = math.sqrt(4.0 * 160)
    assert float(norm[0]) == np.float32(n) and all(((u - 2 / n).abs() <= 4 * E / n * 2).all() for u in g)
    by_address = [u.data_ptr() for u in g]
    et.et_grad_norm(s, [1] * 4, by_address, norm.data_ptr())
    assert abs(float(norm[0]) - 1.0) <= 8 * E


@pytest.mark.parametrize("dtype,width", [(F, 1), (F, 100), (F, 8200), (B, 8), (B, 264), (B, 8200), (F, 140003), (B, 300000)])
@pytest.mark.parametrize("call", ["logp", "policy"])
def test_rows_with_all_their_mass_on_one_token(dtype, width, call):
    """p = 1 to within e^-80: the log probability is 0, to the last bit."""
    M = 600 if width < 20000 else 5
    s, tdt = _stack(M, width, dtype)
    y = torch.full((M, width), -100.0, dtype=tdt, device=DEV)
    t = torch.randint(0, width, (M,), device=DEV, dtype=torch.int32)
    y[torch.arange(M, device=DEV), t.long()] = 3.0
    lp = torch.full((M,), float("nan"), device=DEV)
    if call == "logp":
        et.et_token_logp(s, y, t, lp)
    else:
        et.et_loss_policy_grad(s, y, t, torch.ones(M, device=DEV), None, logp=lp)
    assert (lp == 0).all()


# logit scales: 1, and one whose product with log2(e) is far from an fp32 number (1e-7 of it)
@pytest.mark.parametrize("scale", [1.0, 0.9])
@pytest.mark.parametrize("dtype", [F, B])
@pytest.mark.parametrize("low,high", [(0.9, 1.0), (0.3, 0.9), (1e-4, 0.05)])
@pytest.mark.parametrize("call", ["logp", "policy"])
def test_errors_of_log_probabilities_have_no_sign(dtype, low, high, call, scale):
    """The mean error over many rows: a log probability is added up over sequences, where errors of one sign do not cancel."""
    M, width, scale = 32768, 264, float(np.float32(scale))
    s, tdt = _stack(M, width, dtype)
    g = torch.Generator(device=DEV)
    g.manual_seed(3)
    y = torch.randn(M, width, generator=g, device=DEV)
    t = torch.randint(0, width, (M,), generator=g, device=DEV, dtype=torch.int32)
    at = torch.arange(M, device=DEV)
    p = low + (high - low) * torch.rand(M, generator=g, device=DEV).double()
    y[at, t.long()] = -float("inf")
    y[at, t.long()] = ((torch.logsumexp(scale * y.double(), 1) + torch.log(p / (1 - p))) / scale).float()      # the wanted share
    y = y.to(tdt)
    lp = torch.empty(M, device=DEV)
    if call == "logp":
        et.et_token_logp(s, y, t, lp, logit_scale=scale)
    else:
        et.et_loss_policy_grad(s, y, t, torch.ones(M, device=DEV), None, logp=lp, logit_scale=scale)
    z = scale * y.double()
    total = torch.logsumexp(z, 1)
    want = z[at, t.long()] - total
    err = lp.double() - want
    # Roundings to nearest have no sign: of the sum (about 16 of them at e of it, independent), of lp itself (e |lp|): six standard
    # deviations of their mean over M rows.  A term passes up to three exponentials (its own, the lanes' join, the warps' join); the
    # unit's mean error is within 0.2e-8 of what is taken off, but 2.2e-8 for exponents in [-1, 0].  The largest term is exact.
    spread = E * (4 + float(want.abs().max())) / math.sqrt(3)
    share = float((1 - torch.exp(z.amax(1) - total)).mean())
    assert abs(float(err.mean())) <= 6 * spread / math.sqrt(M) + 3 * 2.2e-8 * share, (float(err.mean()), share)


@pytest.mark.parametrize("scale", [1e-30, 1e-33, 1e-35, 1.5e-38, 3e-38])
def test_logit_scales_near_the_end_of_fp32(scale):
    """Logits of 1e30 and more under a scale that brings them back to ordinary ones, down to where d scale leaves fp32."""
    scale = float(np.float32(scale))
    M, width = 9, 1000
    s, _ = _stack(M, width, F)
    g = torch.Generator(device=DEV)
    g.manual_seed(2)
    y = torch.randn(M, width, generator=g, device=DEV) * min(2 / scale, 5e37)
    y[1, 3] = -INF
    y[2, 5:] = -INF
    t = torch.randint(0, 5, (M,), generator=g, device=DEV, dtype=torch.int32)
    lp = torch.empty(M, device=DEV)
    et.et_token_logp(s, y, t, lp, logit_scale=scale)
    z = scale * y.double()
    want = z[torch.arange(M, device=DEV), t.long()] - torch.logsumexp(z, 1)
    # exponents up to 20: e (3 x 20 + 4 + a few levels of the sum) and lp's own rounding; scale log2(e) is good to 2^-24 of itself and the
    # smallest number
    tol = E * (64 + 40 + 2 * want.abs()) + 20 * 1.5e-45 / scale
    assert ((lp.double() - want).abs() <= tol).all(), (lp, want)


@pytest.mark.parametrize("value,max_norm", [(1e30, 1e-9), (1e35, 1e-4), (3e38, 1e-3), (3e38, 1e-8), (1e38, 1e-38), (1e-38, 1e-44)])
def test_factors_below_fp32(value, max_norm):
    """max_norm / norm below fp32's normal numbers (and below all of them): the clipped gradients are ordinary numbers."""
    d = 64
    s = et.et_stack_create([(d, d, 0, 1, -1)], 8, F)
    W, b = torch.zeros(d, d, device=DEV), torch.zeros(d, device=DEV)
    ws = torch.empty(et.et_stack_workspace_bytes(s), dtype=torch.uint8, device=DEV)
    et.et_stack_bind(s, [W], [b], ws)
    gen = torch.Generator(device=DEV)
    gen.manual_seed(4)
    g = [torch.rand(d, d, generator=gen, device=DEV) * value, torch.rand(d, generator=gen, device=DEV) * value]
    out, norm = [torch.full_like(x, float("nan")) for x in g], torch.empty(2, device=DEV)
    n = math.sqrt(sum(float((x.double() ** 2).sum()) for x in g))
    mx = float(np.float32(max_norm))
    et.et_clip_grads(s, [1, 1], g, out, mx, norm)
    assert (float(norm[0]) == INF) if n > 3.41e38 else abs(float(norm[0]) - n) <= 2 * E * n
    assert float(norm[1]) > 0 and abs(float(norm[1]) - mx / n) <= E * mx / n + 1.5e-45
    for x, o in zip(g, out):
        want = x.double() * (mx / n)                     # the factor and two products round; results below 2^-126 to the step there
        assert ((o.double() - want).abs() <= 4 * E * want + 2.9e-45).all()
    et.et_update_clipped(s, [1, 1], g, -1.0, mx)         # W <- W + clipped
    assert torch.equal(W, out[0]) and torch.equal(b, out[1])
    # Adam's state moves too: a finite norm is a step
    st = [[torch.ones_like(W), torch.ones_like(b)], [torch.ones_like(W), torch.ones_like(b)]]
    et.et_stack_set_optimizer(s, et.ET_OPT_ADAM, st[0], st[1])
    et.et_update_clipped(s, [1, 1], g, 0.0, mx)
    assert all((x != 1).all() for x in st[0] + st[1])


@pytest.mark.parametrize("dtype,d", [(F, 512), (B, 512), (F, 510)])
def test_cost_of_a_table_counts_every_row(dtype, d):
    """The profiled time of a table's gradient is that of writing all of it, tables beyond the scratch included; nothing else changes."""
    M, tdt = 64, torch.bfloat16 if dtype == B else torch.float32
    for V in (1000, 100000, 400000):
        et.et_debug_guard_regions(True)
        s = et.et_stack_create([(V, d, 0, 1, -1, et.ET_LAYER_EMBEDDING)], M, dtype)
        et.et_debug_guard_regions(False)
        T = torch.full((V, d), 0.5, dtype=tdt, device=DEV)
        ws = torch.empty(et.et_stack_workspace_bytes(s), dtype=torch.uint8, device=DEV)
        et.et_stack_bind(s, [T], [None], ws)
        x = torch.arange(M, device=DEV, dtype=torch.int32) * 7 % V
        y, dY = torch.empty(M, d, dtype=tdt, device=DEV), torch.ones(M, d, dtype=tdt, device=DEV)
        t_dw, t_dy, _ = et.et_profile_costs(s, x, y, dY, 5)
        # the device's memory takes 8 TB/s at the most; what stays in L2 (126 MB) need not have reached it yet
        assert t_dw[0] * 1e-3 >= (V * d * 4 - 140e6) / 8e12 and t_dw[1] == 0 and t_dy[0] == 0 and t_dy[1] == 0
        st, bad = et.et_debug_check_guards(s)
        assert st == et.ET_OK, bad
        assert (T == 0.5).all() and (y == 0.5).all()
        grad = torch.full((V, d), float("nan"), device=DEV)
        et.et_backward_elastic(s, dY, [1, 0], [grad, None])
        want = torch.zeros(V, device=DEV).index_add_(0, x.long(), torch.ones(M, device=DEV))
        assert torch.equal(grad, want[:, None].expand(V, d))


def _above_a_table(kind):
    import workloads as wl
    if kind == "attention":
        return B, 120, [wl.embedding_layer(50, 384, 2.0), wl.attention_layer(128, 2, 40), wl.Layer(128, 72)]
    if kind == "gather":                                 # the gathered matrix is formed
        return F, 60, [wl.embedding_layer(50, 8, 2.0)] + wl.conv_layers(8, 24, 5, 6) + [wl.Layer(24, 16)]
    if kind == "convolution":                            # the convolution's GEMMs fetch the patches themselves
        return B, 144, [wl.embedding_layer(50, 128, 2.0)] + wl.conv_layers(128, 64, 6, 12) + [wl.Layer(64, 72)]
    return B, 150, [wl.embedding_layer(50, 64, 2.0), wl.batchnorm_layer(64, act=wl.ACT_RELU), wl.Layer(64, 72)]


@pytest.mark.parametrize("kind", ["attention", "gather", "convolution", "batchnorm"])
def test_layers_without_tensors_directly_above_a_table(kind):
    """The table's gradient through them; and their backward time is charged to a selection of the table."""
    import workloads as wl
    from oracle import elastic_oracle as orc
    dtype, M, layers = _above_a_table(kind)
    tdt = torch.bfloat16 if dtype == B else torch.float32
    rng, L = np.random.default_rng(6), len(layers)
    W, b = [], []
    for ly in layers:
        k = ly.kind
        if k in (wl.KIND_ATTENTION, wl.KIND_IM2COL):
            w_, b_ = np.zeros(0), np.zeros(0)
        elif k == wl.KIND_EMBEDDING:
            w_, b_ = rng.normal(size=(ly.in_features, ly.out_features)) * 0.4, np.zeros(0)
        elif k == wl.KIND_BATCHNORM:
            w_, b_ = 1 + 0.1 * rng.normal(size=ly.out_features), 0.3 * rng.normal(size=ly.out_features)
        else:
            w_, b_ = rng.normal(size=(ly.in_features, ly.out_features)) / np.sqrt(ly.in_features), 0.1 * rng.normal(size=ly.out_features)
        W.append(torch.from_numpy(w_).to(tdt).to(DEV))
        b.append(torch.from_numpy(b_).to(tdt).to(DEV))
    s = et.et_stack_create(layers, M, dtype)
    ws = torch.empty(et.et_stack_workspace_bytes(s), dtype=torch.uint8, device=DEV)
    et.et_stack_bind(s, W, b, ws)
    et.et_stack_set_embedding_scale(s, 2.0)
    ids = rng.integers(0, 50, M).astype(np.int32)
    x = torch.from_numpy(ids).to(DEV)
    y = torch.empty(M, layers[-1].out_width, dtype=tdt, device=DEV)
    dY = torch.from_numpy(rng.normal(size=y.shape)).to(tdt).to(DEV)
    et.et_forward_stack(s, x, y)
    mask = np.zeros(2 * L, dtype=np.uint8)
    mask[0] = mask[-1] = 1
    grads = [None] * (2 * L)
    grads[0], grads[-1] = torch.full(W[0].shape, float("nan"), device=DEV), torch.full(b[-1].shape, float("nan"), device=DEV)
    et.et_backward_elastic(s, dY, mask, grads)
    torch.cuda.synchronize()
    assert et.et_device_status(s) == et.ET_OK
    host = lambda ts: [t.double().cpu().numpy() for t in ts]  # noqa: E731
    saved = orc.forward(layers, host(W), host(b), ids)
    want, _ = orc.backward_masked(layers, host(W), saved, dY.double().cpu().numpy(), mask)
    rel = lambda a, o: np.abs(a.double().cpu().numpy() - o).max() / np.abs(o).max()  # noqa: E731
    tol = 3e-2 if dtype == B else 1e-4                   # the bars of the other whole-stack tests
    assert rel(y, saved.a[-1]) <= tol and rel(grads[0], want[0]) <= tol and rel(grads[-1], want[2 * L - 1]) <= tol
    t_dw, t_dy, _ = et.et_profile_costs(s, x, y, dY, 3)
    assert t_dw[0] > 0 and t_dy[0] == 0 and t_dw[1] == 0
    if kind in ("attention", "gather"):
        only = np.zeros(2 * L, dtype=np.uint8)
        only[0] = 1
        assert t_dy[1] > 0                               # charged: a strict selection pays t_dy of everything above its deepest tensor
        assert et.et_time_selective(only, t_dw, t_dy) >= t_dw[0] + t_dy[1]
    else:
        assert t_dy[1] == 0


@pytest.mark.parametrize("dtype", [F, B])
@pytest.mark.parametrize("loss", ["policy", "preference"])
def test_whole_step_captured_and_replayed(dtype, loss):
    """Lookup, layers, token loss, masked backward and clipped update in one graph: the eager steps, bit for bit, on new ids each time."""
    import workloads as wl
    M, V, OUT = 600, 300, 264
    layers = [wl.embedding_layer(V, 128, 0.5), wl.Layer(128, 256, act=wl.ACT_GELU_TANH), wl.Layer(256, 128, residual_src=1), wl.Layer(128, OUT)]
    tdt = torch.bfloat16 if dtype == B else torch.float32
    gen = torch.Generator(device=DEV)
    gen.manual_seed(8)
    W0 = [torch.randn(V if ly.kind == wl.KIND_EMBEDDING else ly.in_features, ly.out_features, generator=gen, device=DEV) / math.sqrt(ly.in_features)
          for ly in layers]
    b0 = [torch.zeros(0 if ly.kind == wl.KIND_EMBEDDING else ly.out_features, device=DEV) for ly in layers]
    batches = [torch.randint(-1, V + 1, (M,), generator=gen, device=DEV, dtype=torch.int32) for _ in range(4)]
    t = torch.randint(0, OUT, (M,), generator=gen, device=DEV, dtype=torch.int32)
    adv, begin = torch.randn(M, generator=gen, device=DEV), _dev([0, 100, 250, 400, 590], torch.int32)
    mask = np.array([1, 0, 1, 1, 0, 1, 1, 1], dtype=np.uint8)
    results = []
    for captured in (False, True):
        s = et.et_stack_create(layers, M, dtype)
        W, b = [w.clone().to(tdt) for w in W0], [v.clone().to(tdt) for v in b0]
        ws = torch.empty(et.et_stack_workspace_bytes(s), dtype=torch.uint8, device=DEV)
        et.et_stack_bind(s, W, b, ws)
        et.et_stack_set_embedding_scale(s, 0.5)
        params = [p for pair in zip(W, b) for p in pair]
        st = [[torch.zeros(p.shape, device=DEV) for p in params] for _ in range(2)]
        et.et_stack_set_optimizer(s, et.ET_OPT_ADAM, st[0], st[1])
        et.et_stack_set_optimizer_step(s, 1)
        x, y = batches[0].clone(), torch.empty(M, OUT, dtype=tdt, device=DEV)
        dY, stats, norm = torch.empty_like(y), torch.zeros(4, device=DEV), torch.zeros(2, device=DEV)
        grads = [torch.zeros(p.shape, device=DEV) if m else None for p, m in zip(params, mask)]

        def step(stream):
            et.et_forward_stack(s, x, y, stream=stream)
            if loss == "policy":
                et.et_loss_policy_grad(s, y, t, adv, dY, loss_dev=stats, stream=stream)
            else:
                et.et_loss_preference_grad(s, y, t, begin, dY, loss_dev=stats, stream=stream)
            et.et_backward_elastic(s, dY, mask, grads, stream=stream)
            et.et_update_clipped(s, mask, grads, 0.01, 1e-3, norm, stream=stream)

        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        seen, graph = [], None
        for i, ids in enumerate(batches):
            torch.cuda.synchronize()
            x.copy_(ids)
            torch.cuda.synchronize()
            if i == 0 or not captured:
                step(side)
            else:
                if graph is None:
                    graph = torch.cuda.CUDAGraph()
                    with torch.cuda.graph(graph, stream=side):
                        step(side)
                graph.replay()
            torch.cuda.synchronize()
            seen += [stats.clone(), norm.clone(), y.clone()]
        assert et.et_device_status(s) == et.ET_OK
        results.append(seen + [p.clone() for p in params] + [v for ts in st for v in ts])
        del graph
    assert all(torch.equal(a, c) for a, c in zip(*results))
    assert not torch.equal(results[0][2], results[0][5])             # the batches differ


@pytest.mark.parametrize("value", [0x7fffffff, 0x80000000, 0xfffffff0, 5000])
def test_a_foreign_row_counter_leads_to_no_row_outside(value):
    """The counter that hands out rows, overwritten by something else: no row outside the logits is read or written, and binding
    again puts it right."""
    M, width = 1000, 32008
    s, tdt = _stack(M, width, B)
    ws, W, b = torch.empty(et.et_stack_workspace_bytes(s), dtype=torch.uint8, device=DEV), s._keep[0], s._keep[1]
    et.et_stack_bind(s, W, b, ws)
    g = torch.Generator(device=DEV)
    g.manual_seed(7)
    room = torch.full((M + 4, width), 7.0, dtype=tdt, device=DEV)
    dY = room[2:M + 2]
    y = torch.randn(M, width, generator=g, device=DEV).to(tdt)
    t, adv = torch.randint(0, width, (M,), generator=g, device=DEV, dtype=torch.int32), torch.ones(M, device=DEV)
    want = torch.empty_like(y)
    et.et_loss_policy_grad(s, y, t, adv, want)
    torch.cuda.synchronize()
    word = ws[33 * 4:34 * 4].view(torch.int32)           # the status region's word 33
    assert int(word[0]) == 0
    word.fill_(value - (1 << 32) if value >= 1 << 31 else value)
    et.et_loss_policy_grad(s, y, t, adv, dY)
    torch.cuda.synchronize()
    assert (room[:2] == 7).all() and (room[-2:] == 7).all()
    done = (dY == want).all(1) | (dY == 7.0).all(1)
    assert done.all() and (dY[0] == want[0]).all()       # each row is right or was not come to
    et.et_stack_bind(s, W, b, ws)
    et.et_loss_policy_grad(s, y, t, adv, dY)
    torch.cuda.synchronize()
    assert torch.equal(dY, want)


@pytest.mark.parametrize("opt", ["sgd", "adam"])
def test_elastic_schedule_of_a_table_with_masters_and_clipping(opt):
    """Token ids, fp32 masters of bf16 tensors, clipped updates and re-selection together: the stored tensors stay the rounded masters,
    tensors that a step does not select stay as they are."""
    import workloads as wl
    from paper_2312_14227_b200.elastic_loop import ElasticLoop
    M, V, D, OUT = 96, 61, 48, 72
    layers = [wl.embedding_layer(V, D, 1.5), wl.Layer(D, 80, act=wl.ACT_GELU_TANH), wl.Layer(80, OUT)]
    g = torch.Generator(device=DEV)
    g.manual_seed(5)
    W = [(torch.randn(ly.in_features, ly.out_features, generator=g, device=DEV) * 0.2).bfloat16() for ly in layers]
    b = [torch.zeros(0 if ly.kind == wl.KIND_EMBEDDING else ly.out_features, dtype=torch.bfloat16, device=DEV) for ly in layers]
    s = et.et_stack_create(layers, M, B)
    ws = torch.empty(et.et_stack_workspace_bytes(s), dtype=torch.uint8, device=DEV)
    et.et_stack_bind(s, W, b, ws)
    et.et_stack_set_embedding_scale(s, 1.5)
    params = [p for pair in zip(W, b) for p in pair]
    st = [[torch.zeros(p.shape, device=DEV) for p in params] for _ in range(2)]
    ids = torch.randint(0, V, (M,), generator=g, device=DEV, dtype=torch.int32)
    t, adv = torch.randint(0, OUT, (M,), generator=g, device=DEV, dtype=torch.int32), torch.randn(M, generator=g, device=DEV)
    loss = lambda y, dY, out, stream: et.et_loss_policy_grad(s, y, t, adv, dY, loss_dev=out, stream=stream)  # noqa: E731
    loop = ElasticLoop(s, W, b, ids, None, lr=0.05, period=6, window=2, rho=0.4, t_dw=np.ones(6), t_dy=np.ones(6), master=True,
                       loss=loss, max_norm=0.01)
    if opt == "adam":
        et.et_stack_set_optimizer(s, et.ET_OPT_ADAM, st[0], st[1])
        et.et_stack_set_optimizer_step(s, 1)
    first = [p.clone() for p in params]
    out = loop.run(2)
    assert out["masks"][0].tolist() == [1, 0, 1, 1, 1, 1] and len(out["importances"]) == 1
    assert all(not torch.equal(p, q) for p, q, m in zip(params, first, out["masks"][0]) if m)
    loop.mask = np.array([0, 0, 0, 0, 1, 1], dtype=np.uint8)
    before = [p.clone() for p in loop.master]
    out = loop.run(1, elastic=False)
    assert out["masks"][0].tolist() == [0, 0, 0, 0, 1, 1] and np.isfinite(out["losses"]).all()
    for i, (p, m, q) in enumerate(zip(params, loop.master, before)):
        assert torch.equal(p, m.bfloat16()) and torch.equal(m, q) == (i < 4)
