"""The decoder block's layers at the ends of their ranges."""
import numpy as np
import pytest
import torch

import paper_2312_14227_b200 as et
from oracle import block_oracle as blk
from paper_2312_14227_b200.elastic_loop import ElasticLoop
from test_gpu_block_layers import DEV, TDT, B, F, Run, desc, dev, f64, seed_of, within
from test_gpu_seq_attention import Attn

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------------------ caps
@pytest.mark.parametrize("cap", [0.01, 1.0, 1e3, 1e5, 1e6, 1e9, 1e30])
@pytest.mark.parametrize("dim", [64, 128])
def test_caps_of_any_size(dim, cap):
    """A cap far above the scores changes nothing, one far below leaves their signs: an error of the cap's tanh is one of the score itself,
    not of the cap."""
    Attn(270, 2, 1, dim, seqs=[0, 133, 262], cap=cap, std=2.0, seed=3).check()
    Attn(270, 2, 1, dim, causal=False, cap=cap, slopes=[0.05, 0.5], std=2.0, seed=4).check()


def test_a_capped_key_that_is_not_a_number_is_seen():
    """Rows that see it have no score for it: their output is NaN, as it is without a cap."""
    for cap in (0.0, 20.0):
        for dim in (64, 128):
            for key in (5, 6):
                a = Attn(150, 1, 1, dim, cap=cap)
                a.x[key, dim:2 * dim] = float("nan")
                y, _ = a.run()
                assert bool(torch.isnan(y[key:]).all()), (cap, dim, key)


# ------------------------------------------------------------------------------------------ many rows and heads
def check_heads(a, groups):
    """Output and gradient of the given key heads' groups against the oracle."""
    y, dX = a.run()
    see = blk.visible(a.M, a.seqs, a.causal, a.prefix)
    g, dim = a.heads // a.kv, a.dim
    x, dY = f64(a.x).reshape(a.M, -1, dim), f64(a.dY).reshape(a.M, -1, dim)
    q = [h for n in groups for h in range(n * g, n * g + g)]
    cols = q + [a.heads + n for n in groups] + [a.heads + a.kv + n for n in groups]
    flat = lambda t: np.ascontiguousarray(t).reshape(a.M, -1)  # noqa: E731
    o, oe, d, de = blk.attention(flat(x[:, cols]), len(q), len(groups), dim, see, a.scale, a.cap,
                                 None if a.slopes is None else [a.slopes[h] for h in q], flat(dY[:, q]))
    within("y", y.reshape(a.M, -1, dim)[:, q].reshape(a.M, -1), o, oe)
    within("dX", dX.reshape(a.M, -1, dim)[:, cols].reshape(a.M, -1), d, de)


LONG = [0, 333, 340, 900, 1090]                          # lengths above and below a block, one of few keys; rows of no sequence behind
FORMS = {"causal": dict(), "none": dict(causal=False), "capped-prefix": dict(cap=30.0, prefix=[0, 3, 200, 1000]),
         "bias": dict(causal=False, bias=True), "capped-bias": dict(cap=20.0, bias=True)}


@pytest.mark.parametrize("dim", [40, 64, 128])
@pytest.mark.parametrize("form", sorted(FORMS))
def test_blocks_of_two_halves(form, dim):
    """30 heads over 1100 rows: 150 forward blocks of two halves, D in a launch of its own, clusters of two (dq) and four (dk, dv)."""
    k = dict(FORMS[form])
    slopes = [0.02 * (h + 1) for h in range(30)] if k.pop("bias", False) else None
    check_heads(Attn(1100, 30, 15, dim, seqs=LONG, slopes=slopes, std=1.5, seed=dim, **k), [0, 14])


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("form", ["causal", "capped-bias"])
def test_blocks_that_share_no_item(form, dim):
    """64 heads, each with its own key head: a block an item in every pass."""
    k = dict(FORMS[form])
    slopes = [0.01 * (h + 1) for h in range(64)] if k.pop("bias", False) else None
    check_heads(Attn(1100, 64, 64, dim, seqs=LONG, slopes=slopes, seed=dim, **k), [0, 31, 63])


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("form", sorted(FORMS))
def test_clusters_of_eight(form, dim):
    """Four heads over 2000 rows: eight blocks join an item's sums in both passes of the gradient."""
    k = dict(FORMS[form])
    slopes = [0.02, 0.3, -0.01, 0.0] if k.pop("bias", False) else None
    check_heads(Attn(2000, 4, 2, dim, seqs=[0, 1200, 1210, 1700, 1990], slopes=slopes, std=1.5, seed=dim, **k), [0, 1])


def test_clusters_of_eight_behind_a_launch_for_the_dots():
    """20 heads that share two key heads: D by itself, eight blocks a key tile."""
    check_heads(Attn(2000, 20, 2, 64, seqs=[0, 1200, 1210, 1700, 1990], seed=1), [1])


# ------------------------------------------------------------------------------------------ millions of rows
def test_dense_fp32_layer_of_millions_of_rows():
    """Whole numbers that every format holds, so that results are exact whatever the order of the sums."""
    rng = np.random.default_rng(1)
    M, K, N = 4_194_305, 8, 16
    W, b = dev(rng.integers(-1, 2, (K, N)), F), dev(rng.integers(-2, 3, N), F)
    x = torch.randint(-1, 2, (M, K), device=DEV).to(TDT[F])
    r = Run([desc(et.ET_LAYER_DENSE, K, N, act=et.ET_ACT_RELU)], M, F, [W], [b], x=x)
    r.dY = torch.randint(-1, 2, (M, N), device=DEV).to(TDT[F])
    grads = [torch.full((K, N), float("nan"), device=DEV), torch.full((N,), float("nan"), device=DEV)]
    y, dX = r([1, 1], grads)
    z = (x.double() @ W.double() + b.double()).float()
    assert torch.equal(y, z.clamp(min=0))
    dz = r.dY * (z > 0)
    assert torch.equal(dX, (dz.double() @ W.double().T).float())
    assert torch.equal(grads[1].double(), dz.double().sum(0))
    assert torch.equal(grads[0].double(), x.double().T @ dz.double())


@pytest.mark.parametrize("dtype,M", [(B, 2_097_153), (F, 2_097_153), (F, 4_194_305)])
def test_gated_layer_of_millions_of_rows(dtype, M):
    """Whole numbers that every format holds, so that results are exact whatever the order of the sums."""
    rng = np.random.default_rng(M)
    K = h = 8
    W, b = dev(rng.integers(-1, 2, (K, 2 * h)), dtype), dev(rng.integers(-2, 3, 2 * h), dtype)
    x = torch.randint(-1, 2, (M, K), device=DEV).to(TDT[dtype])
    r = Run([desc(et.ET_LAYER_GATED, K, 2 * h, fold=2, act=et.ET_ACT_RELU)], M, dtype, [W], [b], x=x)
    r.dY = torch.randint(-1, 2, (M, h), device=DEV).to(TDT[dtype])
    grads = [torch.full((K, 2 * h), float("nan"), device=DEV), torch.full((2 * h,), float("nan"), device=DEV)]
    y, dX = r([1, 1], grads)
    z = x.float() @ W.float() + b.float()                # at most 10
    zg, zu, g = z[:, :h], z[:, h:], r.dY.float()
    assert torch.equal(y.float(), zg.clamp(min=0) * zu)
    dz = torch.cat([g * zu * (zg > 0), g * zg.clamp(min=0)], 1)
    assert torch.equal(dX.float(), dz @ W.float().T)     # at most 160
    assert torch.equal(grads[1].double(), dz.double().sum(0))
    assert torch.equal(grads[0].double(), x.double().T @ dz.double())


# ------------------------------------------------------------------------------------------ gates near 0
@pytest.mark.parametrize("above", [False, True])
def test_gates_near_zero(above):
    """Z is kept in steps of 2^-24 below 2^-14; a positive ReLU gate stays positive, so that its slope stays 1."""
    tiny = [2.0 ** -e for e in (14, 20, 24, 25, 26, 40, 100, 126)]
    W, b = torch.zeros(8, 16, dtype=torch.bfloat16, device=DEV), dev([0] * 8 + [1] * 8, B)
    W[:, :8] = torch.eye(8, device=DEV)
    x = dev([tiny, [-t for t in tiny], [0] * 8, [1] * 8], B)
    layers, w, c = [desc(et.ET_LAYER_GATED, 8, 16, fold=2, act=et.ET_ACT_RELU)], [W], [b]
    if above:
        layers.append(desc(et.ET_LAYER_DENSE, 8, 8))
        w.append(torch.eye(8, device=DEV).to(torch.bfloat16))
        c.append(dev([0] * 8, B))
    r = Run(layers, 4, B, w, c, x=x)
    g = torch.full((16,), float("nan"), device=DEV)
    y, dX = r([0, 1] + [0, 0] * above, [None, g] + [None, None] * above)
    z, dy = f64(x), f64(r.dY)
    assert np.array_equal(f64(y), np.maximum(z, 0))
    assert np.array_equal(f64(dX), dy * (z > 0))
    within("db", g[:8], (dy * (z > 0)).sum(0), 8 * blk.E * np.abs(dy).sum(0))
    within("db", g[8:], (dy * np.maximum(z, 0)).sum(0), (np.abs(dy) * (2.0 ** -24 + blk.U * np.abs(z))).sum(0))


# ------------------------------------------------------------------------------------------ dropout in the training loop
def loop_of(dropout_seed):
    rng = np.random.default_rng(8)
    layers = [desc(et.ET_LAYER_DENSE, 24, 40, act=1), desc(et.ET_LAYER_DROPOUT, 40, 40, drop=0.3), desc(et.ET_LAYER_DENSE, 40, 16)]
    W = [dev(rng.normal(size=(24, 40)) / 5, F), torch.zeros(0, device=DEV), dev(rng.normal(size=(40, 16)) / 6, F)]
    b = [dev(np.zeros(40), F), torch.zeros(0, device=DEV), dev(np.zeros(16), F)]
    s = et.et_stack_create(layers, 50, F)
    ws = torch.empty(et.et_stack_workspace_bytes(s), dtype=torch.uint8, device=DEV)
    et.et_stack_bind(s, W, b, ws)
    x, target = dev(rng.normal(size=(50, 24)), F), dev(rng.normal(size=(50, 16)), F)
    t = np.ones(6)
    t[2:4] = 0
    loop = ElasticLoop(s, W, b, x, target, 0.05, 4, 2, 0.6, t, t, dropout_seed=dropout_seed)
    loop.keep = ws
    return loop


def test_every_step_of_the_loop_drops_other_elements():
    """Step i of a loop with a seed is a step with {seed, i}, the same in its forward and its backward pass, over calls of run; behind run
    nothing is dropped."""
    loop, hand = loop_of(2 ** 64 - 5), loop_of(None)
    got = np.concatenate([loop.run(3, elastic=False)["losses"], loop.run(4, elastic=False)["losses"]])
    losses = torch.zeros(7, device=DEV)
    for i in range(7):
        et.et_stack_set_dropout_seed(hand.stack, seed_of(2 ** 64 - 5, i))
        et.et_forward_stack(hand.stack, hand.x, hand.y)
        et.et_loss_mse_grad(hand.stack, hand.y, hand.target, hand.dY, losses[i:])
        et.et_backward_elastic(hand.stack, hand.dY, hand.all_mask, flags=et.ET_FLAG_FUSE_SGD, lr=0.05)
        torch.cuda.synchronize()
    assert np.array_equal(got, losses.cpu().numpy().astype(np.float64))
    for p, q in zip(loop.params, hand.params):
        assert torch.equal(p, q)
    ys = []
    for seed in (False, True):
        if seed:
            et.et_stack_set_dropout_seed(loop.stack, None)
        et.et_forward_stack(loop.stack, loop.x, loop.y)
        ys.append(loop.y.clone())
    assert torch.equal(*ys)
    assert np.isfinite(loop_of(1).run(9)["losses"]).all()


@pytest.mark.parametrize("handle", [False, True])
def test_a_loop_on_another_stream_reads_what_that_stream_wrote(handle):
    """Snapshots, importances and losses are ordered with the steps, however late the stream is."""
    loop, other = loop_of(3), loop_of(3)
    want = loop.run(5)
    side = torch.cuda.Stream()
    other.stream = side.cuda_stream if handle else side
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(200_000_000)                   # about 0.1 s
    got = other.run(5)
    assert np.array_equal(got["losses"], want["losses"])
    assert np.array_equal(got["importances"], want["importances"]) and np.array_equal(got["masks"], want["masks"])
    for p, q in zip(loop.params, other.params):          # on the current stream: run's work comes before it
        assert torch.equal(p, q)
