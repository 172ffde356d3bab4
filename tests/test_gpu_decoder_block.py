"""Decoder blocks as they are used: token ids to logits through norm, projections, rotary positions, masked attention, dropout with the
residual and the gated feed-forward layer, a token loss, the masked backward pass and a clipped update, against float64 autograd of the same
formulas.

The bar is that of the other bf16 stacks: each tensor's largest error within 2e-2 of its largest entry (storage rounding of a dozen
chained bf16 layers)."""
import math

import numpy as np
import pytest
import torch

import paper_2312_14227_b200 as et
from oracle import block_oracle as blk
from paper_2312_14227_b200.elastic_loop import ElasticLoop

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF = torch.bfloat16
TOL = 2e-2
V, D, HEADS, KV, DIM, HID = 96, 128, 4, 2, 32, 200
SEQS, PREFIX, P, THETA, CAP = [0, 70, 71, 150], [9, 0, 30], 0.1, 10000.0, 20.0
M = 160


def desc(kind, i, o, **k):
    return et.et_layer_desc(**{"in_features": i, "out_features": o, "fold": 1, "residual_src": -1, "kind": kind, **k})


QKV = (HEADS + 2 * KV) * DIM


def block(first):
    """Layers of one block whose input is a_first."""
    dense, norm = et.ET_LAYER_DENSE, et.ET_LAYER_NORM
    f = first
    return [desc(norm, D, D, eps=1e-5), desc(dense, D, QKV),
            desc(et.ET_LAYER_ROTARY, QKV, QKV, heads=HEADS, kv_heads=KV, head_dim=DIM, axes=2, sections=(10, 6, 0), theta=THETA),
            desc(et.ET_LAYER_MASKED_ATTENTION, QKV, HEADS * DIM, heads=HEADS, kv_heads=KV, head_dim=DIM, mask=et.ET_MASK_CAUSAL, softcap=CAP),
            desc(dense, HEADS * DIM, D), desc(et.ET_LAYER_DROPOUT, D, D, drop=P, residual_src=f),
            desc(norm, D, D, eps=1e-5), desc(et.ET_LAYER_GATED, D, 2 * HID, fold=2, act=et.ET_ACT_SILU), desc(dense, HID, D),
            desc(et.ET_LAYER_DROPOUT, D, D, drop=P, residual_src=f + 6)]


class Model:
    def __init__(self, blocks=2, seed=0):
        rng = np.random.default_rng(seed)
        self.layers = [desc(et.ET_LAYER_EMBEDDING, V, D)]
        for _ in range(blocks):
            self.layers += block(len(self.layers))
        self.layers += [desc(et.ET_LAYER_NORM, D, D, eps=1e-5), desc(et.ET_LAYER_DENSE, D, V)]
        et.et_debug_guard_regions(True)
        self.s = et.et_stack_create(self.layers, M, et.ET_BF16)
        et.et_debug_guard_regions(False)
        t = lambda a: torch.from_numpy(np.asarray(a, dtype=np.float32)).to(BF).to(DEV)  # noqa: E731
        self.W, self.b = [], []
        for d in self.layers:
            k, i, o = d.kind, d.in_features, d.out_features
            if k == et.ET_LAYER_EMBEDDING:
                self.W.append(t(rng.normal(size=(i, o)))); self.b.append(None)
            elif k == et.ET_LAYER_NORM:
                self.W.append(t(1 + 0.1 * rng.normal(size=o))); self.b.append(t(0.1 * rng.normal(size=o)))
            elif k in (et.ET_LAYER_DENSE, et.ET_LAYER_GATED):
                self.W.append(t(rng.normal(size=(i, o)) / math.sqrt(i))); self.b.append(t(0.05 * rng.normal(size=o)))
            else:
                self.W.append(None); self.b.append(None)
        self.ws = torch.empty(et.et_stack_workspace_bytes(self.s), dtype=torch.uint8, device=DEV)
        self.ws.fill_(0xFF)
        et.et_stack_bind(self.s, self.W, self.b, self.ws)
        i32 = lambda a: torch.tensor(np.asarray(a), dtype=torch.int32, device=DEV)  # noqa: E731
        self.pos = np.stack([rng.integers(0, 3000, M), rng.integers(0, 60, M)])
        self.seed, self.step = 1234567, 3
        self.seed_dev = torch.tensor([self.seed, self.step], dtype=torch.int64, device=DEV)
        et.et_stack_set_sequences(self.s, i32(SEQS), i32(PREFIX))
        et.et_stack_set_positions(self.s, i32(self.pos))
        et.et_stack_set_dropout_seed(self.s, self.seed_dev)
        self.ids, self.targets = i32(rng.integers(0, V, M)), i32(rng.integers(0, V, M))
        w = (np.arange(M) < SEQS[-1]).astype(np.float32)
        self.weights = torch.from_numpy(w / w.sum()).to(DEV)
        self.adv = torch.from_numpy(rng.normal(size=M).astype(np.float32)).to(DEV)
        self.y, self.dY = torch.empty(M, V, dtype=BF, device=DEV), torch.empty(M, V, dtype=BF, device=DEV)
        self.L = len(self.layers)
        self.params = [p for pair in zip(self.W, self.b) for p in pair]
        self.all = np.array([p is not None for p in self.params], dtype=np.uint8)

    def step_(self, mask, grads=None, **k):
        et.et_forward_stack(self.s, self.ids, self.y)
        et.et_loss_policy_grad(self.s, self.y, self.targets, self.adv, self.dY, weights=self.weights)
        et.et_backward_elastic(self.s, self.dY, mask, grads, **k)

    def reference(self):
        """Logits, and the gradients of all tensors for the library's own dY."""
        leaf = [p.double().requires_grad_() if p is not None else None for p in self.params]
        a = [None, leaf[0][self.ids.long()]]
        see = torch.from_numpy(blk.visible(M, SEQS, True, PREFIX)).to(DEV)
        inside = torch.arange(M, device=DEV) < SEQS[-1]
        for l, d in enumerate(self.layers[1:], 1):
            x, w, b = a[l], leaf[2 * l], leaf[2 * l + 1]
            if d.kind == et.ET_LAYER_NORM:
                y = torch.nn.functional.layer_norm(x, (D,), w, b, 1e-5)
            elif d.kind == et.ET_LAYER_DENSE:
                y = x @ w + b
            elif d.kind == et.ET_LAYER_GATED:
                z = x @ w + b
                y = torch.nn.functional.silu(z[:, :HID]) * z[:, HID:]
            elif d.kind == et.ET_LAYER_ROTARY:
                n = 16
                freq = torch.tensor([THETA ** (-k / n) for k in range(n)], device=DEV, dtype=torch.float64)
                pos = torch.from_numpy(self.pos).to(DEV).double()
                ang = torch.cat([pos[0][:, None] * freq[:10], pos[1][:, None] * freq[10:]], 1)[:, None]
                h = x.view(M, -1, DIM)
                u, v = h[:, :HEADS + KV, :n], h[:, :HEADS + KV, n:]
                t = torch.cat([u * ang.cos() - v * ang.sin(), v * ang.cos() + u * ang.sin()], 2)
                y = torch.cat([t, h[:, HEADS + KV:]], 1).reshape(M, QKV)
            elif d.kind == et.ET_LAYER_MASKED_ATTENTION:
                h = x.view(M, -1, DIM).transpose(0, 1)
                q, k, v = h[:HEADS], h[HEADS:HEADS + KV].repeat_interleave(2, 0), h[HEADS + KV:].repeat_interleave(2, 0)
                z = CAP * torch.tanh(q @ k.transpose(1, 2) / math.sqrt(DIM) / CAP)
                p = torch.softmax(z.masked_fill(~see, -1e30), -1) * inside[:, None]
                y = (p @ v).transpose(0, 1).reshape(M, -1)
            else:
                keep = torch.from_numpy(blk.kept(0, M * D, float(np.float32(P)), self.seed, self.step, l).reshape(M, D)).to(DEV)
                y = x * keep / (1 - P) + a[d.residual_src]
            a.append(y)
        live = [p for p in leaf if p is not None]
        g = iter(torch.autograd.grad(a[-1], live, self.dY.double()))
        return a[-1].detach(), [next(g) if p is not None else None for p in leaf]

    def check_status(self):
        assert et.et_device_status(self.s) == et.ET_OK
        st, bad = et.et_debug_check_guards(self.s)
        assert st == et.ET_OK, bad


def compare(m, grads, mask, want):
    for t in range(2 * m.L):
        if mask[t]:
            e = (grads[t].double() - want[t]).abs().max() / want[t].abs().max()
            assert e <= TOL, (t, m.layers[t // 2].kind, float(e))


@pytest.mark.parametrize("two_streams", [1, 0])
def test_every_tensor_selected(two_streams):
    m = Model()
    et.et_stack_set_option(m.s, et.ET_OPTION_TWO_STREAMS, two_streams)
    grads = [torch.full(p.shape, float("nan"), device=DEV) if p is not None else None for p in m.params]
    m.step_(m.all, grads)
    m.check_status()
    y, want = m.reference()
    assert (m.y.double() - y).abs().max() <= TOL * y.abs().max()
    compare(m, grads, m.all, want)


@pytest.mark.parametrize("deepest", [4, 10, 14, 15, 16, 22, 24, 34, 44])
def test_masks_of_every_depth(deepest):
    """From the QKV layer's kernel under rotary and attention to the logits: what lies below is neither run nor touched."""
    m = Model()
    mask = m.all.copy()
    mask[:deepest] = 0
    mask[deepest + 3:2 * m.L - 2:2] = 0
    grads = [torch.full(p.shape, float("nan"), device=DEV) if b else None for p, b in zip(m.params, mask)]
    before = [p.clone() if p is not None else None for p in m.params]
    rep = et.Report(m.L)
    m.step_(mask, grads, report=rep)
    m.check_status()
    d = next(t for t in range(2 * m.L) if mask[t]) // 2
    assert rep.deepest == d and rep.dgrad.tolist() == [int(l > d) for l in range(m.L)]
    compare(m, grads, mask, m.reference()[1])
    for p, q in zip(m.params, before):
        assert p is None or torch.equal(p, q)


def test_a_whole_step_captured_and_replayed_on_other_inputs():
    """Forward, loss, backward, clipped update with masters; ids, bounds, positions and the dropout step change in memory."""
    def build():
        m = Model(blocks=1, seed=3)
        m.W32, m.b32 = ([p.float() if p is not None else None for p in q] for q in (m.W, m.b))
        et.et_stack_bind_master(m.s, m.W32, m.b32)
        m.grads = [torch.zeros(p.shape, device=DEV) if p is not None else None for p in m.params]
        return m

    def run(m, stream=None):
        et.et_forward_stack(m.s, m.ids, m.y, stream=stream)
        et.et_loss_policy_grad(m.s, m.y, m.targets, m.adv, m.dY, weights=m.weights, stream=stream)
        et.et_backward_elastic(m.s, m.dY, m.all, m.grads, stream=stream)
        et.et_update_clipped(m.s, m.all, m.grads, 0.05, 0.5, stream=stream)

    def change(m, i):
        g = torch.Generator(device=DEV)
        g.manual_seed(i)
        m.ids.copy_(torch.randint(0, V, (M,), generator=g, device=DEV, dtype=torch.int32))
        m.seed_dev[1] = i

    eager, captured = build(), build()
    side = torch.cuda.Stream()
    run(captured, side)                                  # first call outside the capture: modules are loaded
    torch.cuda.synchronize()
    for p, q in zip(captured.params, eager.params):
        if p is not None:
            p.copy_(q)
    for a, b in ((captured.W32, eager.W32), (captured.b32, eager.b32)):
        for p, q in zip(a, b):
            if p is not None:
                p.copy_(q)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        run(captured, side)
    for i in range(4):
        for m in (eager, captured):
            change(m, i)
        run(eager)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(eager.y, captured.y)
        for p, q in zip(eager.params, captured.params):
            assert p is None or torch.equal(p, q)
    eager.check_status()
    captured.check_status()


def test_costs_of_layers_without_tensors_go_to_the_bias_below():
    m = Model(blocks=1)
    et.et_forward_stack(m.s, m.ids, m.y)
    m.dY.normal_()
    t_dw, t_dy, t_fwd = et.et_profile_costs(m.s, m.ids, m.y, m.dY, iters=3)
    kinds = [d.kind for d in m.layers]
    for l, k in enumerate(kinds):
        if k in (et.ET_LAYER_ROTARY, et.ET_LAYER_MASKED_ATTENTION, et.ET_LAYER_DROPOUT):
            assert not t_dw[2 * l:2 * l + 2].any() and not t_dy[2 * l:2 * l + 2].any()
    assert t_dy[5] > 0 and t_dy[11] > 0                  # biases of the QKV projection and of the one below a dropout layer
    g = kinds.index(et.ET_LAYER_GATED)
    assert t_dw[2 * g] > 0 and t_dw[2 * g + 1] > 0 and t_dy[2 * g] > 0
    assert t_dy[2 * g + 1] == 0                          # dZ is formed in the error-gradient product of the dense layer above
    assert t_fwd > 0
    m.check_status()


def test_elastic_schedule_runs_over_decoder_blocks():
    """Windows, importances, re-selection and masked steps over a stack with every new kind of layer: every selection is feasible, empty
    slots are never selected, frozen tensors keep their bits in masked steps."""
    m = Model(blocks=1, seed=5)
    slot = lambda q: [p if p is not None else torch.zeros(0, dtype=BF, device=DEV) for p in q]  # noqa: E731
    et.et_forward_stack(m.s, m.ids, m.y)
    m.dY.normal_()
    t_dw, t_dy, t_fwd = et.et_profile_costs(m.s, m.ids, m.y, m.dY, iters=3)

    def loss(y, dY, out, stream):
        et.et_loss_policy_grad(m.s, y, m.targets, m.adv, dY, weights=m.weights, loss_dev=out, stream=stream)

    loop = ElasticLoop(m.s, slot(m.W), slot(m.b), m.ids, None, 0.02, 4, 2, 0.5, t_dw, t_dy, t_fwd, loss=loss)
    out = loop.run(8)
    assert np.isfinite(out["losses"]).all() and len(out["masks"]) == 8
    for mask in out["masks"]:
        assert not (mask & ~m.all.astype(bool)).any()
    chosen = out["masks"][3]
    before = [p.clone() if p is not None else None for p in m.params]
    m.step_(chosen, flags=et.ET_FLAG_FUSE_SGD, lr=0.02)
    m.check_status()
    for t, (p, q) in enumerate(zip(m.params, before)):
        if p is not None and not chosen[t]:
            assert torch.equal(p, q), t
