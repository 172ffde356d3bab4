"""Masked attention against the float64 oracle, through the C ABI: every element within the bound that the oracle forms from the formats'
roundings (oracle/block_oracle.py)."""
import numpy as np
import pytest
import torch

import paper_2312_14227_b200 as et
from oracle import block_oracle as blk

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF = torch.bfloat16


def rows_of(rng, *shape, std=1.0):
    return torch.from_numpy((rng.normal(size=shape) * std).astype(np.float32)).to(BF).to(DEV)


def f64(t):
    return t.double().cpu().numpy()


class Attn:
    """A stack of one attention layer with the gradient of its input."""

    def __init__(self, M, heads, kv, dim, seqs=None, causal=True, prefix=None, cap=0.0, slopes=None, seq_len=0, scale=0.0, seed=0, std=1.0):
        rng = np.random.default_rng(seed)
        self.M, self.heads, self.kv, self.dim = M, heads, kv, dim
        d = et.et_layer_desc(in_features=(heads + 2 * kv) * dim, out_features=heads * dim, fold=1, residual_src=-1,
                             kind=et.ET_LAYER_MASKED_ATTENTION, heads=heads, kv_heads=kv, head_dim=dim, seq_len=seq_len,
                             mask=et.ET_MASK_CAUSAL if causal else et.ET_MASK_NONE, softcap=cap, scale=scale)
        et.et_debug_guard_regions(True)
        self.s = et.et_stack_create([d], M, et.ET_BF16)
        et.et_debug_guard_regions(False)
        self.ws = torch.empty(et.et_stack_workspace_bytes(self.s), dtype=torch.uint8, device=DEV)
        self.ws.fill_(0xFF)                              # NaN in whatever is not written before it is read
        et.et_stack_bind(self.s, [None], [None], self.ws)
        self.x, self.dY = rows_of(rng, M, d.in_features, std=std), rows_of(rng, M, d.out_features)
        # guard rows behind the outputs
        self.y = torch.full((M + 1, d.out_features), 7.0, dtype=BF, device=DEV)
        self.dX = torch.full((M + 1, d.in_features), 7.0, dtype=BF, device=DEV)
        et.et_stack_set_input_gradient(self.s, self.dX)
        self.seqs, self.prefix, self.causal, self.cap, self.scale, self.slopes = seqs, prefix, causal, cap, scale, slopes
        if seqs is not None:
            i32 = lambda v: None if v is None else torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
            self.begin, self.pre = i32(seqs), i32(prefix)
            et.et_stack_set_sequences(self.s, self.begin, self.pre)
        else:
            n = seq_len or M
            self.seqs = list(range(0, M + 1, n))
        if slopes is not None:
            et.et_stack_set_distance_bias(self.s, 0, torch.tensor(slopes, dtype=torch.float32, device=DEV))

    def run(self, back=True):
        et.et_forward_stack(self.s, self.x, self.y)
        if back:
            et.et_backward_elastic(self.s, self.dY, [0, 0])
        assert et.et_device_status(self.s) == et.ET_OK
        st, bad = et.et_debug_check_guards(self.s)
        assert st == et.ET_OK, bad
        assert bool((self.y[self.M] == 7).all()) and bool((self.dX[self.M] == 7).all())
        return self.y[:self.M], self.dX[:self.M]

    def check(self, x=None):
        y, dX = self.run()
        see = blk.visible(self.M, self.seqs, self.causal, self.prefix)
        x = f64(self.x) if x is None else x
        o, oe, g, ge = blk.attention(x, self.heads, self.kv, self.dim, see, self.scale, self.cap, self.slopes, f64(self.dY))
        for name, a, b, e in (("y", f64(y), o, oe), ("dX", f64(dX), g, ge)):
            off = np.abs(a - b) - e
            assert np.isfinite(a).all(), name
            assert off.max() <= 1e-30, (name, np.unravel_index(off.argmax(), off.shape), float(off.max()), float((np.abs(a - b) / np.maximum(e, 1e-30)).max()))


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("M", [1, 2, 63, 64, 65, 127, 128, 129, 200, 255, 256, 257, 385])
def test_lengths(M, causal):
    Attn(M, 2, 1, 64, causal=causal, seed=M).check()


@pytest.mark.parametrize("dim", [8, 16, 40, 64, 72, 96, 120, 128])
def test_head_widths(dim):
    Attn(150, 3, 3, dim, causal=True, seed=dim).check()


@pytest.mark.parametrize("heads,kv", [(1, 1), (4, 1), (6, 2), (5, 5), (8, 2)])
def test_shared_heads(heads, kv):
    Attn(140, heads, kv, 64, seed=heads).check()
    Attn(70, heads, kv, 128, causal=False, seed=heads).check()


SEQS = {"tile-ends": [0, 64, 128, 256, 300], "ones": list(range(0, 71)), "empty-ones": [0, 0, 5, 5, 5, 130, 130, 200, 200],
        "holes-at-the-ends": [30, 140, 190], "all-empty": [40, 40, 40], "one-row": [130, 131], "many": [0] * 40 + [3] * 70 + [120] + [121] * 1100 + [250]}


@pytest.mark.parametrize("name", sorted(SEQS))
@pytest.mark.parametrize("causal", [True, False])
def test_sequences(name, causal):
    b = SEQS[name]
    Attn(max(b[-1], 210 if name == "holes-at-the-ends" else b[-1] + 13), 2, 1, 64, seqs=b, causal=causal).check()


@pytest.mark.parametrize("prefix", [[0, 0, 0], [5, 1000, -3], [130, 64, 128], [1, 2, 200]])
def test_prefixes(prefix):
    Attn(460, 2, 2, 64, seqs=[0, 140, 210, 455], prefix=prefix).check()


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("cap,slopes,causal", [(5.0, None, True), (50.0, None, False), (0.0, [0.5, 0.01], True), (0.0, [-0.02, 0.0], False), (2.0, [0.25, 3.0], True)])
def test_capped_scores_and_distance_bias(dim, cap, slopes, causal):
    Attn(270, 2, 1, dim, seqs=[0, 133, 262], causal=causal, cap=cap, slopes=slopes, std=2.0).check()


def test_runs_of_one_length_and_a_given_scale():
    Attn(5 * 37, 2, 1, 64, seq_len=37, causal=True, scale=0.3).check()
    Attn(3 * 128, 1, 1, 128, seq_len=128, causal=False, scale=0.02).check()


def test_scores_far_apart():
    """One key takes nearly all of the weight; maxima grow from tile to tile, so that the output is rescaled."""
    a = Attn(300, 1, 1, 64, causal=False)
    ramp = torch.linspace(0.2, 6.0, 300, device=DEV)[:, None]
    a.x[:, 64:128] = (a.x[:, 64:128].float() * ramp).to(BF)
    a.x[:, :64] *= 2
    a.check()


def test_rows_of_no_sequence_may_hold_anything():
    for bad in (float("nan"), float("inf"), -3.0e38):
        for causal in (True, False):
            a = Attn(300, 2, 1, 64, seqs=[17, 130, 250], causal=causal)
            clean = f64(a.x)
            for sl in (slice(0, 17), slice(250, 300)):
                a.x[sl] = bad
                a.dY[sl] = bad
                clean[sl] = 0
            y, dX = a.run()
            assert not y[:17].any() and not y[250:].any() and not dX[:17].any() and not dX[250:].any()
            a.dY[:17] = 0
            a.dY[250:] = 0
            before = y.clone(), dX.clone()
            a.check(clean)
            assert torch.equal(before[0], a.y[:300]) and torch.equal(before[1], a.dX[:300])


def test_bounds_out_of_range_are_clamped_and_others_stay_inside():
    a = Attn(200, 2, 1, 64, seqs=[0, 90, 200])
    a.begin.copy_(torch.tensor([-7, 90, 2 ** 31 - 1], dtype=torch.int32))
    a.check()
    rng = np.random.default_rng(5)
    a = Attn(200, 2, 1, 64, seqs=[0] * 34, prefix=[0] * 33)
    for _ in range(5):                                   # not non-decreasing: nothing out of range is read or written
        a.begin.copy_(torch.from_numpy(rng.integers(-2 ** 31, 2 ** 31, 34).astype(np.int32)))
        a.pre.copy_(torch.from_numpy(rng.integers(-2 ** 31, 2 ** 31, 33).astype(np.int32)))
        a.run()
        a.begin.copy_(torch.from_numpy(rng.integers(-50, 250, 34).astype(np.int32)))
        a.run()


def test_forward_only_leaves_the_gradient_alone_and_runs_repeat_to_the_bit():
    a = Attn(777, 4, 2, 128, seqs=[0, 300, 770], prefix=[20, 0], cap=20.0, slopes=[0.1, 0.2, 0.3, 0.4])
    a.run(back=False)
    assert bool((a.dX == 7).all())
    y, dX = (t.clone() for t in a.run())
    for _ in range(3):
        u, v = a.run()
        assert torch.equal(y, u) and torch.equal(dX, v)


def test_the_last_layers_output_cannot_take_the_gradient():
    a = Attn(20, 1, 1, 64)
    a.run()
    with pytest.raises(et.EtError):
        et.et_backward_elastic(a.s, a.y, [0, 0])


def test_captured_call_follows_the_bounds_in_memory():
    a = Attn(300, 2, 1, 64, seqs=[0, 100, 300], prefix=[10, 0])
    a.run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        et.et_forward_stack(a.s, a.x, a.y, stream=side)
        et.et_backward_elastic(a.s, a.dY, [0, 0], stream=side)
    for seqs, prefix in (([0, 200, 290], [0, 70]), ([5, 5, 128], [1, 300])):
        a.begin.copy_(torch.tensor(seqs, dtype=torch.int32))
        a.pre.copy_(torch.tensor(prefix, dtype=torch.int32))
        a.x.copy_(rows_of(np.random.default_rng(seqs[1]), *a.x.shape))
        a.y.fill_(7)
        a.dX.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        got = a.y[:300].clone(), a.dX[:300].clone()
        a.seqs, a.prefix = seqs, prefix
        a.check()
        assert torch.equal(got[0], a.y[:300]) and torch.equal(got[1], a.dX[:300])


def test_two_stacks_on_two_streams():
    jobs = [Attn(1500, 4, 2, 128, seqs=[0, 700, 1490], seed=1), Attn(1100, 6, 3, 64, causal=False, cap=9.0, seed=2)]
    want = [[t.clone() for t in a.run()] for a in jobs]
    streams = [torch.cuda.Stream() for _ in jobs]
    torch.cuda.synchronize()
    for _ in range(20):
        for a, st in zip(jobs, streams):
            et.et_forward_stack(a.s, a.x, a.y, stream=st)
            et.et_backward_elastic(a.s, a.dY, [0, 0], stream=st)
    torch.cuda.synchronize()
    for a, w in zip(jobs, want):
        assert torch.equal(a.y[:a.M], w[0]) and torch.equal(a.dX[:a.M], w[1])


def test_offsets_beyond_32_bits():
    """Rows of 7168 columns, 4.3e9 elements: the last sequences against the same rows in a small stack."""
    heads, kv, dim, M = 52, 2, 128, 602_000
    assert M * (heads + 2 * kv) * dim > 2 ** 32
    tail = 500
    seqs = list(range(0, M - tail, 1003)) + [M - tail, M - tail + 190, M - 3]
    d = et.et_layer_desc(in_features=(heads + 2 * kv) * dim, out_features=heads * dim, fold=1, residual_src=-1, kind=et.ET_LAYER_MASKED_ATTENTION,
                         heads=heads, kv_heads=kv, head_dim=dim, mask=et.ET_MASK_CAUSAL)
    out = []
    small = None
    for rows, s in ((M, seqs), (tail, [0, 190, tail - 3])):
        stack = et.et_stack_create([d], rows, et.ET_BF16)
        ws = torch.empty(et.et_stack_workspace_bytes(stack), dtype=torch.uint8, device=DEV)
        et.et_stack_bind(stack, [None], [None], ws)
        if rows == M:
            x = torch.empty(rows, d.in_features, dtype=BF, device=DEV)
            dY = torch.empty(rows, d.out_features, dtype=BF, device=DEV)
            for t in (x, dY):
                t.view(-1)[:2 ** 20].normal_()
                t.view(-1)[2 ** 20:] = 0.25
                t[M - tail - 64:].normal_()
            small = x[M - tail:].clone(), dY[M - tail:].clone()
        else:
            x, dY = small
        y, dX = torch.empty(rows, d.out_features, dtype=BF, device=DEV), torch.empty_like(x)
        et.et_stack_set_sequences(stack, torch.tensor(s, dtype=torch.int32, device=DEV))
        et.et_stack_set_input_gradient(stack, dX)
        et.et_forward_stack(stack, x, y)
        et.et_backward_elastic(stack, dY, [0, 0])
        assert et.et_device_status(stack) == et.ET_OK
        out.append((y[rows - tail:].clone(), dX[rows - tail:].clone()))
        del x, dY, y, dX, ws
        stack.close()
        torch.cuda.empty_cache()
    for a, b in zip(*out):
        # the tiles that a row's keys fall into differ: equal up to two roundings of each step
        assert (a.double() - b.double()).abs().max() <= 2.0 ** -6 * b.double().abs().max()
        assert not a[-3:].any()
