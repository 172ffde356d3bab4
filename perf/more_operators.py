"""Cases for the layers of a decoder block in a stack that is fine-tuned on token sequences.

  attention   softmax attention over packed sequences: causal and prefix masks, document bounds, capped scores, a bias by
              distance, shared key / value heads (ET_LAYER_MASKED_ATTENTION)
  rotary      rotary positions of one to three axes on the query and key heads (ET_LAYER_ROTARY)
  gated       gated feed-forward block: both projections, activation and product, then the projection back (ET_LAYER_GATED)
  dropout     dropout from a counter-based generator, with the residual (ET_LAYER_DROPOUT)

"fwd" is the forward pass, "step" the forward and the backward pass, which returns the gradient of the stack's input and,
where there are weights, applies their gradients (plain SGD) and returns the weights.

`own` False: plain torch operations in 32 bits (64 for angles), rounded once.
`own` True: the library's calls.
"""
import math

import torch

own = False
DEV = "cuda"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


# ------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # one short prompt: a few rows, launch latency counts
        attention("attention-small", "step", rows=37, heads=4, kv=2, dim=64, seqs=1),
        # a packed batch of documents, padded at its end; four query heads share a key head
        attention("attention-documents", "step", rows=8192, heads=16, kv=4, dim=128, seqs=13, pad=77),
        # prompts that every row of a sequence sees whole, answers causal; capped scores; a head width between the tiles'
        attention("attention-prefix-capped", "step", rows=4000, heads=12, kv=12, dim=80, seqs=5, prefix=True, cap=30.0),
        # one long document, a bias that falls with distance, forward only
        attention("attention-long-bias", "fwd", rows=24576, heads=16, kv=2, dim=128, seqs=1, bias=True),
        # images of a batch, every patch sees its whole image; many short sequences
        attention("attention-images", "step", rows=64 * 197, heads=12, kv=12, dim=64, seqs=64, causal=False, even=True),
        # a prompt's positions: few rows, one axis
        rotary("rotary-small", "fwd", rows=37, heads=4, kv=2, dim=64, sections=(32,), dtype="f32"),
        # video tokens: time, height and width, the axes' own spectra
        rotary("rotary-video", "step", rows=32760, heads=16, kv=16, dim=128, sections=(22, 21, 21), own_spectrum=True, dtype="bf16"),
        # a small block in fp32
        gated("gated-small-f32", "step", rows=100, d=136, hidden=344, act="silu", dtype="f32"),
        # the block in inference: forward only, an odd number of rows
        gated("gated-forward", "fwd", rows=2049, d=1024, hidden=2816, act="gelu", dtype="bf16"),
        # a training step of a large block
        gated("gated-step", "step", rows=8192, d=2048, hidden=5632, act="silu", dtype="bf16"),
        # dropout on few rows of an odd width
        dropout("dropout-small-f32", "fwd", rows=50, width=197, p=0.1, residual=True, dtype="f32"),
        # dropout behind a projection, added to the residual stream of a large batch
        dropout("dropout-residual", "step", rows=32768, width=4096, p=0.1, residual=True, dtype="bf16"),
    ]


def attention(name, pass_, rows, heads, kv, dim, seqs, causal=True, prefix=False, cap=0.0, bias=False, pad=0, even=False):
    """pad: rows behind the last sequence; even: sequences of one length."""
    return {"name": name, "op": "attention", "pass": pass_, "rows": rows, "heads": heads, "kv": kv, "dim": dim, "seqs": seqs,
            "causal": causal, "prefix": prefix, "cap": cap, "bias": bias, "pad": pad, "even": even}


def rotary(name, pass_, rows, heads, kv, dim, sections, dtype, own_spectrum=False, adjacent=False, theta=10000.0):
    s = list(sections) + [0, 0]
    return {"name": name, "op": "rotary", "pass": pass_, "rows": rows, "heads": heads, "kv": kv, "dim": dim, "axes": len(sections),
            "s0": s[0], "s1": s[1], "s2": s[2], "own_spectrum": own_spectrum, "adjacent": adjacent, "theta": theta, "dtype": dtype}


def gated(name, pass_, rows, d, hidden, act, dtype):
    return {"name": name, "op": "gated", "pass": pass_, "rows": rows, "d": d, "hidden": hidden, "act": act, "dtype": dtype}


def dropout(name, pass_, rows, width, p, residual, dtype):
    return {"name": name, "op": "dropout", "pass": pass_, "rows": rows, "width": width, "p": p, "residual": residual, "dtype": dtype}


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attention", "attention", "rotary", "gated", "dropout"])
    pass_ = rng.choice(["fwd", "step"])
    dtype = rng.choice(["f32", "bf16"])
    kv = rng.choice([1, 2, 3, 4, 8])
    heads = kv * rng.choice([1, 2, 4])
    dim = rng.choice([32, 64, 64, 80, 96, 128, 128])
    if op == "attention":
        most = 16384 if pass_ == "fwd" else 8192
        rows = _log_int(rng, 1, min(most, int(math.sqrt((6e11 if pass_ == "fwd" else 1.7e11) / (heads * dim)))))
        seqs = _log_int(rng, 1, min(rows, 64))
        causal = rng.random() < 0.75
        c = attention("", pass_, rows, heads, kv, dim, seqs, causal, causal and rng.random() < 0.3, rng.choice([0.0, 0.0, 20.0, 50.0]),
                      rng.random() < 0.3, 0 if rng.random() < 0.5 else rng.randrange(0, 1 + rows // 8))
    elif op == "rotary":
        pairs = dim // 2 if rng.random() < 0.7 else dim // 4
        axes = rng.choice([1, 2, 3])
        a = pairs // axes
        rows = _log_int(rng, 1, min(65536, 130_000_000 // ((heads + 2 * kv) * dim)))
        c = rotary("", pass_, rows, heads, kv, dim, [pairs - a * (axes - 1)] + [a] * (axes - 1), dtype, rng.random() < 0.5,
                   rng.random() < 0.5, rng.choice([10000.0, 500000.0]))
    elif op == "gated":
        d = 8 * _log_int(rng, 4, 256 if dtype == "bf16" else 64)
        hidden = 8 * _log_int(rng, 4, 704 if dtype == "bf16" else 128)
        rows = _log_int(rng, 1, 8192 if dtype == "bf16" else 512)
        c = gated("", pass_, rows, d, hidden, rng.choice(["silu", "gelu", "relu"]), dtype)
    else:
        width = _log_int(rng, 16, 4096)
        if dtype == "bf16":
            width = -(-width // 8) * 8
        c = dropout("", pass_, _log_int(rng, 1, min(65536, 100_000_000 // width)), width, rng.choice([0.05, 0.1, 0.5]),
                    rng.random() < 0.7, dtype)
    del c["name"]
    return c


# ------------------------------------------------------------------------------------------ inputs
def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _randn(g, *shape, dtype=torch.float32):
    return torch.randn(*shape, generator=g, device=DEV, dtype=dtype)


def _bounds(c, seed):
    """Begins of the sequences and the end of the last one; lengths of 1 upwards, drawn."""
    end, n = c["rows"] - c["pad"], c["seqs"]
    if c["even"]:
        return [end // n * i for i in range(n)] + [end]
    g = torch.Generator()
    g.manual_seed(seed + 1)
    n = min(n, end)
    cuts = (torch.randperm(end - 1, generator=g)[:n - 1] + 1).sort().values.tolist() if n > 1 else []
    return [0] + cuts + [end]


def prepare(case, seed):
    c, g, op = case, _gen(seed), case["op"]
    s = {"c": c}
    rows = c["rows"]
    dt = DTYPES[c.get("dtype", "bf16")]
    if op in ("attention", "rotary"):
        width = (c["heads"] + 2 * c["kv"]) * c["dim"]
        s["x"] = _randn(g, rows, width, dtype=dt)
    if op == "attention":
        out = c["heads"] * c["dim"]
        s["bounds"] = _bounds(c, seed)
        s["seq_begin"] = torch.tensor(s["bounds"], dtype=torch.int32, device=DEV)
        if c["prefix"]:
            lens = (s["seq_begin"][1:] - s["seq_begin"][:-1]).float()
            s["prefix"] = (lens * torch.rand(len(lens), generator=g, device=DEV)).to(torch.int32)
        if c["bias"]:
            s["slopes"] = torch.exp2(-8.0 * torch.arange(1, c["heads"] + 1, device=DEV, dtype=torch.float32) / c["heads"])
    elif op == "rotary":
        out = width
        # positions of a long context; on several axes frames, rows and columns
        top = [65536, 512, 512] if c["axes"] == 1 else [4096, 512, 512]
        s["positions"] = torch.stack([torch.randint(0, top[a], (rows,), generator=g, device=DEV, dtype=torch.int32)
                                      for a in range(c["axes"])])
    elif op == "gated":
        d, h = c["d"], c["hidden"]
        out = d
        s["x"] = _randn(g, rows, d, dtype=dt)
        s["W1"] = (_randn(g, d, 2 * h) / math.sqrt(d)).to(dt)
        s["b1"] = (0.1 * _randn(g, 2 * h)).to(dt)
        s["W2"] = (_randn(g, h, d) / math.sqrt(h)).to(dt)
        s["b2"] = (0.1 * _randn(g, d)).to(dt)
    else:
        out = c["width"]
        s["x"] = _randn(g, rows, out, dtype=dt)
        s["seed"] = torch.randint(-2 ** 62, 2 ** 62, (2,), generator=g, device=DEV, dtype=torch.int64)
    s["y"] = torch.empty(rows, out, device=DEV, dtype=dt)
    if c["pass"] == "step":
        s["dY"] = _randn(g, rows, out, dtype=dt)
        s["dX"] = torch.empty_like(s["x"])
    if own:
        _bind(s)
    return s


ACTS = {"gelu": 1, "relu": 2, "silu": 3}
LR = 1e-6                    # no loss is descended here: small enough that the weights keep their size over many passes
WEIGHTS = ("W1", "b1", "W2", "b2")


def _bind(s):
    """The stack a user keeps: created once, its tensors, workspace and the device arrays of its layers attached."""
    import numpy as np
    import paper_2312_14227_b200 as et
    c, op = s["c"], s["c"]["op"]
    desc = lambda **k: et.et_layer_desc(**{"fold": 1, "residual_src": -1, **k})  # noqa: E731
    none = [None]
    W, b = none, none
    if op == "attention":
        layers = [desc(in_features=s["x"].shape[1], out_features=c["heads"] * c["dim"], kind=et.ET_LAYER_MASKED_ATTENTION,
                       heads=c["heads"], kv_heads=c["kv"], head_dim=c["dim"],
                       mask=et.ET_MASK_CAUSAL if c["causal"] else et.ET_MASK_NONE, softcap=c["cap"])]
    elif op == "rotary":
        w = s["x"].shape[1]
        layers = [desc(in_features=w, out_features=w, kind=et.ET_LAYER_ROTARY, heads=c["heads"], kv_heads=c["kv"], head_dim=c["dim"],
                       axes=c["axes"], sections=(c["s0"], c["s1"], c["s2"]), theta=c["theta"],
                       pairing=et.ET_ROTARY_ADJACENT if c["adjacent"] else et.ET_ROTARY_HALVES,
                       spectrum=et.ET_ROTARY_OWN_SPECTRUM if c["own_spectrum"] else et.ET_ROTARY_ONE_SPECTRUM)]
    elif op == "gated":
        layers = [desc(in_features=c["d"], out_features=2 * c["hidden"], act=ACTS[c["act"]], fold=2, kind=et.ET_LAYER_GATED),
                  desc(in_features=c["hidden"], out_features=c["d"])]
        W, b = [s["W1"], s["W2"]], [s["b1"], s["b2"]]
    else:
        layers = [desc(in_features=c["width"], out_features=c["width"], kind=et.ET_LAYER_DROPOUT, drop=c["p"],
                       residual_src=0 if c["residual"] else -1)]
    stack = et.et_stack_create(layers, c["rows"], et.ET_F32 if c.get("dtype") == "f32" else et.ET_BF16)
    workspace = torch.empty(et.et_stack_workspace_bytes(stack), dtype=torch.uint8, device=DEV)
    et.et_stack_bind(stack, W, b, workspace)
    if op == "attention":
        et.et_stack_set_sequences(stack, s["seq_begin"], s.get("prefix"))
        if c["bias"]:
            et.et_stack_set_distance_bias(stack, 0, s["slopes"])
    elif op == "rotary":
        et.et_stack_set_positions(stack, s["positions"])
    elif op == "dropout":
        et.et_stack_set_dropout_seed(stack, s["seed"])
    if c["pass"] == "step":
        et.et_stack_set_input_gradient(stack, s["dX"])
    s["mask"] = np.full(2 * len(layers), 1 if op == "gated" else 0, dtype=np.uint8)
    s["stack"] = stack


# ------------------------------------------------------------------------------------------ one pass
def run(state):
    s, c = state, state["c"]
    if own:
        import paper_2312_14227_b200 as et
        et.et_forward_stack(s["stack"], s["x"], s["y"])
        if c["pass"] == "fwd":
            return s["y"]
        out = {"y": s["y"], "dX": s["dX"]}
        if c["op"] == "gated":
            et.et_backward_elastic(s["stack"], s["dY"], s["mask"], flags=et.ET_FLAG_FUSE_SGD, lr=LR)
            out.update({k: s[k] for k in WEIGHTS})
        else:
            et.et_backward_elastic(s["stack"], s["dY"], s["mask"])
        return out
    return {"attention": _attention_plain, "rotary": _rotary_plain, "gated": _gated_plain, "dropout": _dropout_plain}[c["op"]](s, c)


def _row_bounds(s, c):
    """For every row the first key that it sees and the one behind the last; equal where it is in no sequence."""
    begin = s["seq_begin"].long()
    at = torch.arange(c["rows"], device=DEV)
    q = torch.bucketize(at, begin, right=True) - 1
    inside = (q >= 0) & (q < len(begin) - 1)
    q = q.clamp(0, len(begin) - 2)
    lo, hi = begin[q], begin[q + 1]
    if c["causal"]:
        last = at + 1
        if "prefix" in s:
            last = torch.maximum(last, lo + s["prefix"].long()[q])
        hi = torch.minimum(hi, last)
    zero = torch.zeros_like(lo)
    return torch.where(inside, lo, zero), torch.where(inside, hi, zero)


def _attention_plain(s, c):
    rows, heads, kv, dim = c["rows"], c["heads"], c["kv"], c["dim"]
    group, scale, step = heads // kv, 1.0 / math.sqrt(dim), c["pass"] == "step"
    x = s["x"].float()
    q = x[:, :heads * dim].view(rows, heads, dim).transpose(0, 1)
    k = x[:, heads * dim:(heads + kv) * dim].view(rows, kv, dim).transpose(0, 1)
    v = x[:, (heads + kv) * dim:].view(rows, kv, dim).transpose(0, 1)
    lo, hi = _row_bounds(s, c)
    at = torch.arange(rows, device=DEV)
    y = torch.empty(heads, rows, dim, device=DEV)
    if step:
        dy = s["dY"].float().view(rows, heads, dim).transpose(0, 1)
        dq = torch.empty(heads, rows, dim, device=DEV)
        dk, dv = torch.zeros(kv, rows, dim, device=DEV), torch.zeros(kv, rows, dim, device=DEV)
    hb = max(1, min(heads, 500_000_000 // rows ** 2))                    # heads, and rows of one head, at a time
    block = max(1, min(rows, 500_000_000 // rows))
    for h in range(0, heads, hb):
        hs = slice(h, min(heads, h + hb))
        shared = torch.arange(heads, device=DEV)[hs] // group
        kh, vh = k[shared], v[shared]
        for r in range(0, rows, block):
            i = slice(r, min(rows, r + block))
            z = (q[hs, i] @ kh.transpose(1, 2)) * scale
            if c["cap"]:
                t = torch.tanh(z / c["cap"])
                z = t * c["cap"]
            if c["bias"]:
                z = z - s["slopes"][hs, None, None] * (at[i, None] - at[None]).abs()
            seen = (at[None] >= lo[i, None]) & (at[None] < hi[i, None])
            z = z.masked_fill(~seen, float("-inf"))
            m = z.amax(2, keepdim=True)
            m = torch.where(m == float("-inf"), torch.zeros_like(m), m)
            p = torch.exp(z - m)
            total = p.sum(2, keepdim=True)
            p = p / torch.where(total == 0, torch.ones_like(total), total)
            y[hs, i] = p @ vh
            if step:
                dp = dy[hs, i] @ vh.transpose(1, 2)
                dz = p * (dp - (dp * p).sum(2, keepdim=True))
                if c["cap"]:
                    dz = dz * (1 - t * t)
                dz = dz * scale
                dq[hs, i] = dz @ kh
                dk.index_add_(0, shared, dz.transpose(1, 2) @ q[hs, i])
                dv.index_add_(0, shared, p.transpose(1, 2) @ dy[hs, i])
    y = y.transpose(0, 1).reshape(rows, heads * dim).to(s["x"].dtype)
    if not step:
        return y
    dx = torch.cat([t.transpose(0, 1).reshape(rows, -1) for t in (dq, dk, dv)], 1)
    return {"y": y, "dX": dx.to(s["x"].dtype)}


def _spectrum(c):
    """Axis and frequency of every pair."""
    sections = [c["s0"], c["s1"], c["s2"]][:c["axes"]]
    total = sum(sections)
    axis, freq = [], []
    for a, n in enumerate(sections):
        for j in range(n):
            exponent = j / n if c["own_spectrum"] else len(axis) / total
            axis.append(a)
            freq.append(c["theta"] ** -exponent)
    return axis, freq


def _rotary_plain(s, c):
    axis, freq = _spectrum(c)
    n = len(axis)
    angle = s["positions"].double()[torch.tensor(axis, device=DEV)].T * torch.tensor(freq, dtype=torch.float64, device=DEV)
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]

    def turn(x, sin):
        x = x.float().view(c["rows"], c["heads"] + 2 * c["kv"], c["dim"])
        out = x.clone()
        t = x[:, :c["heads"] + c["kv"]]
        one, two = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if c["adjacent"] else (slice(0, n), slice(n, 2 * n))
        out[:, :c["heads"] + c["kv"], one] = t[..., one] * cos - t[..., two] * sin
        out[:, :c["heads"] + c["kv"], two] = t[..., two] * cos + t[..., one] * sin
        return out.view(c["rows"], -1)

    y = turn(s["x"], sin).to(s["x"].dtype)
    return y if c["pass"] == "fwd" else {"y": y, "dX": turn(s["dY"], -sin).to(s["x"].dtype)}


def _act_plain(z, kind):
    """Activation and its slope."""
    if kind == "silu":
        g = 1 / (1 + torch.exp(-z))
        return z * g, g * (1 + z * (1 - g))
    if kind == "relu":
        on = (z > 0).to(z.dtype)
        return z * on, on
    c0, c1 = math.sqrt(2 / math.pi), 0.044715
    t = torch.tanh(c0 * (z + c1 * z ** 3))
    return 0.5 * z * (1 + t), 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * c0 * (1 + 3 * c1 * z * z)


def _gated_plain(s, c):
    h = c["hidden"]
    x, W1, W2 = s["x"].float(), s["W1"].float(), s["W2"].float()
    z = x @ W1 + s["b1"].float()
    f, slope = _act_plain(z[:, :h], c["act"])
    a = f * z[:, h:]
    y = (a @ W2 + s["b2"].float()).to(s["x"].dtype)
    if c["pass"] == "fwd":
        return y
    dy = s["dY"].float()
    da = dy @ W2.T
    dz = torch.cat([da * z[:, h:] * slope, da * f], 1)
    out = {"y": y, "dX": (dz @ W1.T).to(s["x"].dtype)}
    for k, g in zip(WEIGHTS, (x.T @ dz, dz.sum(0), a.T @ dy, dy.sum(0))):
        out[k] = s[k].copy_(s[k].float() - LR * g)
    return out


def _philox(counter, key):
    """Ten rounds of Philox 4x32 (Salmon et al. 2011) on int64 tensors that hold 32-bit words."""
    low = 0xFFFFFFFF
    c0, c1, c2, c3 = counter
    k0, k1 = key
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = ((b >> 32) & low) ^ c1 ^ k0, b & low, ((a >> 32) & low) ^ c3 ^ k1, a & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    return c0, c1, c2, c3


def _kept(s, c):
    """Which elements stay: word e % 4 of the block e / 4 of element e, layer 0, is at least p 2^32."""
    low = 0xFFFFFFFF
    n = c["rows"] * c["width"]
    block = torch.arange(-(-n // 4), device=DEV)
    seed, step = s["seed"][0], s["seed"][1]
    words = _philox((block & low, block >> 32, (step & low).expand_as(block), torch.zeros_like(block)), (seed & low, (seed >> 32) & low))
    return torch.stack(words, 1).view(-1)[:n].view(c["rows"], c["width"]) >= round(c["p"] * 2 ** 32)


def _dropout_plain(s, c):
    kept = _kept(s, c)
    scale = 1.0 / (1.0 - round(c["p"] * 2 ** 32) / 2 ** 32)
    zero = torch.zeros((), device=DEV)
    x = s["x"].float()
    y = torch.where(kept, x * scale, zero)
    if c["residual"]:
        y = y + x
    y = y.to(s["x"].dtype)
    if c["pass"] == "fwd":
        return y
    dy = s["dY"].float()
    dx = torch.where(kept, dy * scale, zero)
    if c["residual"]:
        dx = dx + dy
    return {"y": y, "dX": dx.to(s["x"].dtype)}


# ------------------------------------------------------------------------------------------ work
def work(case):
    c = case
    step, elt, rows = c["pass"] == "step", 4 if c.get("dtype") == "f32" else 2, c["rows"]
    if c["op"] == "attention":
        width, out = (c["heads"] + 2 * c["kv"]) * c["dim"], c["heads"] * c["dim"]
        # pairs of rows that see one another, for sequences of the mean length
        length = (rows - c["pad"]) / c["seqs"]
        pairs = c["seqs"] * (length * (length + 1) / 2 if c["causal"] else length * length)
        products = 2 + 5 * step                                          # two forward, five backward
        return {"bytes": rows * (width + out) * 2 * (1 + step), "flops": products * 2.0 * pairs * c["heads"] * c["dim"]}
    if c["op"] == "rotary":
        width = (c["heads"] + 2 * c["kv"]) * c["dim"]
        pairs = rows * (c["heads"] + c["kv"]) * (c["s0"] + c["s1"] + c["s2"])
        return {"bytes": 2 * rows * width * elt * (1 + step) + 4 * rows * c["axes"], "flops": 6.0 * pairs * (1 + step)}
    if c["op"] == "gated":
        d, h = c["d"], c["hidden"]
        weights = 3 * d * h + 2 * h + d
        return {"bytes": (2 * rows * d * (1 + step) + weights * (1 + step)) * elt, "flops": 6.0 * rows * d * h * (1 + 2 * step)}
    n = rows * c["width"]
    return {"bytes": 2 * n * elt * (1 + step), "flops": 2.0 * n * (1 + step)}


# ------------------------------------------------------------------------------------------ the definition, in 64 bits
def exact(case, seed):
    """From the formulas, one sequence and head (or one piece) at a time; gradients by differentiating them."""
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    c = case
    return {"attention": _attention_exact, "rotary": _rotary_exact, "gated": _gated_exact, "dropout": _dropout_exact}[c["op"]](s, c)


def _attention_exact(s, c):
    heads, kv, dim, step = c["heads"], c["kv"], c["dim"], c["pass"] == "step"
    x = s["x"].double()
    y = torch.zeros(c["rows"], heads * dim, device=DEV, dtype=torch.float64)
    dx = torch.zeros_like(x) if step else None
    prefix = s["prefix"].tolist() if "prefix" in s else [0] * c["seqs"]
    for n, (b, e) in enumerate(zip(s["bounds"][:-1], s["bounds"][1:])):
        for r in range(b, e, 8192):                                      # rows of the sequence, 8192 at a time
            r1 = min(e, r + 8192)
            e1 = max(r1, min(e, b + prefix[n])) if c["causal"] else e      # keys behind are seen by none of these rows
            i, j = torch.arange(r, r1, device=DEV)[:, None], torch.arange(b, e1, device=DEV)[None]
            hidden = (j > i) & (j - b >= prefix[n]) if c["causal"] else None
            for h in range(heads):
                at_k, at_v = (heads + h // (heads // kv)) * dim, (heads + kv + h // (heads // kv)) * dim
                q = x[r:r1, h * dim:(h + 1) * dim].clone().requires_grad_(step)
                k = x[b:e1, at_k:at_k + dim].clone().requires_grad_(step)
                v = x[b:e1, at_v:at_v + dim].clone().requires_grad_(step)
                z = torch.einsum("id,jd->ij", q, k) / dim ** 0.5
                if c["cap"] > 0:
                    z = c["cap"] * torch.tanh(z / c["cap"])
                if c["bias"]:
                    z = z - s["slopes"][h].double() * (i - j).abs()
                if hidden is not None:
                    z = torch.where(hidden, torch.full((), -math.inf, device=DEV, dtype=torch.float64), z)
                o = torch.softmax(z, -1) @ v
                y[r:r1, h * dim:(h + 1) * dim] = o.detach()
                if step:
                    gq, gk, gv = torch.autograd.grad(o, (q, k, v), s["dY"][r:r1, h * dim:(h + 1) * dim].double())
                    dx[r:r1, h * dim:(h + 1) * dim] = gq
                    dx[b:e1, at_k:at_k + dim] += gk
                    dx[b:e1, at_v:at_v + dim] += gv
    return {"y": y, "dX": dx} if step else y


def _rotary_exact(s, c):
    """A pair as a complex number, turned by exp(i angle)."""
    axis, freq = _spectrum(c)
    n, blocks = len(axis), c["heads"] + c["kv"]
    angle = torch.stack([s["positions"][a].double() * f for a, f in zip(axis, freq)], 1)
    turn = torch.polar(torch.ones_like(angle), angle)[:, None]

    def apply(x, turn):
        out = x.double().clone().view(c["rows"], -1, c["dim"])
        part = out[:, :blocks, :2 * n]
        pair = part.reshape(c["rows"], blocks, n, 2) if c["adjacent"] else part.reshape(c["rows"], blocks, 2, n).transpose(2, 3)
        z = torch.complex(pair[..., 0].contiguous(), pair[..., 1].contiguous()) * turn
        pair = torch.stack([z.real, z.imag], -1)
        out[:, :blocks, :2 * n] = (pair if c["adjacent"] else pair.transpose(2, 3)).reshape(c["rows"], blocks, 2 * n)
        return out.view(c["rows"], -1)

    y = apply(s["x"], turn)
    return y if c["pass"] == "fwd" else {"y": y, "dX": apply(s["dY"], turn.conj())}


def _gated_exact(s, c):
    step = c["pass"] == "step"
    x, W1, b1, W2, b2 = (s[k].double().requires_grad_(step) for k in ("x", "W1", "b1", "W2", "b2"))
    gate, up = torch.addmm(b1, x, W1).split(c["hidden"], 1)
    act = {"silu": torch.nn.functional.silu, "relu": torch.relu,
           "gelu": lambda t: torch.nn.functional.gelu(t, approximate="tanh")}[c["act"]]
    y = torch.addmm(b2, act(gate) * up, W2)
    if not step:
        return y
    g = torch.autograd.grad(y, (x, W1, b1, W2, b2), s["dY"].double())
    new = [(w - LR * d).detach() for w, d in zip((W1, b1, W2, b2), g[1:])]
    return {"y": y.detach(), "dX": g[0], **dict(zip(WEIGHTS, new))}


def _dropout_exact(s, c):
    """The generator written out on 16-bit halves, so that no product leaves 53 bits; in pieces."""
    half = lambda v: (v // 65536, v % 65536)  # noqa: E731

    def product(m, v):
        (mh, ml), (vh, vl) = half(m), half(v)
        mid = mh * vl + (ml * vl) // 65536
        mid2 = ml * vh + mid % 65536
        return mh * vh + mid // 65536 + mid2 // 65536, (mid2 % 65536) * 65536 + (ml * vl) % 65536

    n = c["rows"] * c["width"]
    seed, step = (int(v) % 2 ** 64 for v in s["seed"].tolist())
    limit = round(c["p"] * 2 ** 32)
    kept = torch.empty(-(-n // 4) * 4, dtype=torch.bool, device=DEV)
    piece = 1 << 24
    for at in range(0, -(-n // 4), piece):
        block = torch.arange(at, min(-(-n // 4), at + piece), device=DEV)
        w = [block % 2 ** 32, block // 2 ** 32, torch.full_like(block, step % 2 ** 32), torch.zeros_like(block)]
        key = [seed % 2 ** 32, seed // 2 ** 32]
        for _ in range(10):
            h0, l0 = product(0xD2511F53, w[0])
            h1, l1 = product(0xCD9E8D57, w[2])
            w = [h1 ^ w[1] ^ key[0], l1, h0 ^ w[3] ^ key[1], l0]
            key = [(key[0] + 0x9E3779B9) % 2 ** 32, (key[1] + 0xBB67AE85) % 2 ** 32]
        kept[4 * at:4 * (at + len(block))] = (torch.stack(w, -1) >= limit).flatten()
    factor = kept[:n].view(c["rows"], c["width"]).double() / (1 - limit / 2 ** 32) + (1.0 if c["residual"] else 0.0)
    y = s["x"].double() * factor
    return y if c["pass"] == "fwd" else {"y": y, "dX": s["dY"].double() * factor}
