"""Cases for the operators that stand round a stack in a fine-tuning step on token sequences.

  policy      clipped policy loss with a KL term on the stack's output, loss and gradient (et_loss_policy_grad)
  score       log probabilities of given tokens under the stack's output (et_token_logp)
  preference  paired log-ratio loss over sequences, loss and gradient (et_loss_preference_grad)
  clip        global norm of the selected gradients, clipped copies of them (et_clip_grads)
  update      global norm, then the masked optimiser step on the clipped gradients (et_update_clipped)
  lookup      scaled embedding lookup, the first layer of a stack (ET_LAYER_EMBEDDING, et_forward_stack)
  embed       the lookup and the gradient of its table, exported or applied (et_backward_elastic)

`own` False: plain torch operations in 32 bits (64 where long sums or differences need them), rounded once.
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
        # a toy policy's update: few tokens, a small vocabulary, launch latency counts
        policy("policy-small-f32", rows=48, width=1000, dtype="f32", kl=0.05),
        # one micro-batch of rollouts, vocabulary padded to a multiple of 8 for the bf16 stack
        policy("policy-rollout", rows=4096, width=32008, vocab=32003, dtype="bf16", kl=0.02),
        # a large micro-batch under a large vocabulary
        policy("policy-large-vocab", rows=8192, width=131072, dtype="bf16", kl=0.02),
        # scoring a batch for the old or the reference log probabilities: forward only
        score("score-batch", rows=2048, width=50264, vocab=50257, dtype="bf16"),
        # a few short pairs in fp32, rows that start off every 16-byte boundary
        preference("preference-small-f32", pairs=3, length=24, width=4099, dtype="f32"),
        # pairs of ordinary length, ragged, prompts masked out
        preference("preference-batch", pairs=8, length=512, width=32000, dtype="bf16"),
        # a small network's gradients: latency of norm and clip together
        clip("clip-small", d=136, blocks=2, share=1.0),
        # 24 blocks of 1024 -> 4096 -> 1024, some of the tensors selected
        clip("clip-elastic", d=1024, blocks=24, share=0.4),
        # Adam on fp32 masters of a bf16 network, every tensor selected
        update("update-adam-master", d=1024, blocks=12, share=1.0, dtype="bf16", opt="adam"),
        # lookup of a batch of token sequences
        lookup("lookup-batch", rows=16384, vocab=32000, d=1024, dtype="bf16"),
        # a small fp32 table, widths that are no multiple of 16
        embed("embed-small-f32", rows=300, vocab=1000, d=200, dtype="f32", sgd=False),
        # a batch of token ids drawn as words are (few frequent, many rare), the gradient exported
        embed("embed-batch", rows=32768, vocab=65536, d=2048, dtype="bf16", sgd=False),
    ]


def policy(name, rows, width, dtype, kl, vocab=0, clip_high=0.2, scale=1.0, masked=0.15):
    return {"name": name, "op": "policy", "rows": rows, "width": width, "vocab": vocab, "dtype": dtype, "kl": kl,
            "clip_high": clip_high, "scale": scale, "masked": masked}


def score(name, rows, width, dtype, vocab=0, scale=1.0):
    return {"name": name, "op": "score", "rows": rows, "width": width, "vocab": vocab, "dtype": dtype, "scale": scale}


def preference(name, pairs, length, width, dtype, vocab=0, kind="sigmoid", smoothing=0.0, prompt=0.25):
    return {"name": name, "op": "preference", "pairs": pairs, "length": length, "width": width, "vocab": vocab, "dtype": dtype,
            "kind": kind, "smoothing": smoothing, "prompt": prompt}


def clip(name, d, blocks, share):
    return {"name": name, "op": "clip", "d": d, "blocks": blocks, "share": share}


def update(name, d, blocks, share, dtype, opt):
    return {"name": name, "op": "update", "d": d, "blocks": blocks, "share": share, "dtype": dtype, "opt": opt}


def lookup(name, rows, vocab, d, dtype):
    return {"name": name, "op": "lookup", "rows": rows, "vocab": vocab, "d": d, "dtype": dtype}


def embed(name, rows, vocab, d, dtype, sgd):
    return {"name": name, "op": "embed", "rows": rows, "vocab": vocab, "d": d, "dtype": dtype, "sgd": sgd}


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["policy", "score", "preference", "clip", "update", "lookup", "embed"])
    dtype = rng.choice(["f32", "bf16"])

    def width_vocab(hi):
        w = _log_int(rng, 500, hi)
        if dtype == "bf16":
            w = -(-w // 8) * 8
        return w, (0 if rng.random() < 0.5 else w - rng.randrange(1, 8))

    if op in ("policy", "score"):
        width, vocab = width_vocab(131072)
        rows = _log_int(rng, 1, min(16384, max(2, 400_000_000 // width)))
        if op == "score":
            c = score("", rows, width, dtype, vocab, rng.choice([1.0, 0.7, 1.25]))
        else:
            c = policy("", rows, width, dtype, rng.choice([0.0, 0.01, 0.1]), vocab, rng.choice([0.2, 0.28]), rng.choice([1.0, 0.8]),
                       rng.choice([0.0, 0.15, 0.5]))
    elif op == "preference":
        width, vocab = width_vocab(65536)
        pairs = _log_int(rng, 1, 24)
        length = _log_int(rng, 2, min(1024, max(3, 300_000_000 // (2 * pairs * width))))
        c = preference("", pairs, length, width, dtype, vocab, rng.choice(["sigmoid", "sigmoid", "ipo", "hinge"]), 0.0, rng.choice([0.0, 0.25, 0.5]))
        if c["kind"] == "sigmoid":
            c["smoothing"] = rng.choice([0.0, 0.1])
    elif op in ("clip", "update"):
        d = 8 * _log_int(rng, 4, 128)
        blocks = _log_int(rng, 1, 24 if op == "clip" else 12)
        share = rng.choice([0.2, 0.5, 1.0])
        c = clip("", d, blocks, share) if op == "clip" else update("", d, blocks, share, dtype, rng.choice(["sgd", "sgdw", "adam"]))
    else:
        vocab = _log_int(rng, 100, 131072)
        d = 8 * _log_int(rng, 4, 512)
        rows = _log_int(rng, 1, min(65536, max(2, 60_000_000 // d)))
        vocab = min(vocab, max(100, 100_000_000 // d))
        c = lookup("", rows, vocab, d, dtype) if op == "lookup" else embed("", rows, vocab, d, dtype, rng.random() < 0.5)
    del c["name"]
    return c


# ------------------------------------------------------------------------------------------ inputs
def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _rand(g, *shape):
    return torch.rand(*shape, generator=g, device=DEV)


def _randn(g, *shape, dtype=torch.float32):
    return torch.randn(*shape, generator=g, device=DEV, dtype=dtype)


def _zipf(g, rows, vocab):
    """Token ids with frequencies like 1 / rank, the ranks scattered over the vocabulary."""
    rank = torch.exp(_rand(g, rows).double() * math.log(vocab + 1.0)).long().clamp(1, vocab) - 1
    perm = torch.randperm(vocab, generator=g, device=DEV)
    return perm[rank].to(torch.int32)


def _logits(g, rows, width, dtype, targets):
    y = _randn(g, rows, width, dtype=dtype) * 2
    at = torch.arange(rows, device=DEV)
    y[at, targets.long()] += (4 + 3 * _randn(g, rows)).to(dtype)     # sampled tokens are likelier than others
    return y


def _vocab(c):
    return c["vocab"] or c["width"]


def _tensors(c):
    """Names and shapes of a network's tensors: norm, d -> 4 d, 4 d -> d per block; and which are selected."""
    shapes = []
    for _ in range(c["blocks"]):
        d = c["d"]
        shapes += [(d,), (d,), (d, 4 * d), (4 * d,), (4 * d, d), (d,)]
    n = len(shapes)
    chosen = [((7 * i) % n + 0.5) / n < c["share"] or i == n - 1 for i in range(n)]
    return shapes, chosen


def _flat(c):
    """Places of the selected tensors in one flat buffer (each on a multiple of 8 elements) and its length."""
    shapes, chosen = _tensors(c)
    at, places = 0, []
    for s, ch in zip(shapes, chosen):
        places.append(at if ch else None)
        if ch:
            at += -(-math.prod(s) // 8) * 8
    return shapes, chosen, places, at


def _pad_mask(c):
    shapes, chosen, places, n = _flat(c)
    m = torch.zeros(n, dtype=torch.bool, device=DEV)
    for s, p in zip(shapes, places):
        if p is not None:
            m[p:p + math.prod(s)] = True
    return m


def prepare(case, seed):
    c, g, op = case, _gen(seed), case["op"]
    s = {"c": c}
    if op in ("policy", "score", "preference"):
        dt, width, vocab = DTYPES[c["dtype"]], c["width"], _vocab(c)
        if op == "preference":
            lens = (c["length"] * (0.5 + 0.5 * _rand(g, 2 * c["pairs"]))).long().clamp(min=1)
            begin = torch.zeros(2 * c["pairs"] + 1, dtype=torch.int64, device=DEV)
            begin[1:] = torch.cumsum(lens, 0)
            rows = 2 * c["pairs"] * c["length"]                        # the batch's rows; those behind the last sequence are unused
            s["begin"] = begin.to(torch.int32)
        else:
            rows = c["rows"]
        s["targets"] = torch.randint(0, vocab, (rows,), generator=g, device=DEV, dtype=torch.int32)
        s["y"] = _logits(g, rows, width, dt, s["targets"])
        s["rows"] = rows
        if op == "policy":
            keep = (_rand(g, rows) >= c["masked"]).float()
            keep[0] = 1
            s["weights"] = keep / keep.sum().clamp(min=1)
            s["adv"] = _randn(g, rows)
            lp = _logp(s["y"], s["targets"], vocab, c["scale"])
            delta = 0.15 * _randn(g, rows)
            # ratios stay 1e-3 off the borders of the clipping range, where 32 bits could fall on either side
            for border in (math.log(0.8), math.log(1 + c["clip_high"])):
                near = (delta - border).abs() < 1e-3
                delta = torch.where(near, delta + 4e-3, delta)
            s["old"] = lp - delta
            s["ref"] = lp + 0.2 * _randn(g, rows)
            s["dY"] = torch.empty_like(s["y"])
            s["stats"] = torch.empty(4, device=DEV)
        if op in ("policy", "score"):
            s["logp"] = torch.empty(rows, device=DEV)
        if op == "preference":
            at = torch.arange(rows, device=DEV)
            seq = torch.bucketize(at, begin[1:], right=True).clamp(max=2 * c["pairs"] - 1)
            s["weights"] = ((at - begin[seq]).float() >= c["prompt"] * lens[seq].float()).float()
            used = torch.where(at < begin[-1], s["weights"], torch.zeros_like(s["weights"]))
            lp = _logp(s["y"], s["targets"], vocab, 1.0)
            sums = torch.zeros(2 * c["pairs"], device=DEV, dtype=torch.float64).index_add_(0, seq, lp.double() * used.double())
            s["ref"] = (sums + 3 * _randn(g, 2 * c["pairs"]).double()).float()
            s["dY"] = torch.empty_like(s["y"])
            s["stats"] = torch.empty(4, device=DEV)
            s["seq_logp"] = torch.empty(2 * c["pairs"], device=DEV)
        layers = [(8, width, 0, 1, -1)]
    elif op in ("clip", "update"):
        shapes, chosen, places, n = _flat(c)
        real = _pad_mask(c)
        s["grad"] = _randn(g, n) * 1e-3 * real
        # a clipping step: the norm is above the threshold, as it is in the steps that clipping is there for
        s["max_norm"] = 0.5e-3 * math.sqrt(sum(math.prod(sh) for sh, ch in zip(shapes, chosen) if ch))
        s["norm"] = torch.empty(2, device=DEV)
        if op == "clip":
            s["clipped"] = torch.zeros(n, device=DEV)
        else:
            s["w32"] = _randn(g, n) * 0.02 * real
            if c["dtype"] == "bf16":
                s["w"] = s["w32"].to(torch.bfloat16)
            if c["opt"] != "sgd":
                s["m"] = _randn(g, n) * 1e-4 * real
            if c["opt"] == "adam":
                s["v"] = _rand(g, n) * 1e-6 * real
        d = c["d"]
        layers = [(d, d, 0, 1, -1, 1, 1e-5), (d, 4 * d, 0, 1, -1), (4 * d, d, 0, 1, -1)] * c["blocks"]
    else:
        dt = DTYPES[c["dtype"]]
        s["ids"] = _zipf(g, c["rows"], c["vocab"])
        s["table"] = _randn(g, c["vocab"], c["d"], dtype=dt) * 0.02
        s["scale"] = math.sqrt(c["d"])
        s["y"] = torch.empty(c["rows"], c["d"], device=DEV, dtype=dt)
        if op == "embed":
            s["dY"] = _randn(g, c["rows"], c["d"], dtype=dt) * 1e-3
            if not c["sgd"]:
                s["grad"] = torch.empty(c["vocab"], c["d"], device=DEV)
        layers = [(c["vocab"], c["d"], 0, 1, -1, 5)]
    if own:
        _bind(s, layers)
    return s


LR = 1e-3
ADAM = {"beta1": 0.9, "beta2": 0.999, "eps": 1e-8}
SGDW = {"momentum": 0.9, "weight_decay": 5e-4}
KINDS = {"sigmoid": 0, "ipo": 1, "hinge": 2}
BETA = 0.1


def _bind(s, layers):
    """The stack a user keeps: created once, its tensors and workspace attached."""
    import numpy as np
    import paper_2312_14227_b200 as et
    c, op = s["c"], s["c"]["op"]
    storage = et.ET_BF16 if c.get("dtype") == "bf16" else et.ET_F32
    dt = torch.bfloat16 if storage == et.ET_BF16 else torch.float32
    rows = s["rows"] if op in ("policy", "score", "preference") else 8 if op in ("clip", "update") else c["rows"]
    stack = et.et_stack_create(layers, rows, storage)
    workspace = torch.empty(et.et_stack_workspace_bytes(stack), dtype=torch.uint8, device=DEV)
    if op in ("clip", "update"):
        shapes, chosen, places, n = _flat(c)
        idle = torch.zeros(4 * c["d"] * c["d"], device=DEV, dtype=dt)      # tensors that are not selected are not touched
        idle32 = torch.zeros(4 * c["d"] * c["d"], device=DEV)
        part = lambda buf, other, i: buf[places[i]:places[i] + math.prod(shapes[i])] if chosen[i] else other[:math.prod(shapes[i])]  # noqa: E731
        w = s.get("w", s.get("w32"))
        tensors = [idle[:math.prod(sh)] if w is None else part(w, idle, i) for i, sh in enumerate(shapes)]
        et.et_stack_bind(stack, tensors[0::2], tensors[1::2], workspace)
        s["mask"] = np.array(chosen, dtype=np.uint8)
        s["grads"] = [part(s["grad"], idle32, i) if chosen[i] else None for i in range(len(shapes))]
        if op == "clip":
            s["outs"] = [part(s["clipped"], idle32, i) if chosen[i] else None for i in range(len(shapes))]
        else:
            if dt == torch.bfloat16:
                masters = [part(s["w32"], idle32, i) for i in range(len(shapes))]
                et.et_stack_bind_master(stack, masters[0::2], masters[1::2])
            state = [[part(s[k], idle32, i) for i in range(len(shapes))] if k in s else None for k in ("m", "v")]
            if c["opt"] == "adam":
                et.et_stack_set_optimizer(stack, et.ET_OPT_ADAM, state[0], state[1], **ADAM)
                et.et_stack_set_optimizer_step(stack, 10)
            elif c["opt"] == "sgdw":
                et.et_stack_set_optimizer(stack, et.ET_OPT_SGDW, state[0], **SGDW)
    elif op in ("lookup", "embed"):
        et.et_stack_bind(stack, [s["table"]], [None], workspace)
        et.et_stack_set_embedding_scale(stack, s["scale"])
        s["mask"] = np.array([1, 0], dtype=np.uint8)
    else:
        w = torch.zeros(8 * c["width"], device=DEV, dtype=dt)
        et.et_stack_bind(stack, [w], [torch.zeros(c["width"], device=DEV, dtype=dt)], workspace)
    s["stack"] = stack


# ------------------------------------------------------------------------------------------ one pass
def run(state):
    s, c = state, state["c"]
    return (_run_own if own else _run_plain)(s, c, c["op"])


def _run_own(s, c, op):
    import paper_2312_14227_b200 as et
    if op == "score":
        et.et_token_logp(s["stack"], s["y"], s["targets"], s["logp"], vocab=c["vocab"], logit_scale=c["scale"])
        return s["logp"]
    if op == "policy":
        et.et_loss_policy_grad(s["stack"], s["y"], s["targets"], s["adv"], s["dY"], weights=s["weights"], logp_old=s["old"], logp_ref=s["ref"],
                               logp=s["logp"], loss_dev=s["stats"], vocab=c["vocab"], logit_scale=c["scale"], clip_low=0.2,
                               clip_high=c["clip_high"], kl_coef=c["kl"])
        return {"dY": s["dY"], "logp": s["logp"], "stats": s["stats"]}
    if op == "preference":
        et.et_loss_preference_grad(s["stack"], s["y"], s["targets"], s["begin"], s["dY"], weights=s["weights"], ref_logp=s["ref"],
                                   seq_logp=s["seq_logp"], loss_dev=s["stats"], kind=KINDS[c["kind"]], vocab=c["vocab"], beta=BETA,
                                   label_smoothing=c["smoothing"])
        return {"dY": s["dY"], "seq_logp": s["seq_logp"], "stats": s["stats"]}
    if op == "clip":
        et.et_clip_grads(s["stack"], s["mask"], s["grads"], s["outs"], s["max_norm"], s["norm"])
        return {"clipped": s["clipped"], "norm": s["norm"]}
    if op == "update":
        et.et_update_clipped(s["stack"], s["mask"], s["grads"], LR, s["max_norm"], s["norm"])
        return {k: s[k] for k in ("norm", "w", "w32", "m", "v") if k in s}
    et.et_forward_stack(s["stack"], s["ids"], s["y"])
    if op == "lookup":
        return s["y"]
    flags = et.ET_FLAG_FUSE_SGD if c["sgd"] else 0
    et.et_backward_elastic(s["stack"], s["dY"], s["mask"], None if c["sgd"] else [s["grad"], None], flags=flags, lr=LR)
    return {"y": s["y"], "table": s["table"]} if c["sgd"] else {"y": s["y"], "grad": s["grad"]}


def _logp(y, targets, vocab, scale):
    z = y[:, :vocab].float() * scale
    m = z.amax(1, keepdim=True)
    total = (z - m).exp_().sum(1)
    return z.gather(1, targets.long()[:, None])[:, 0] - m[:, 0] - total.log()


def _logit_grad(y, targets, vocab, scale, coef):
    """coef[row] * d logp[row] / d y, rounded once to y's type; rows whose coefficient is 0 and columns from vocab on get 0."""
    z = y[:, :vocab].float() * scale
    z -= z.amax(1, keepdim=True)
    p = z.exp_()
    p *= (-coef * scale / p.sum(1))[:, None]
    p[torch.arange(len(y), device=y.device), targets.long()] += coef * scale
    out = torch.zeros_like(y)
    out[:, :vocab] = torch.where((coef != 0)[:, None], p, torch.zeros((), device=y.device)).to(y.dtype)
    return out


def _run_plain(s, c, op):
    if op == "score":
        return _logp(s["y"], s["targets"], _vocab(c), c["scale"])
    if op == "policy":
        lp = _logp(s["y"], s["targets"], _vocab(c), c["scale"])
        w, a = s["weights"], s["adv"]
        live = w != 0
        r = (lp - s["old"]).exp()
        rc = r.clamp(1 - 0.2, 1 + c["clip_high"])
        clipped = r * a > rc * a
        d = s["ref"] - lp
        gain = torch.where(clipped, rc * a, r * a)
        kl = d.expm1() - d
        coef = w * (torch.where(clipped, torch.zeros_like(r), -a * r) - c["kl"] * d.expm1())
        coef = torch.where(live, coef, torch.zeros_like(coef))
        wd = w.double()
        parts = [-(wd * gain).sum(), (wd * kl).sum(), (wd * clipped).sum()]
        stats = torch.stack([parts[0] + c["kl"] * parts[1]] + parts).float()
        return {"dY": _logit_grad(s["y"], s["targets"], _vocab(c), c["scale"], coef), "logp": torch.where(live, lp, torch.zeros_like(lp)), "stats": stats}
    if op == "preference":
        return _preference_plain(s, c)
    if op in ("clip", "update"):
        norm = s["grad"].double().square().sum().sqrt()
        coef = (s["max_norm"] / norm).clamp(max=1.0)
        report = torch.stack([norm, coef]).float()
        g = s["grad"] * coef.float()
        if op == "clip":
            return {"clipped": g, "norm": report}
        return {"norm": report, **_step_plain(s, c, g)}
    ids = s["ids"].long()
    y = (s["table"][ids].float() * s["scale"]).to(s["table"].dtype)
    if op == "lookup":
        return y
    grad = torch.zeros(c["vocab"], c["d"], device=DEV).index_add_(0, ids, s["dY"].float()) * s["scale"]
    if not c["sgd"]:
        return {"y": y, "grad": grad}
    s["table"].copy_(s["table"].float() - LR * grad)
    return {"y": y, "table": s["table"]}


def _step_plain(s, c, g):
    w = s["w32"]
    if c["opt"] == "sgd":
        w.sub_(LR * g)
    elif c["opt"] == "sgdw":
        s["m"].mul_(SGDW["momentum"]).add_(LR * g)
        w.copy_(w - s["m"] - SGDW["weight_decay"] * w)
    else:
        s["m"].copy_(ADAM["beta1"] * s["m"] + (1 - ADAM["beta1"]) * g)
        s["v"].copy_(ADAM["beta2"] * s["v"] + (1 - ADAM["beta2"]) * g * g)
        c1, c2 = 1 / (1 - ADAM["beta1"] ** 10), 1 / (1 - ADAM["beta2"] ** 10)
        w.sub_(LR * (s["m"] * c1) / ((s["v"] * c2).sqrt() + ADAM["eps"]))
    if "w" in s:
        s["w"].copy_(w)
    return {k: s[k] for k in ("w", "w32", "m", "v") if k in s}


def _preference_plain(s, c):
    lp = _logp(s["y"], s["targets"], _vocab(c), 1.0).double()
    begin, n = s["begin"].long(), 2 * c["pairs"]
    at = torch.arange(s["rows"], device=DEV)
    inside = at < begin[-1]
    seq = torch.bucketize(at, begin[1:], right=True).clamp(max=n - 1)
    w = torch.where(inside, s["weights"], torch.zeros_like(s["weights"])).double()
    sums = torch.zeros(n, device=DEV, dtype=torch.float64).index_add_(0, seq, torch.where(w != 0, w * lp, torch.zeros_like(lp)))
    loss, slope, stats = _pair_loss(sums, s["ref"].double(), c)
    coef = torch.where(w != 0, w * slope[seq], torch.zeros_like(w)).float()
    return {"dY": _logit_grad(s["y"], s["targets"], _vocab(c), 1.0, coef), "seq_logp": sums.float(), "stats": stats.float()}


def _pair_loss(sums, ref, c):
    """Loss, its slope for each sequence's log probability, and the reported numbers; 64 bits."""
    reward = BETA * (sums - ref)
    chosen, rejected = reward[0::2], reward[1::2]
    x, e = chosen - rejected, c["smoothing"]
    if c["kind"] == "sigmoid":
        each = (1 - e) * torch.log1p(torch.exp(-x.abs())) + e * torch.log1p(torch.exp(-x.abs())) + (1 - e) * (-x).clamp(min=0) + e * x.clamp(min=0)
        dx = e / (1 + torch.exp(-x)) - (1 - e) / (1 + torch.exp(x))
    elif c["kind"] == "ipo":
        each = (x / BETA - 1 / (2 * BETA)) ** 2
        dx = 2 * (x / BETA - 1 / (2 * BETA)) / BETA
    else:
        each = (1 - x).clamp(min=0)
        dx = -(x < 1).double()
    slope = torch.stack([dx, -dx], 1).reshape(-1) * BETA / c["pairs"]
    return each.mean(), slope, torch.stack([each.mean(), chosen.mean(), rejected.mean(), (x > 0).double().mean()])


# ------------------------------------------------------------------------------------------ work
def work(case):
    c, op = case, case["op"]
    e = 2 if c.get("dtype") == "bf16" else 4
    if op == "policy":
        n = c["rows"] * c["width"]
        return {"bytes": n * e * (2 - c["masked"]) + c["rows"] * 28, "flops": 8 * n * (1 - c["masked"])}
    if op == "score":
        return {"bytes": c["rows"] * (_vocab(c) * e + 8), "flops": 4 * c["rows"] * _vocab(c)}
    if op == "preference":
        n = 2 * c["pairs"] * c["length"] * c["width"]
        live = 0.75 * (1 - c["prompt"])                               # sequences are 3/4 of the longest on average
        return {"bytes": n * e * (1 + live), "flops": 8 * n * live}
    if op in ("clip", "update"):
        shapes, chosen, places, n = _flat(c)
        if op == "clip":
            return {"bytes": 8 * n, "flops": 3 * n}
        per = 4 + 8 + (2 if e == 2 else 0) + {"sgd": 0, "sgdw": 8, "adam": 16}[c["opt"]]
        return {"bytes": per * n, "flops": n * {"sgd": 5, "sgdw": 7, "adam": 16}[c["opt"]]}
    # distinct ids among `rows` draws whose frequencies fall like 1 / rank
    h = math.log(c["vocab"] + 1.0)
    top = min(c["vocab"], 4096)
    distinct = sum(1 - math.exp(-c["rows"] * math.log1p(1.0 / k) / h) for k in range(1, top + 1))
    k = top
    while k < c["vocab"]:
        step = min(1024, c["vocab"] - k)
        distinct += step * (1 - math.exp(-c["rows"] * math.log1p(1.0 / (k + step / 2)) / h))
        k += step
    n, t = c["rows"] * c["d"], distinct * c["d"]
    total = t * e + n * e + 4 * c["rows"]
    if op == "embed":
        total += n * e + (2 * t * e if c["sgd"] else 4 * c["vocab"] * c["d"])
    return {"bytes": total, "flops": n if op == "lookup" else 3 * n}


# ------------------------------------------------------------------------------------------ 64 bits
def exact(case, seed):
    global own
    kept, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = kept
    c, op = case, case["op"]
    if op in ("policy", "score", "preference"):
        return _exact_tokens(s, c, op)
    if op in ("clip", "update"):
        g = s["grad"].double()
        norm = torch.linalg.vector_norm(g)
        k = torch.minimum(torch.ones_like(norm), s["max_norm"] / norm)
        g, report = g * k, torch.stack([norm, k])
        if op == "clip":
            return {"clipped": g, "norm": report}
        out, w = {"norm": report}, s["w32"].double()
        if c["opt"] == "sgd":
            w = w - LR * g
        elif c["opt"] == "sgdw":
            out["m"] = 0.9 * s["m"].double() + LR * g
            w = w - out["m"] - 5e-4 * w
        else:
            b1, b2 = 0.9, 0.999
            out["m"] = b1 * s["m"].double() + (1 - b1) * g
            out["v"] = b2 * s["v"].double() + (1 - b2) * g ** 2
            w = w - LR * (out["m"] / (1 - b1 ** 10)) / (torch.sqrt(out["v"] / (1 - b2 ** 10)) + 1e-8)
        out["w32"] = w
        if "w" in s:
            out["w"] = w
        return out
    table, ids = s["table"].double(), s["ids"].long()
    y = table[ids] * s["scale"]
    if op == "lookup":
        return y
    order = torch.argsort(ids, stable=True)
    run_sum = torch.cat([torch.zeros(1, c["d"], device=DEV, dtype=torch.float64), torch.cumsum(s["dY"].double()[order], 0)])
    ends = torch.searchsorted(ids[order].contiguous(), torch.arange(c["vocab"] + 1, device=DEV))
    grad = (run_sum[ends[1:]] - run_sum[ends[:-1]]) * s["scale"]
    return {"y": y, "grad": grad} if not c["sgd"] else {"y": y, "table": table - LR * grad}


def _exact_tokens(s, c, op):
    scale = c.get("scale", 1.0)
    rows, width, vocab = s["rows"], c["width"], _vocab(c)
    step = max(1, 100_000_000 // width)
    t = s["targets"].long()[:, None]
    lp = torch.empty(rows, dtype=torch.float64, device=DEV)
    for i in range(0, rows, step):
        z = scale * s["y"][i:i + step, :vocab].double()
        lp[i:i + step] = z.gather(1, t[i:i + step])[:, 0] - torch.logsumexp(z, 1)
    if op == "score":
        return lp
    out = {}
    if op == "policy":
        w, a = s["weights"].double(), s["adv"].double()
        r = torch.exp(lp - s["old"].double())
        d = s["ref"].double() - lp
        lo, hi = 1 - 0.2, 1 + c["clip_high"]
        surrogate = torch.minimum(r * a, torch.clamp(r, lo, hi) * a)
        off = ((a > 0) & (r > hi)) | ((a < 0) & (r < lo))
        kl = torch.exp(d) - 1 - d
        coef = w * (-a * r * (~off) - c["kl"] * (torch.exp(d) - 1))
        first, second = -(w * surrogate).sum(), (w * kl).sum()
        out["stats"] = torch.stack([first + c["kl"] * second, first, second, (w * off).sum()])
        out["logp"] = lp * (w != 0)
    else:
        b = s["begin"].tolist()
        w = s["weights"].double().clone()
        w[b[-1]:] = 0
        sums = torch.stack([(w[b[q]:b[q + 1]] * lp[b[q]:b[q + 1]]).sum() for q in range(2 * c["pairs"])])
        reward = BETA * (sums - s["ref"].double())
        x = reward[0::2] - reward[1::2]
        x = x.clone().requires_grad_(True)
        if c["kind"] == "sigmoid":
            f = torch.nn.functional.logsigmoid
            each = -(1 - c["smoothing"]) * f(x) - c["smoothing"] * f(-x)
        elif c["kind"] == "ipo":
            each = (x / BETA - 0.5 / BETA) ** 2
        else:
            each = torch.relu(1 - x)
        each.mean().backward()
        coef = torch.zeros_like(w)
        for p in range(c["pairs"]):
            for q, sign in ((2 * p, 1.0), (2 * p + 1, -1.0)):
                coef[b[q]:b[q + 1]] = sign * BETA * x.grad[p] * w[b[q]:b[q + 1]]
        out["seq_logp"] = sums
        out["stats"] = torch.stack([each.detach().mean(), reward[0::2].mean(), reward[1::2].mean(), (x.detach() > 0).double().mean()])
    grad = torch.zeros(rows, width, dtype=torch.float64, device=DEV)
    for i in range(0, rows, step):
        z = scale * s["y"][i:i + step, :vocab].double()
        p = torch.softmax(z, 1)
        k = coef[i:i + step, None] * scale
        grad[i:i + step, :vocab] = -k * p
        grad[i:i + step].scatter_add_(1, t[i:i + step], k)
    out["dY"] = grad
    return out
