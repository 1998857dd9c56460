"""Timed operators of preference tuning with low-rank adapters: the parts of one
such step that the framework's kernels compute, each through its public entry
point and in a plain form of elementary torch operations.

  adapters    ClientAdapters: every client's own low-rank pair beside a
              projection that all clients share.  Forward
                  v_t = A_s x_t,  y_t = base_t + scale B_s v_t
              (s: the slot of row t's client; no slot: y_t = base_t, v_t = 0)
              and backward
                  dv_t = scale B_s^T dy_t,  dx_t = dres_t + A_s^T dv_t,
                  dA_s = sum_t dv_t x_t^T,  dB_s = scale sum_t dy_t v_t^T
  preference  PreferenceLoss: sequences 2p (preferred) and 2p + 1 (rejected),
                  l_s = sum over labelled t of (x_t[label] - logsumexp(x_t)),
                  z_p = beta ((l_2p - ref_2p) - (l_2p+1 - ref_2p+1)),
                  L_p = (1 - eps) softplus(-z_p) + eps softplus(z_p)
              and the gradient of g sum_p L_p by the logits
  clip        GradNorm: n = sqrt(sum of all squares), c = min(1, m / (n + 1e-6)),
              every gradient times c

prepare() draws what a program holds before the call, run() makes one pass,
exact() computes the outputs from the definitions in float64.  Where `own` is
true run() calls the framework's operators, else it computes the plain form.
"""

from __future__ import annotations

import math
import random

import torch

own = False

VOCAB = 130528   # ChatGLM-6B's tokenizer
ROUNDING = 8     # elements: views of a flat buffer start 16-byte aligned
# hidden, FFN width
SHAPES = {"chatglm6b": (4096, 16384), "h1280": (1280, 3328), "h256": (256, 1024)}


def _adapters(name, what, dims, rank, clients, per_client, lens, **kw):
    c = dict(name=name, kind="adapters", what=what, inn=dims[0], out=dims[1], rank=rank, clients=clients,
             per_client=per_client, min_len=lens[0], max_len=lens[1], len_seed=0, slots=clients, bare=0, dtype="bf16")
    c.update(kw)
    return c


def _preference(name, train, pairs, lens, **kw):
    c = dict(name=name, kind="preference", train=train, pairs=pairs, min_len=lens[0], max_len=lens[1], len_seed=0,
             vocab=VOCAB, pad=0, dtype="bf16", beta=0.1, smoothing=0.0, ref=True, masked=0, empty=False)
    c.update(kw)
    return c


def _clip(name, layout, shape, layers, width, **kw):
    c = dict(name=name, kind="clip", layout=layout, shape=shape, layers=layers, width=width, max_norm=1.0,
             dtype="f32")
    c.update(kw)
    return c


def listed():
    qkv = (4096, 12288)  # the fused query / key / value projection at hidden 4096
    return [
        # one client generating: its one new token through its own rank-8 pair
        _adapters("adapters_one_token", "fwd", qkv, 8, 1, 1, (1, 1)),
        # 64 clients generating, one token each; some without an adapter
        _adapters("adapters_64_tokens", "fwd", qkv, 16, 64, 1, (1, 1), bare=6),
        # short ragged prompts of a small model; clients that share adapters
        _adapters("adapters_prompts_h1280", "fwd", (1280, 3840), 24, 8, 1, (1, 257), slots=3, len_seed=1),
        # a training forward over long contexts, 32 clients
        _adapters("adapters_fwd_32x1", "fwd", qkv, 16, 32, 1, (512, 2048)),
        # fp32 debug mode of a small model, odd lengths: forward's and backward's launches
        _adapters("adapters_bwd_f32_h256", "bwd", (256, 768), 8, 3, 2, (5, 131), dtype="f32", len_seed=2),
        # a training backward: 8 clients with 4 sequences each, rank 32
        _adapters("adapters_bwd_8x4", "bwd", qkv, 32, 8, 4, (128, 1024)),
        # the largest: the backward over long contexts, 32 clients
        _adapters("adapters_bwd_32x1", "bwd", qkv, 16, 32, 1, (512, 2048)),
        # log-probabilities of one short pair under the frozen reference model
        _preference("preference_reference_pair", False, 1, (37, 61), ref=False),
        # fp32 debug mode: small vocabulary, padded rows, masked ids, a sequence without labels
        _preference("preference_f32_small", True, 3, (9, 70), vocab=1000, pad=24, dtype="f32", smoothing=0.1,
                    masked=8, empty=True, len_seed=1),
        # a training step's loss and gradient: 8 pairs of answers to ordinary prompts
        _preference("preference_train_8", True, 8, (128, 512), len_seed=2),
        # clipping the adapters' gradients of 26 blocks (52 small tensors)
        _clip("clip_adapters_26", "adapters", "chatglm6b", 26, 16),
        # clipping two blocks' full fine-tuning gradients (24 tensors, 0.4 G elements)
        _clip("clip_blocks_2", "blocks", "chatglm6b", 2, 0),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng: random.Random):
    what = rng.choice(("tokens", "prompts", "fwd", "bwd", "bwd", "adapters_f32", "reference", "train", "loss_f32",
                       "clip", "clip"))
    seed = rng.randrange(1 << 16)
    dims = rng.choice(((4096, 12288), (4096, 4096), (1280, 3840), (1280, 1280), (256, 768), (520, 1032)))
    rank = 8 * rng.choice((1, 1, 2, 2, 3, 4, 5, 6, 8))
    if what == "tokens":
        clients = _log_uniform(rng, 1, 256)
        c = _adapters("", "fwd", dims, rank, clients, 1, (1, 1), bare=rng.randint(0, clients // 4))
    elif what in ("prompts", "fwd", "bwd"):
        clients, per = rng.choice(((1, 1), (2, 1), (3, 2), (4, 2), (8, 1), (8, 4), (16, 1), (24, 1)))
        longest = 300 if what == "prompts" else 1100
        lens = sorted((_log_uniform(rng, 1, longest), _log_uniform(rng, 1, longest)))
        c = _adapters("", "bwd" if what == "bwd" else "fwd", dims, rank, clients, per, lens)
        c["slots"] = rng.randint(1, clients)
        c["bare"] = rng.choice((0, 0, clients // 4))
    elif what == "adapters_f32":
        dims = rng.choice(((1280, 3840), (256, 768), (256, 1024), (520, 1032)))
        clients = rng.randint(1, 8)
        lens = sorted((_log_uniform(rng, 1, 300), _log_uniform(rng, 1, 300)))
        c = _adapters("", rng.choice(("fwd", "bwd")), dims, rank, clients, 1, lens, dtype="f32",
                      slots=rng.randint(1, clients))
    elif what == "reference":
        c = _preference("", False, _log_uniform(rng, 1, 16), sorted((_log_uniform(rng, 2, 300),
                                                                     _log_uniform(rng, 2, 300))), ref=False)
        c["vocab"] = rng.choice((VOCAB, 65024, 32000, 8200))
    elif what == "train":
        c = _preference("", True, _log_uniform(rng, 1, 12), sorted((_log_uniform(rng, 2, 300),
                                                                    _log_uniform(rng, 2, 300))))
        c["vocab"] = rng.choice((VOCAB, 65024, 32000, 8200))
        c["pad"] = rng.choice((0, 32, 224))
        c["beta"], c["smoothing"] = rng.choice((0.05, 0.1, 0.3)), rng.choice((0.0, 0.0, 0.1))
        c["empty"] = rng.random() < 0.2
    elif what == "loss_f32":
        c = _preference("", rng.random() < 0.7, rng.randint(1, 40), sorted((_log_uniform(rng, 2, 90),
                                                                            _log_uniform(rng, 2, 90))), dtype="f32")
        c["vocab"] = 8 * rng.randint(8, 1000)
        c["pad"] = 8 * rng.randint(0, 4)
        c["masked"] = rng.choice((0, 8, 40))
    else:
        layout = rng.choice(("adapters", "prefix", "blocks", "ragged"))
        shape = rng.choice(("chatglm6b", "h1280", "h256"))
        layers = rng.randint(1, 26)
        if layout == "blocks" and shape == "chatglm6b":
            layers = 1
        width = {"adapters": rank, "prefix": rng.choice((16, 64, 100, 128)), "blocks": 0,
                 "ragged": _log_uniform(rng, 3, 200000)}[layout]
        c = _clip("", layout, shape, layers, width, max_norm=rng.choice((0.1, 1.0, 1.0, 1e4)),
                  dtype=rng.choice(("f32", "f32", "bf16")))
    if "len_seed" in c:
        c["len_seed"] = seed
    del c["name"]
    return c


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------

def _tdt(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _randn(g, shape, dtype, std=1.0):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).mul_(std).to(dtype)


def _bounds(lens):
    cu = [0]
    for n in lens:
        cu.append(cu[-1] + n)
    return cu


def _adapter_batch(c):
    """(row bounds of the sequences, sequence bounds of the clients, each client's slot or -1)."""
    g = random.Random(c["len_seed"])
    lens = [g.randint(c["min_len"], c["max_len"]) for _ in range(c["clients"] * c["per_client"])]
    slot = [i % c["slots"] for i in range(c["clients"])]
    g.shuffle(slot)
    for i in g.sample(range(c["clients"]), c["bare"]):
        slot[i] = -1
    return _bounds(lens), [i * c["per_client"] for i in range(c["clients"] + 1)], slot


def _client_rows(c):
    """The first row of each client, and the end of the last."""
    cu, csp, _ = _adapter_batch(c)
    return [cu[s] for s in csp]


def _prepare_adapters(c, seed):
    cu, csp, slot = _adapter_batch(c)
    T, r, inn, out, n = cu[-1], c["rank"], c["inn"], c["out"], c["slots"]
    g, dt = _gen(seed), _tdt(c)
    s = {"case": c, "scale": 2.0, "slot": slot,
         "x": _randn(g, (T, inn), dt), "a": _randn(g, (n, r, inn), dt, inn ** -0.5), "b": _randn(g, (n, out, r), dt, 0.02),
         "rows": torch.tensor(_client_rows(c), device="cuda"), "slots": torch.tensor(slot, device="cuda"),
         "longest": max(b - a for a, b in zip(_client_rows(c), _client_rows(c)[1:]))}
    if c["what"] == "fwd":
        s["base"] = _randn(g, (T, out), dt)
        s["y"] = torch.empty_like(s["base"])
        s["v"] = torch.empty((T, r), dtype=torch.float32, device="cuda")
    else:
        s["dy"], s["dres"] = _randn(g, (T, out), dt, 0.01), _randn(g, (T, inn), dt, 0.01)
        s["v"] = torch.zeros((T, r), dtype=torch.float32, device="cuda")
        rows = _client_rows(c)
        for i, k in enumerate(slot):
            if k >= 0:
                s["v"][rows[i]:rows[i + 1]] = s["x"][rows[i]:rows[i + 1]].float() @ s["a"][k].float().t()
        s["dx"] = torch.empty_like(s["x"])
        s["da"] = torch.empty((n, r, inn), dtype=torch.float32, device="cuda")
        s["db"] = torch.empty((n, out, r), dtype=torch.float32, device="cuda")
    if own:  # the descriptor, handle and workspace that a program keeps beside its batch
        from paper_2406_14898_amd import BatchDesc, ClientAdapters
        s["batch"] = BatchDesc(cu, csp)
        s["op"] = ClientAdapters(n, r, inn, out, c["dtype"], s["scale"])
        s["ws"] = s["op"].workspace(s["batch"])
    return s


def _labels(c):
    """(row bounds, labels): the first quarter of a sequence is its prompt, the last token has no next one."""
    g = random.Random(c["len_seed"])
    lens = [g.randint(c["min_len"], c["max_len"]) for _ in range(2 * c["pairs"])]
    cu, lab = _bounds(lens), []
    for i, n in enumerate(lens):
        bare = c["empty"] and i == 1
        lab += [-100 if bare or t < n // 4 or t == n - 1 else g.randrange(c["vocab"] - c["masked"]) for t in range(n)]
    return cu, lab


def _prepare_preference(c, seed):
    cu, lab = _labels(c)
    T, V, g, dt = cu[-1], c["vocab"], _gen(seed), _tdt(c)
    std = 1.5
    s = {"case": c, "grad_scale": 1.0 / c["pairs"], "logits": _randn(g, (T, V + c["pad"]), dt, std),
         "labels": torch.tensor(lab, dtype=torch.int32, device="cuda"), "ref": None,
         "cu": torch.tensor(cu, device="cuda")}
    if c["masked"]:
        s["logits"][:, V - c["masked"]:V] = -math.inf
    # the inputs differ by seed in their labels too
    shift = torch.randint(0, V - c["masked"], (T,), generator=g, device="cuda", dtype=torch.int32)
    s["labels"] = torch.where(s["labels"] >= 0, (s["labels"] + shift) % (V - c["masked"]), s["labels"])
    if c["ref"]:
        count = torch.tensor([sum(1 for x in lab[a:b] if x >= 0) for a, b in zip(cu, cu[1:])], device="cuda")
        mean = -count * (math.log(V) + std * std / 2)
        s["ref"] = (mean + 5.0 * torch.randn(2 * c["pairs"], generator=g, device="cuda")).float()
    if own:  # the batch, handle, workspace and outputs that a program keeps
        from paper_2406_14898_amd import BatchDesc, PreferenceLoss
        s["batch"] = BatchDesc(cu, [0, 2 * c["pairs"]])
        s["op"] = PreferenceLoss(V, c["dtype"], c["beta"], c["smoothing"])
        s["ws"] = s["op"].workspace(s["batch"])
    f = dict(dtype=torch.float32, device="cuda")
    s["logp"], s["loss"], s["total"] = (torch.empty(n, **f) for n in (2 * c["pairs"], c["pairs"], 1))
    if c["train"]:
        s["dlogits"] = torch.empty_like(s["logits"])
    return s


def _sizes(c):
    H, ffn = SHAPES[c["shape"]]
    if c["layout"] == "adapters":
        one = [c["width"] * H, 3 * H * c["width"]]
    elif c["layout"] == "prefix":
        one = [c["width"] * H, c["width"] * H]
    elif c["layout"] == "blocks":
        one = [3 * H * H, 3 * H, H * H, H, ffn * H, ffn, H * ffn, H, H, H, H, H]
    else:  # any sizes, one element and none among them
        w = c["width"]
        return [max(0, (w * (i * i + 1)) % (2 * w + 1) - (i == 3) * 2 * w) if i != 1 else 1 for i in range(2 * c["layers"])]
    return one * c["layers"]


def _views(flat, c):
    out, off = [], 0
    for n in _sizes(c):
        out.append(flat[off:off + n])
        off += -(-n // ROUNDING) * ROUNDING
    return out


def _clip_inputs(c, seed):
    n = sum(-(-k // ROUNDING) * ROUNDING for k in _sizes(c))
    flat = _randn(_gen(seed), (max(n, ROUNDING),), _tdt(c), 0.01)
    return flat, _views(flat, c)


def _prepare_clip(c, seed):
    flat, grads = _clip_inputs(c, seed)
    s = {"case": c, "grads": grads, "flat": torch.zeros_like(flat)}
    s["clipped"] = _views(s["flat"], c)
    if own:  # the handle with its workspace
        from paper_2406_14898_amd import GradNorm
        s["op"] = GradNorm(grads)
    return s


def prepare(case, seed):
    return {"adapters": _prepare_adapters, "preference": _prepare_preference,
            "clip": _prepare_clip}[case["kind"]](case, seed)


# ---------------------------------------------------------------------------
# One pass: the framework's operators
# ---------------------------------------------------------------------------

def _own_adapters(s):
    op = s["op"]
    if s["case"]["what"] == "fwd":
        op.forward(s["batch"], s["slot"], s["x"], s["a"], s["b"], s["base"], s["y"], s["v"], s["ws"])
        return {"y": s["y"], "v": s["v"]}
    s["da"].zero_()  # gradients accumulate
    s["db"].zero_()
    op.backward(s["batch"], s["slot"], s["dy"], s["x"], s["a"], s["b"], s["v"], s["dres"], s["dx"], s["da"], s["db"],
                s["ws"])
    return {"dx": s["dx"], "da": s["da"], "db": s["db"]}


def _own_preference(s):
    op = s["op"]
    op.forward(s["batch"], s["logits"], s["labels"], s["ref"], s["logp"], s["loss"], s["total"], s["ws"])
    out = {"logp": s["logp"], "loss": s["loss"], "total": s["total"]}
    if s["case"]["train"]:
        op.backward(s["batch"], s["logits"], s["labels"], s["grad_scale"], s["dlogits"], s["ws"])
        out["dlogits"] = s["dlogits"]
    return out


def _own_clip(s):
    norm = s["op"].clip(s["case"]["max_norm"], out=s["clipped"])
    return {"norm": norm, "grads": s["flat"]}


# ---------------------------------------------------------------------------
# One pass: the plain forms
# ---------------------------------------------------------------------------

def _padded(s, rows):
    """Clients' rows side by side, [clients, longest, width] in fp32, zero past a client's end."""
    at = s["rows"][:-1, None] + torch.arange(s["longest"], device="cuda")
    inside = at < s["rows"][1:, None]
    return rows.float()[at.clamp(max=rows.shape[0] - 1)] * inside[..., None]


def _packed(s, padded, T):
    """Back to the packed rows."""
    t = torch.arange(T, device="cuda")
    client = torch.searchsorted(s["rows"], t, right=True) - 1
    return padded[client, t - s["rows"][client]]


def _plain_adapters(s):
    c, T, dt = s["case"], s["x"].shape[0], s["x"].dtype
    has = (s["slots"] >= 0).float()[:, None, None]
    a = s["a"].float()[s["slots"].clamp(min=0)] * has
    b = s["b"].float()[s["slots"].clamp(min=0)] * has
    x = _padded(s, s["x"])
    if c["what"] == "fwd":
        v = torch.bmm(x, a.transpose(1, 2).contiguous())
        d = torch.bmm(v, b.transpose(1, 2).contiguous())
        return {"y": (s["base"].float() + s["scale"] * _packed(s, d, T)).to(dt), "v": _packed(s, v, T)}
    dy, v = _padded(s, s["dy"]), _padded(s, s["v"])
    dv = s["scale"] * torch.bmm(dy, b)
    dx = s["dres"].float() + _packed(s, torch.bmm(dv, a), T)
    da = torch.bmm(dv.transpose(1, 2).contiguous(), x) * has
    db = s["scale"] * torch.bmm(dy.transpose(1, 2).contiguous(), v) * has
    n = s["a"].shape[0]
    pick = (torch.arange(n, device="cuda")[:, None] == s["slots"]).float()  # slots x clients
    return {"dx": dx.to(dt), "da": (pick @ da.reshape(da.shape[0], -1)).view(n, *da.shape[1:]),
            "db": (pick @ db.reshape(db.shape[0], -1)).view(n, *db.shape[1:])}


def _plain_preference(s):
    c, V = s["case"], s["case"]["vocab"]
    x = s["logits"][:, :V].float()
    top = x.max(1, keepdim=True).values
    e = torch.exp(x - top)
    total = e.sum(1, keepdim=True)
    has = s["labels"] >= 0
    lab = s["labels"].clamp(min=0).long()[:, None]
    tok = (x.gather(1, lab) - top).double() - total.double().log()
    T, S = x.shape[0], 2 * c["pairs"]
    seq = torch.searchsorted(s["cu"], torch.arange(T, device="cuda"), right=True) - 1
    mine = (torch.arange(S, device="cuda")[:, None] == seq) & has
    logp = torch.where(mine, tok[:, 0], 0.0).sum(1)
    d = logp if s["ref"] is None else logp - s["ref"].double()
    z = c["beta"] * (d[0::2] - d[1::2])
    soft = lambda u: torch.clamp(u, min=0) + torch.log1p(torch.exp(-u.abs()))  # noqa: E731
    loss = (1 - c["smoothing"]) * soft(-z) + c["smoothing"] * soft(z)
    out = {"logp": logp.float(), "loss": loss.float(), "total": loss.sum().reshape(1).float()}
    if c["train"]:
        dz = (c["smoothing"] - 1) / (1 + torch.exp(z)) + c["smoothing"] / (1 + torch.exp(-z))
        k = (s["grad_scale"] * c["beta"] * torch.stack([dz, -dz], 1).reshape(-1))[seq] * has
        p = e.mul_((-k / total[:, 0]).float()[:, None])
        p.scatter_add_(1, lab, k.float()[:, None])
        s["dlogits"][:, :V] = p
        s["dlogits"][:, V:] = 0
        out["dlogits"] = s["dlogits"]
    return out


def _plain_clip(s):
    # squares in 64 bits: their sums are long
    norm = sum((g.double() * g.double()).sum() for g in s["grads"]).sqrt()
    k = torch.clamp(s["case"]["max_norm"] / (norm + 1e-6), max=1.0).float()
    _ = [o.copy_(g.float() * k) for g, o in zip(s["grads"], s["clipped"])]
    return {"norm": norm.float().reshape(1), "grads": s["flat"]}


def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"adapters": _own_adapters, "preference": _own_preference, "clip": _own_clip}[kind](state)
    return {"adapters": _plain_adapters, "preference": _plain_preference, "clip": _plain_clip}[kind](state)


def work(case):
    """Each input once, each output once."""
    c = case
    e = 4.0 if c["dtype"] == "f32" else 2.0
    if c["kind"] == "clip":
        n = sum(_sizes(c))
        return {"bytes": 2 * e * n, "flops": 3.0 * n}
    if c["kind"] == "preference":
        cu, lab = _labels(c)
        T, L, V = cu[-1], sum(1 for x in lab if x >= 0), c["vocab"]
        # a row without a label has no part in the loss: its logits need not be read
        moved = e * (L * V + (T * (V + c["pad"]) if c["train"] else 0)) + 4.0 * T
        return {"bytes": moved, "flops": (8.0 if c["train"] else 4.0) * L * V}
    cu, csp, slot = _adapter_batch(c)
    T, r, inn, out = cu[-1], c["rank"], c["inn"], c["out"]
    rows = _client_rows(c)
    live = sum(rows[i + 1] - rows[i] for i, k in enumerate(slot) if k >= 0)
    used = len({k for k in slot if k >= 0})
    pairs = used * r * (inn + out)
    if c["what"] == "fwd":
        return {"bytes": e * (live * inn + 2.0 * T * out + pairs) + 4.0 * T * r, "flops": 2.0 * live * r * (inn + out)}
    return {"bytes": e * (live * (inn + out) + 2.0 * T * inn + pairs) + 4.0 * live * r + 4.0 * c["slots"] * r * (inn + out),
            "flops": 4.0 * live * r * (inn + out)}


# ---------------------------------------------------------------------------
# The same outputs in float64, from the definitions
# ---------------------------------------------------------------------------

def _exact_adapters(c, s):
    rows, scale = _client_rows(c), s["scale"]
    x, a, b = s["x"].double(), s["a"].double(), s["b"].double()
    if c["what"] == "fwd":
        y, v = s["base"].double(), torch.zeros((x.shape[0], c["rank"]), dtype=torch.float64, device="cuda")
        for i, k in enumerate(s["slot"]):
            if k >= 0:
                t = slice(rows[i], rows[i + 1])
                v[t] = x[t] @ a[k].t()
                y[t] += scale * (v[t] @ b[k].t())
        return {"y": y, "v": v}
    dx, v = s["dres"].double(), s["v"].double()
    da, db = torch.zeros_like(a), torch.zeros_like(b)
    for i, k in enumerate(s["slot"]):
        if k >= 0:
            t = slice(rows[i], rows[i + 1])
            dy = s["dy"][t].double()
            dv = scale * (dy @ b[k])
            dx[t] += dv @ a[k]
            da[k] += dv.t() @ x[t]
            db[k] += scale * (dy.t() @ v[t])
    return {"dx": dx, "da": da, "db": db}


def _exact_preference(c, s):
    V, labels = c["vocab"], s["labels"].tolist()
    cu = s["cu"].tolist()
    logp, slopes, rows = [], [], []
    for q in range(2 * c["pairs"]):
        t = [i for i in range(cu[q], cu[q + 1]) if labels[i] >= 0]
        rows.append(torch.tensor(t, dtype=torch.long, device="cuda"))
        if not t:
            logp.append(torch.zeros((), dtype=torch.float64, device="cuda"))
            continue
        x = s["logits"][rows[q]][:, :V].double()
        lab = s["labels"][rows[q]].long()
        logp.append((torch.gather(x, 1, lab[:, None])[:, 0] - torch.logsumexp(x, 1)).sum())
    logp = torch.stack(logp).requires_grad_(True)
    d = logp if s["ref"] is None else logp - s["ref"].double()
    z = c["beta"] * (d[0::2] - d[1::2])
    loss = -(1 - c["smoothing"]) * torch.nn.functional.logsigmoid(z) \
        - c["smoothing"] * torch.nn.functional.logsigmoid(-z)
    out = {"logp": logp.detach(), "loss": loss.detach(), "total": loss.detach().sum().reshape(1)}
    if c["train"]:
        slopes = torch.autograd.grad(s["grad_scale"] * loss.sum(), logp)[0]
        g = torch.zeros(s["logits"].shape, dtype=torch.float64, device="cuda")
        for q in range(2 * c["pairs"]):
            if len(rows[q]):
                p = -slopes[q] * torch.softmax(s["logits"][rows[q]][:, :V].double(), 1)
                p[torch.arange(len(rows[q]), device="cuda"), s["labels"][rows[q]].long()] += slopes[q]
                g[rows[q], :V] = p
        out["dlogits"] = g
    return out


def exact(case, seed):
    c = case
    if c["kind"] == "clip":
        flat, grads = _clip_inputs(c, seed)
        wide = [g.double() for g in grads]
        norm = torch.sqrt(sum(torch.dot(g, g) for g in wide))
        k = min(1.0, c["max_norm"] / (norm.item() + 1e-6))
        out = torch.zeros(flat.shape, dtype=torch.float64, device="cuda")
        for g, o in zip(wide, _views(out, c)):
            o.copy_(g * k)
        return {"norm": norm.reshape(1), "grads": out}
    if c["kind"] == "adapters":
        return _exact_adapters(c, _prepare_adapters(c, seed))
    return _exact_preference(c, _prepare_preference(c, seed))
