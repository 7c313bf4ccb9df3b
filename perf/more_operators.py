"""What a decode step of a grouped rollout runs around its caches, as measurable cases.

A case is a dict of plain values; `prepare` builds what a program holds before the call, `run`
makes one pass through an operator, `exact` is the same result from its definition in 64 bits.
Where `own` is false, `run` computes the operators in elementary torch operations: in 32 bits, the
drawn tokens in 64.

  shared     decode attention of groups of sequences whose first tokens (the prompt) are the same
  sample     the next token of every row of logits: temperature, top-k, top-p, min-p, one given
             uniform number a row; with the log-probability that it was drawn with
  norm       the residual stream after a block and the norm before the next one:
             n = x / rms(x) * post_weight, h' = h + scale * sigmoid(gate) * n, y = h' / rms(h') * weight
  norm_grad  its gradient: of h, x, the gate and both weights

Shapes are the Qwen3-like ones of `workloads.py`: head_dim 128, 16/8 to 40/8 heads, 2048 to 5120
channels, a vocabulary of 151936, pages of 16 to 128 tokens; and generic ones.
"""
import math

import numpy as np
import torch

own = False

D = 128
EPS = 1e-6


def listed():
    return [
        # One prompt with eight short samples: the latency of the smallest grouped call.
        dict(name="shared_1x8_2k", kind="shared", groups=1, per_lo=8, per_hi=8, pre_lo=2001,
             pre_hi=2001, new_lo=1, new_hi=64, hq=16, hkv=8, ps=16),
        # Uneven groups late in a rollout (some samples have ended), odd prompts, large pages.
        dict(name="shared_odd_groups", kind="shared", groups=7, per_lo=1, per_hi=13, pre_lo=777,
             pre_hi=5001, new_lo=3, new_hi=1501, hq=40, hkv=8, ps=64),
        # A rollout batch: eight prompts of 1K to 4K tokens, eight samples each.
        dict(name="shared_8x8_4k", kind="shared", groups=8, per_lo=8, per_hi=8, pre_lo=1024,
             pre_hi=4096, new_lo=64, new_hi=4096, hq=32, hkv=8, ps=32),
        # The largest: long prompts, sixteen samples each, 256 sequences.
        dict(name="shared_16x16_16k", kind="shared", groups=16, per_lo=16, per_hi=16, pre_lo=8192,
             pre_hi=16384, new_lo=512, new_hi=8192, hq=32, hkv=8, ps=32),
        # One user's next token with a model's usual chat settings.
        dict(name="sample_b1_top20", kind="sample", rows=1, vocab=151936, pad=0, dtype="f32",
             filters="topk_topp", masked=0),
        # A rollout step of 256 sequences: the model's own distribution, no filter.
        dict(name="sample_b256_plain", kind="sample", rows=256, vocab=151936, pad=0, dtype="f32",
             filters="none", masked=0),
        # A server's batch, every row with its own settings, a part of the vocabulary masked, rows
        # of a padded head's output.
        dict(name="sample_b64_mixed", kind="sample", rows=64, vocab=151936, pad=128, dtype="bf16",
             filters="mixed", masked=3),
        # A small model's odd vocabulary, a nucleus in fp32.
        dict(name="sample_odd_topp", kind="sample", rows=37, vocab=50021, pad=0, dtype="f32",
             filters="topp", masked=0),
        # Around a block for one new token, no norm behind the block.
        dict(name="norm_step_b1", kind="norm", tokens=1, channels=2048, post=False, gate=False,
             stream="bf16"),
        # Around a gated block with norms on both sides for prompts of 32K tokens.
        dict(name="norm_32k_gated", kind="norm", tokens=32768, channels=4096, post=True, gate=True,
             stream="bf16"),
        # The trainer's gradient on a short odd piece of text, the stream kept in fp32.
        dict(name="norm_grad_odd", kind="norm_grad", tokens=1021, channels=5120, post=True,
             gate=False, stream="f32"),
        # The trainer's gradient on a micro-batch, gated.
        dict(name="norm_grad_32k", kind="norm_grad", tokens=32768, channels=4096, post=True,
             gate=True, stream="bf16"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    most = {}
    for c in listed():
        most[c["kind"]] = max(most.get(c["kind"], 0), work(c)["bytes"])
    # (the plain form fills a group up to its longest sequence, and sorts whole rows)
    room = 16 * 16 * (16384 + 8192) * 8
    while True:
        c = _draw(rng)
        if work(c)["bytes"] > most[c["kind"]]:
            continue
        if c["kind"] == "shared" and \
                c["groups"] * c["per_hi"] * (c["pre_hi"] + c["new_hi"]) * c["hkv"] > room:
            continue
        return c


def _draw(rng):
    kind = rng.choice(["shared", "shared", "sample", "sample", "norm", "norm_grad"])
    if kind == "shared":
        hkv = rng.choice([8, 8, 8, 4, 2, 3])
        per, pre, new = _log_int(rng, 1, 64), _log_int(rng, 8, 32768), _log_int(rng, 1, 8192)
        low = rng.choice([0.05, 0.5, 1.0])
        return dict(kind=kind, groups=_log_int(rng, 1, 32), per_lo=max(1, int(per * low)), per_hi=per,
                    pre_lo=max(1, int(pre * low)), pre_hi=pre, new_lo=max(1, int(new * low)),
                    new_hi=new, hq=hkv * rng.choice([1, 2, 4, 4, 5, 8]), hkv=hkv,
                    ps=rng.choice([16, 16, 32, 64, 128]))
    if kind == "sample":
        vocab = rng.choice([151936, _log_int(rng, 500, 262144)])
        return dict(kind=kind, rows=_log_int(rng, 1, 256), vocab=vocab,
                    pad=rng.choice([0, 0, 3, 128]), dtype=rng.choice(["f32", "bf16"]),
                    filters=rng.choice(["none", "topk", "topp", "minp", "topk_topp", "mixed"]),
                    masked=rng.choice([0, 0, 3, 90]))
    return dict(kind=kind, tokens=_log_int(rng, 1, 32768), channels=8 * _log_int(rng, 32, 1024),
                post=rng.random() < 0.6, gate=rng.random() < 0.5,
                stream=rng.choice(["bf16", "bf16", "f32"]))


def _spread(n, lo, hi, salt, seed=None):
    """n whole numbers, uniform over the range: the same ones for every seed, dealt out in an order
    of the seed's."""
    v = np.random.default_rng([n, salt]).integers(lo, hi + 1, size=n).astype(np.int64)
    return v if seed is None else np.random.default_rng(seed + salt).permutation(v)


def _groups(case, seed=None):
    """(sequences of every group, prompt length of every group, new tokens of every sequence): the
    groups as the case has them, the new tokens dealt out by the seed."""
    per = _spread(case["groups"], case["per_lo"], case["per_hi"], 1)
    pre = _spread(case["groups"], case["pre_lo"], case["pre_hi"], 2)
    return per, pre, _spread(int(per.sum()), case["new_lo"], case["new_hi"], 3, seed)


def work(case):
    kind = case["kind"]
    if kind == "shared":
        per, pre, new = _groups(case)
        whole = pre // case["ps"] * case["ps"]
        tokens = int(whole.sum() + (per * (pre - whole)).sum() + new.sum())
        return {"bytes": tokens * case["hkv"] * 512 + int(per.sum()) * case["hq"] * D * 4,
                "flops": int((per * pre).sum() + new.sum()) * case["hq"] * D * 4}
    if kind == "sample":
        n = case["rows"] * case["vocab"]
        return {"bytes": n * (2 if case["dtype"] == "bf16" else 4) + case["rows"] * 24,
                "flops": n * 4}
    T, C = case["tokens"], case["channels"]
    s = 2 if case["stream"] == "bf16" else 4
    if kind == "norm":   # h, x, gate; h', y; weights
        return {"bytes": T * C * (2 * s + 4 + 2 * case["gate"]) + C * (2 + 2 * case["post"]),
                "flops": T * C * (8 + 5 * case["post"] + 6 * case["gate"])}
    # dy, dh', h', x, gate; dh, dx, dgate; weights and their gradients.  Without a norm and a gate
    # behind the block neither x nor the gate is read.
    return {"bytes": T * C * (3 * s + 4 + 2 * (case["post"] or case["gate"]) + 4 * case["gate"]) +
            C * (6 + 6 * case["post"]),
            "flops": T * C * (14 + 14 * case["post"] + 10 * case["gate"])}


# ------------------------------------------------------------------------------------ inputs
def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _randn(g, *shape, dtype=torch.bfloat16):
    return torch.randn(shape, generator=g, device="cuda", dtype=dtype)


def _i32(v):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(v).astype(np.int32))).cuda()


def prepare(case, seed):
    g, kind = _generator(seed), case["kind"]
    if kind == "shared":
        return _prepare_shared(case, seed, g)
    if kind == "sample":
        return _prepare_sample(case, g)
    T, C = case["tokens"], case["channels"]
    stream = torch.bfloat16 if case["stream"] == "bf16" else torch.float32
    tilt = 1 + 3 * torch.rand(C, generator=g, device="cuda")      # channels of a stream differ in size
    fused = _randn(g, T, 2 * C if case["gate"] else C)            # the block's output (and its gate)
    x = dict(kind=kind, scale=0.4, x=fused[:, :C], gate=fused[:, C:] if case["gate"] else None,
             post=None)
    for w in ("weight", "post") if case["post"] else ("weight",):
        x[w] = (1 + 0.3 * torch.randn(C, generator=g, device="cuda")).to(torch.bfloat16)
    x["h"] = (_randn(g, T, C) * tilt.to(torch.bfloat16)).to(stream)   # (norm_grad: the stream behind)
    if kind == "norm_grad":
        x |= dict(dy=_randn(g, T, C), dh=_randn(g, T, C).to(stream))
    return x


def _prepare_shared(case, seed, g):
    per, pre, new = _groups(case, seed)
    ps, hkv = case["ps"], case["hkv"]
    cu = np.concatenate([[0], np.cumsum(per)])
    lens = np.repeat(pre, per) + new
    first = pre // ps                                             # whole pages that a group shares
    mine = (lens + ps - 1) // ps - np.repeat(first, per)
    P = int(first.sum() + mine.sum())
    perm = torch.randperm(P, generator=g, device="cuda").to(torch.int32).cpu().numpy()
    bt = np.zeros((len(lens), int((lens.max() + ps - 1) // ps)), np.int32)
    at = 0
    for i in range(case["groups"]):
        bt[cu[i]:cu[i + 1], :first[i]] = perm[at:at + first[i]]
        at += first[i]
        for b in range(cu[i], cu[i + 1]):
            bt[b, first[i]:first[i] + mine[b]] = perm[at:at + mine[b]]
            at += mine[b]
    k, v = (torch.empty((P, hkv, ps, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    for t in (k, v):
        t.normal_(generator=g)
    B = len(lens)
    return dict(kind="shared", q=_randn(g, B, case["hq"], D), k=k, v=v, bt=_pages(bt),
                seq_lens=_i32(lens), cu=_i32(cu), pre=_i32(pre), host=(cu, pre, lens),
                out=torch.empty((B, case["hq"], D), dtype=torch.bfloat16, device="cuda"))


def _pages(bt):
    return torch.from_numpy(bt).cuda()


def _prepare_sample(case, g):
    T, V = case["rows"], case["vocab"]
    z = 2.0 * _randn(g, T, V + case["pad"], dtype=torch.float32)
    # what a model favours: a few tokens well above the rest, more or fewer of them from row to row
    hot = torch.randint(0, V, (T, 64), generator=g, device="cuda")
    lift = torch.rand((T, 64), generator=g, device="cuda")
    lift = lift * (4 + 12 * torch.rand((T, 1), generator=g, device="cuda"))
    z.scatter_add_(1, hot, lift)
    if case["masked"]:   # a grammar's mask: so many of 100 tokens are out, the last never
        out = torch.rand((T, V + case["pad"]), generator=g, device="cuda") * 100 < case["masked"]
        out[:, V - 1] = False
        z.masked_fill_(out, -math.inf)
    z = z.to(torch.bfloat16 if case["dtype"] == "bf16" else torch.float32)

    def uniform(lo, hi):
        return lo + (hi - lo) * torch.rand(T, generator=g, device="cuda")

    f = case["filters"]
    x = dict(kind="sample", z=z[:, :V], u=uniform(0, 1).clamp_max(1 - 2.0 ** -24), t=None, k=None,
             p=None, q=None)
    some = torch.randint(0, 6, (T,), generator=g, device="cuda")  # mixed: what a row's request asks for
    if f != "none":
        x["t"] = uniform(0.6, 1.1)
    if f == "mixed":
        x["t"] = torch.where(some == 0, 0.0, x["t"])              # greedy
    if f in ("topk", "topk_topp", "mixed"):
        x["k"] = torch.randint(5, 60, (T,), generator=g, device="cuda").to(torch.int32)
        if f == "topk_topp":
            x["k"].fill_(20)
        if f == "mixed":
            x["k"] = torch.where((some == 1) | (some == 2), x["k"], 0)
    if f in ("topp", "topk_topp", "mixed"):
        x["p"] = uniform(0.8, 0.98)
        if f == "mixed":
            x["p"] = torch.where((some == 2) | (some == 3), x["p"], 1.0)
    if f in ("minp", "mixed"):
        x["q"] = uniform(0.02, 0.1)
        if f == "mixed":
            x["q"] = torch.where(some == 4, x["q"], 0.0)
    return x


# ------------------------------------------------------------------------- one pass of an operator
def run(x):
    return _own(x) if own else _plain(x)


def _own(x):
    from paper_2606_08446_amd import sparrow as S
    kind = x["kind"]
    if kind == "shared":
        return S.shared_prefix_decode_attn(x["q"], x["k"], x["v"], x["bt"], x["seq_lens"], x["cu"],
                                           x["pre"], out=x["out"], out_dtype=S.SPARROW_OUT_BF16)
    if kind == "sample":
        return S.sample(x["z"], x["u"], temperature=x["t"], top_k=x["k"], top_p=x["p"],
                        min_p=x["q"])
    if kind == "norm":
        return S.residual_norm(x["h"], x["x"], x["weight"], post_weight=x["post"], gate=x["gate"],
                               scale=x["scale"], eps=EPS)
    got = S.residual_norm_bwd(x["dy"], x["dh"], x["h"], x["x"], x["weight"], post_weight=x["post"],
                              gate=x["gate"], scale=x["scale"], eps=EPS)
    return [t for t in got if t is not None]


def _plain(x):
    kind = x["kind"]
    if kind == "shared":
        return _attend(x)
    if kind == "sample":
        return _draw_tokens(x)
    w, post, scale = x["weight"].float(), x["post"], x["scale"]
    if kind == "norm":
        h, b = x["h"].float(), x["x"].float()
        if post is not None:
            b = b * torch.rsqrt(b.square().mean(-1, keepdim=True) + EPS) * post.float()
        if x["gate"] is not None:
            b = b / (1 + torch.exp(-x["gate"].float()))
        h = h + scale * b
        y = h * torch.rsqrt(h.square().mean(-1, keepdim=True) + EPS) * w
        return h.to(x["h"].dtype), y.to(torch.bfloat16)
    h, dy = x["h"].float(), x["dy"].float()
    r = torch.rsqrt(h.square().mean(-1, keepdim=True) + EPS)
    hn, u = h * r, dy * w
    dw = (dy * hn).sum(0)
    dh = x["dh"].float() + r * (u - hn * (u * hn).mean(-1, keepdim=True))
    d = scale * dh                                                # of the block's gated, normed output
    n = x["x"].float()
    if post is not None:
        rx = torch.rsqrt(n.square().mean(-1, keepdim=True) + EPS)
        xn = n * rx
        n = xn * post.float()
    out = [dh.to(x["h"].dtype)]
    da = None
    if x["gate"] is not None:
        s = 1 / (1 + torch.exp(-x["gate"].float()))
        da = (d * n * s * (1 - s)).to(torch.bfloat16)
        d = d * s
    if post is not None:
        dpost = (d * xn).sum(0)
        v = d * post.float()
        d = rx * (v - xn * (v * xn).mean(-1, keepdim=True))
    out.append(d.to(torch.bfloat16))
    if da is not None:
        out.append(da)
    out.append(dw)
    if post is not None:
        out.append(dpost)
    return out


def _attend(x):
    cu, pre, lens = x["host"]
    k, v, bt = x["k"], x["v"], x["bt"].long()
    ps, hkv = k.shape[2], k.shape[1]
    head = torch.arange(hkv, device="cuda")[:, None]
    out = torch.empty_like(x["q"])
    for i in range(len(pre)):
        lo, hi = int(cu[i]), int(cu[i + 1])
        n, s = hi - lo, int(pre[i]) // ps
        q = x["q"][lo:hi].float().view(n, hkv, -1, D)
        g = q.shape[2]
        # the shared pages against all the group's rows at once, then each sequence's own pages
        qs = q.transpose(0, 1).reshape(hkv, n * g, D)
        far = bt[lo, :s]
        ks, vs = (c[far[None], head].float().flatten(1, 2) for c in (k, v))
        zs = (qs @ ks.transpose(1, 2).contiguous()).view(hkv, n, g, s * ps).transpose(0, 1)
        np_ = int((lens[lo:hi].max() + ps - 1) // ps)
        near = bt[lo:hi, s:np_]
        kn, vn = (c[near[:, None], head].float().flatten(2, 3) for c in (k, v))
        zn = q @ kn.transpose(2, 3).contiguous()                  # [n][Hkv][g][tokens]
        pos = s * ps + torch.arange(zn.shape[-1], device="cuda")
        zn = zn.masked_fill((pos >= x["seq_lens"][lo:hi, None])[:, None, None], -math.inf)
        z = torch.cat([zs, zn], -1) / math.sqrt(D)
        p = torch.exp(z - z.amax(-1, keepdim=True))
        p = p / p.sum(-1, keepdim=True)
        p_far = p[..., :s * ps].transpose(0, 1).reshape(hkv, n * g, s * ps)
        o = (p_far @ vs).view(hkv, n, g, D).transpose(0, 1) + p[..., s * ps:].contiguous() @ vn
        out[lo:hi] = o.reshape(n, hkv * g, D).to(torch.bfloat16)
    return out


def _draw_tokens(x):
    """In 64 bits throughout: a drawn number lies between two sums of many weights."""
    z = x["z"].double() + 0.0                                     # (-0 is 0)
    T, V = z.shape
    u, t = x["u"].double()[:, None], x["t"]
    greedy = torch.zeros((T, 1), dtype=torch.bool, device="cuda") if t is None else t[:, None] <= 0
    top, at = z.max(1, keepdim=True)
    at = torch.where(z == top, torch.arange(V, device="cuda"), V).amin(1, keepdim=True)
    xs = z - top
    if t is not None:
        xs = xs / torch.where(greedy, 1.0, t.double()[:, None])
    w = torch.exp(xs)
    if x["k"] is not None or x["p"] is not None:
        order = torch.sort(z, dim=1, descending=True, stable=True)[1]
        ws = torch.gather(w, 1, order)
        if x["k"] is not None:
            k = x["k"][:, None]
            ws = ws.masked_fill((torch.arange(V, device="cuda") >= k) & (k > 0), 0)
        keep = ws > 0
        if x["p"] is not None:
            p = x["p"].double()[:, None]
            c = torch.cumsum(ws, 1)
            keep &= (c - ws < p * c[:, -1:]) | (p >= 1)
            keep[:, 0] = True
        w = w * torch.zeros_like(keep).scatter_(1, order, keep)
    if x["q"] is not None:
        w = w.masked_fill(w < x["q"].double()[:, None], 0)
    c = torch.cumsum(w, 1)
    tok = torch.searchsorted(c, u * c[:, -1:], right=True).clamp_max(V - 1)
    lp = torch.gather(xs, 1, tok) - torch.log(c[:, -1:])
    tok, lp = torch.where(greedy, at, tok), torch.where(greedy, 0.0, lp)
    return tok[:, 0].to(torch.int32), lp[:, 0].float()


# ---------------------------------------------------------------------------------- in 64 bits
def exact(case, seed):
    x = prepare(case, seed)
    kind = case["kind"]
    if kind == "shared":
        return _exact_attend(x, case)
    if kind == "sample":
        return _exact_tokens(x, case)
    h, b, w = x["h"].double(), x["x"].double(), x["weight"].double()
    mx = b.pow(2).mean(-1, keepdim=True) + EPS
    n = b if x["post"] is None else b / mx.sqrt() * x["post"].double()
    s = 1.0 if x["gate"] is None else torch.sigmoid(x["gate"].double())
    if kind == "norm":
        h = h + x["scale"] * s * n
        return h, h / (h.pow(2).mean(-1, keepdim=True) + EPS).sqrt() * w
    C = h.shape[1]
    mh, dy = h.pow(2).mean(-1, keepdim=True) + EPS, x["dy"].double()
    # d/dh of w h mh^(-1/2): the direct part, and through mh
    dh = x["dh"].double() + dy * w / mh.sqrt() - (dy * w * h).sum(-1, keepdim=True) * h / (C * mh.pow(1.5))
    d = x["scale"] * dh
    out = [dh]
    dx, dpost = d * s, None
    if x["post"] is not None:
        dpost = (dx * b / mx.sqrt()).sum(0)
        v = dx * x["post"].double()
        dx = v / mx.sqrt() - (v * b).sum(-1, keepdim=True) * b / (C * mx.pow(1.5))
    out.append(dx)
    if x["gate"] is not None:
        out.append(d * n * s * (1 - s))
    out.append((dy * h / mh.sqrt()).sum(0))
    return out if dpost is None else out + [dpost]


def _exact_attend(x, case):
    cu, pre, lens = x["host"]
    ps, hkv, hq = case["ps"], case["hkv"], case["hq"]
    out = torch.empty(x["q"].shape, dtype=torch.float64, device="cuda")
    heads = torch.arange(hkv, device="cuda")[:, None]
    for b in range(len(lens)):
        L = int(lens[b])
        pages = x["bt"][b, :-(-L // ps)].long()
        k, v = (c[pages[None], heads].double().flatten(1, 2)[:, :L] for c in (x["k"], x["v"]))
        q = x["q"][b].double().view(hkv, hq // hkv, D)
        z = torch.matmul(q, k.transpose(1, 2).contiguous()) / math.sqrt(D)
        out[b] = torch.matmul(torch.softmax(z, -1), v.contiguous()).view(hq, D)
    return out


def _exact_tokens(x, case):
    V = case["vocab"]
    z = x["z"].float().cpu().numpy().astype(np.float64)

    def of(name, default):
        return np.full(len(z), default) if x[name] is None else x[name].cpu().numpy()

    u, t, k, p, q = of("u", 0), of("t", 1.0), of("k", 0), of("p", 1.0), of("q", 0.0)
    tokens, lps = np.zeros(len(z), np.int32), np.zeros(len(z))
    for i, row in enumerate(z):
        top = row.max()
        if t[i] <= 0:
            tokens[i] = int(np.argmax(row))
            continue
        e = (row - top) / np.float64(t[i])
        ids = np.nonzero(np.isfinite(row))[0]
        if 0 < k[i] < V or p[i] < 1:
            ids = ids[np.argsort(-row[ids], kind="stable")]       # largest first, lower index first
            if 0 < k[i] < V:
                ids = ids[:k[i]]
            if p[i] < 1:
                c = np.cumsum(np.exp(e[ids]))
                ids = ids[:max(1, int(np.searchsorted(c, np.float64(p[i]) * c[-1], side="left")) + 1)]
            ids = np.sort(ids)
        if q[i] > 0:
            ids = ids[np.exp(e[ids]) >= np.float64(q[i])]
        c = np.cumsum(np.exp(e[ids]))
        j = min(int(np.searchsorted(c, np.float64(u[i]) * c[-1], side="right")), len(ids) - 1)
        tokens[i], lps[i] = ids[j], e[ids[j]] - math.log(c[-1])
    return torch.from_numpy(tokens), torch.from_numpy(lps)
