"""The steps around an 8-bit paged cache, as measurable cases: what a program does between a
layer's q/k/v projection and its attention output.

A case is a dict of plain values; `prepare` builds what a program holds before the call, `run`
makes one pass through an operator, `exact` is the same result from its definition in 64 bits.
Where `own` is false, `run` computes the operators in elementary torch operations in 32 bits.

  rope        q and k heads: RMS norm over the head, weight, half-split position rotation
  rope_grad   its gradient: dq, dk and the two weights' gradients
  append      new rows into an e4m3 cache with a power-of-two scale per (token, KV head), and the
              channel-wise min/max landmarks of the pages they land on
  read        the last tokens of every sequence back as bf16 rows
  dense       decode attention of one new token per sequence over every cached token
  sparse      the same over per-head page lists

Shapes are the Qwen3-like ones of `workloads.py`: head_dim 128, 16/8 to 40/8 heads, contexts of
1K to 64K tokens, pages of 16 to 128 tokens; rotation base 1e6, norm epsilon 1e-6.

The cache holds for K and V each float8_e4m3fn codes [P][Hkv][ps][128], and for both one array of
biased exponents, uint8 [P][Hkv][ps / 4][2][4]: groups of four tokens, K's four bytes, V's four.
A row's value is code * 2^(byte - 127).
"""
import math

import numpy as np
import torch

own = False

D = 128
EPS = 1e-6
BASE = 1e6
E_MIN, E_MAX = -117, 119


def listed():
    return [
        # One user's next token in a 1.7B-like layer: the latency of the smallest call.
        dict(name="rope_step_b1", kind="rope", seqs=1, len_lo=1, len_hi=1, start=4095, hq=16, hkv=8),
        # Prompts of a rollout batch, 8B-like heads, about 64K tokens in ragged rows.
        dict(name="rope_prompts_64k", kind="rope", seqs=64, len_lo=512, len_hi=1536, start=0,
             hq=32, hkv=8),
        # The trainer's gradient on a short, odd piece of text, 14B-like heads.
        dict(name="rope_grad_odd", kind="rope_grad", seqs=3, len_lo=331, len_hi=351, start=0,
             hq=40, hkv=8),
        # The trainer's gradient on a micro-batch of long rollouts.
        dict(name="rope_grad_32k", kind="rope_grad", seqs=4, len_lo=8192, len_hi=8192, start=0,
             hq=32, hkv=8),
        # A decode step of 256 sequences writes one token each.
        dict(name="append_step_b256", kind="append", seqs=256, len_lo=1, len_hi=1, past=1500,
             ps=32, hkv=8),
        # Prompts of 1 to 4K tokens go into the cache, some behind a prefix already there.
        dict(name="append_prompts_64k", kind="append", seqs=32, len_lo=1, len_hi=4096, past=100,
             ps=16, hkv=8),
        # The last odd pieces of a few sequences, as a prompt that goes on reads them.
        dict(name="read_odd_rows", kind="read", seqs=5, len_lo=7, len_hi=203, past=333, ps=16, hkv=8),
        # A rollout batch's cache for a pass over whole texts.
        dict(name="read_64k", kind="read", seqs=16, len_lo=2049, len_hi=6143, past=0, ps=32, hkv=8),
        # One user, one short context, an odd length.
        dict(name="dense_b1_4k", kind="dense", batch=1, hq=16, hkv=8, ps=16, len_lo=4097,
             len_hi=4097),
        # The 1.7B-like rollout batch, dense.
        dict(name="dense_b64_8k_32k", kind="dense", batch=64, hq=16, hkv=8, ps=16, len_lo=8192,
             len_hi=32768),
        # A fixed 1024-token budget at 32K, the serving point of the page-size study.
        dict(name="sparse_b16_1024", kind="sparse", batch=16, hq=16, hkv=8, ps=16, len_lo=32768,
             len_hi=32768, permille=31),
        # The 8B-like rollout batch, the largest cache, 10 % of 32-token pages.
        dict(name="sparse_b256_10pct", kind="sparse", batch=256, hq=32, hkv=8, ps=32, len_lo=16384,
             len_hi=40960, permille=100),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    most = {}
    for c in listed():
        k = "attention" if c["kind"] in ("dense", "sparse") else c["kind"]
        most[k] = max(most.get(k, 0), work(c)["bytes"])
    # (the plain form of attention fills its batch up to the longest sequence)
    room = {"dense": 64 * 32768 * 8, "sparse": 256 * 40960 * 8}
    while True:
        c = _draw(rng)
        k = "attention" if c["kind"] in room else c["kind"]
        if work(c)["bytes"] <= most[k] and (c["kind"] not in room or
                                            c["batch"] * c["len_hi"] * c["hkv"] <= room[c["kind"]]):
            return c


def _draw(rng):
    kind = rng.choice(["rope", "rope_grad", "append", "read", "dense", "sparse"])
    hkv = rng.choice([8, 8, 8, 4, 2, 3])
    hq = hkv * rng.choice([1, 2, 4, 4, 5, 8])
    ps = rng.choice([16, 16, 32, 64, 128])
    if kind in ("dense", "sparse"):
        hi = _log_int(rng, 16, 65536)
        c = dict(kind=kind, batch=_log_int(rng, 1, 256), hq=hq, hkv=hkv, ps=ps,
                 len_lo=max(1, int(hi * rng.choice([0.01, 0.25, 0.6, 1.0]))), len_hi=hi)
        return c if kind == "dense" else c | dict(permille=_log_int(rng, 20, 250))
    hi = _log_int(rng, 1, 8192)
    c = dict(kind=kind, seqs=_log_int(rng, 1, 256),
             len_lo=max(1, int(hi * rng.choice([0.01, 0.5, 1.0]))), len_hi=hi)
    if kind in ("rope", "rope_grad"):
        return c | dict(start=rng.choice([0, 0, 4095, 131071]), hq=hq, hkv=hkv)
    return c | dict(past=rng.choice([0, _log_int(rng, 1, 2000)]), ps=ps, hkv=hkv)


def _lens(n, lo, hi, seed=None):
    """Lengths uniform over the range: the same ones for every seed, dealt to the sequences in an
    order of the seed's."""
    v = np.random.default_rng(n).integers(lo, hi + 1, size=n).astype(np.int64)
    return v if seed is None else np.random.default_rng(seed).permutation(v)


def work(case):
    kind, hkv = case["kind"], case["hkv"]
    if kind in ("rope", "rope_grad"):
        T, H = int(_lens(case["seqs"], case["len_lo"], case["len_hi"]).sum()), case["hq"] + hkv
        if kind == "rope":
            return {"bytes": T * (H * 512 + 4) + 1024, "flops": T * H * D * 8}
        return {"bytes": T * (H * 768 + 4) + 1024 + 1024, "flops": T * H * D * 18}
    if kind in ("append", "read"):
        new = _lens(case["seqs"], case["len_lo"], case["len_hi"])
        T = int(new.sum())
        if kind == "read":
            return {"bytes": T * hkv * (258 + 512), "flops": T * hkv * 2 * D}
        p = case["past"]
        pages = int(((p + new - 1) // case["ps"] - p // case["ps"] + 1).sum())
        old = case["seqs"] if p % case["ps"] else 0
        return {"bytes": T * hkv * (512 + 258) + (pages + old) * hkv * 512, "flops": T * hkv * 5 * D}
    lens = _lens(case["batch"], case["len_lo"], case["len_hi"])
    tokens = lens
    if kind == "sparse":
        n = (lens + case["ps"] - 1) // case["ps"]
        k = _budget(n, case["permille"])
        tokens = np.minimum(k * case["ps"], lens)
    g = case["hq"] // hkv
    return {"bytes": int(tokens.sum()) * hkv * 258 + case["batch"] * case["hq"] * D * 4,
            "flops": int(tokens.sum()) * hkv * g * D * 4}


def _budget(n, permille):
    return np.maximum(1, -(-n * permille // 1000))


# ------------------------------------------------------------------------------------ inputs
def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.bfloat16)


def _i32(v):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(v).astype(np.int32))).cuda()


def _table(g, lens, ps):
    """Block table with one spare page per sequence, physical pages in random order."""
    pages = (lens + ps - 1) // ps + 1
    total = int(pages.sum())
    perm = torch.randperm(total, generator=g, device="cuda").to(torch.int32).cpu().numpy()
    bt = np.zeros((len(lens), int(pages.max())), np.int32)
    ends = np.cumsum(pages)
    for b in range(len(lens)):
        bt[b, :pages[b]] = perm[ends[b] - pages[b]:ends[b]]
    return torch.from_numpy(bt).cuda(), total


def _random_cache(g, pages, hkv, ps):
    """A cache of quantised normal rows, in blocks of pages."""
    k = torch.empty((pages, hkv, ps, D), dtype=torch.float8_e4m3fn, device="cuda")
    v = torch.empty_like(k)
    exps = torch.empty((pages, hkv, ps // 4, 2, 4), dtype=torch.uint8, device="cuda")
    step = max(1, (1 << 28) // (hkv * ps * D))
    for p in range(0, pages, step):
        for j, codes in enumerate((k, v)):
            x = _randn(g, min(step, pages - p), hkv, ps, D)
            c, e = _quantise(x)
            codes[p:p + step] = c
            exps[p:p + step, :, :, j] = e.view(-1, hkv, ps // 4, 4)
    return k, v, exps


def prepare(case, seed):
    g, kind, hkv = _generator(seed), case["kind"], case["hkv"]
    if kind in ("rope", "rope_grad"):
        new, hq = _lens(case["seqs"], case["len_lo"], case["len_hi"], seed), case["hq"]
        T = int(new.sum())
        pos = np.concatenate([case["start"] + np.arange(n) for n in new])
        qkv = _randn(g, T, (hq + 2 * hkv) * D)   # the fused projection's rows
        x = dict(kind=kind, pos=_i32(pos),
                 q=qkv[:, :hq * D].unflatten(1, (hq, D)),
                 k=qkv[:, hq * D:(hq + hkv) * D].unflatten(1, (hkv, D)),
                 inv_freq=torch.from_numpy(BASE ** (-np.arange(0, D, 2) / D)).cuda())
        for w in ("wq", "wk"):
            x[w] = (1 + 0.3 * torch.randn(D, generator=g, device="cuda")).to(torch.bfloat16)
        if kind == "rope_grad":
            x |= dict(dq=_randn(g, T, hq, D), dk=_randn(g, T, hkv, D))
        return x
    if kind in ("append", "read"):
        new = _lens(case["seqs"], case["len_lo"], case["len_hi"], seed)
        ps, lens = case["ps"], new + case["past"]
        T = int(new.sum())
        bt, P = _table(g, lens, ps)
        k8, v8, exps = _random_cache(g, P, hkv, ps)
        x = dict(kind=kind, T=T, k8=k8, v8=v8, exps=exps, bt=bt, seq_lens=_i32(lens),
                 cu=_i32(np.concatenate([[0], np.cumsum(new)])))
        if kind == "append":
            if case["len_hi"] == 1:
                x["cu"] = None    # one token each
            qkv = _randn(g, T, 2 * hkv * D)
            x |= dict(k=_randn(g, T, hkv, D), v=qkv[:, hkv * D:].unflatten(1, (hkv, D)))
            # landmarks of the tokens that are there already: those of a page's first `past` slots
            first = np.zeros(P, np.int64)
            table = bt.cpu().numpy()
            first[table[:, case["past"] // ps]] = case["past"] % ps
            held = torch.arange(ps, device="cuda")[None] < torch.from_numpy(first).cuda()[:, None]
            held = held[:, None, :, None]
            val = k8.float() * _pow2(exps[:, :, :, 0].reshape(P, hkv, ps, 1))
            lo = torch.where(held, val, math.inf).amin(2)
            hi = torch.where(held, val, -math.inf).amax(2)
            some = held.any(2)
            x["meta"] = torch.stack([torch.where(some, lo, 0), torch.where(some, hi, 0)],
                                    2).to(torch.bfloat16)
        return x
    lens = _lens(case["batch"], case["len_lo"], case["len_hi"], seed)
    bt, P = _table(g, lens, case["ps"])
    k8, v8, exps = _random_cache(g, P, hkv, case["ps"])
    x = dict(kind=kind, q=_randn(g, case["batch"], case["hq"], D), k8=k8, v8=v8, exps=exps, bt=bt,
             seq_lens=_i32(lens), out=torch.empty((case["batch"], case["hq"], D),
                                                  dtype=torch.bfloat16, device="cuda"))
    if kind == "sparse":   # ascending random lists, the sequence's last page among them
        n = (lens + case["ps"] - 1) // case["ps"]
        want = _budget(n, case["permille"])
        rng = np.random.default_rng(seed + 1)
        idx = np.full((case["batch"], hkv, int(want.max())), -1, np.int32)
        for b in range(case["batch"]):
            for h in range(hkv):
                idx[b, h, :want[b]] = np.sort(np.append(
                    rng.choice(n[b] - 1, size=want[b] - 1, replace=False), n[b] - 1))
        x |= dict(idx=torch.from_numpy(idx).cuda(), n=_i32(want))
    return x


# ------------------------------------------------------------------------- one pass of an operator
def run(x):
    return _own(x) if own else _plain(x)


def _own(x):
    from paper_2606_08446_amd import sparrow as S
    kind = x["kind"]
    if kind == "rope":
        return S.qk_norm_rope(x["q"], x["k"], x["wq"], x["wk"], x["inv_freq"], x["pos"], EPS)
    if kind == "rope_grad":
        return S.qk_norm_rope_bwd(x["dq"], x["dk"], x["q"], x["k"], x["wq"], x["wk"],
                                  x["inv_freq"], x["pos"], EPS)
    if kind == "append":
        S.append_kv_e4m3(x["k"], x["v"], x["k8"], x["v8"], x["exps"], x["bt"], x["seq_lens"],
                         x["meta"], cu_tokens=x["cu"])
        return x["k8"], x["v8"], x["exps"], x["meta"]
    if kind == "read":
        return S.read_kv_e4m3(x["k8"], x["v8"], x["exps"], x["bt"], x["seq_lens"], x["cu"], x["T"])
    if kind == "dense":
        return S.dense_decode_attn_e4m3(x["q"], x["k8"], x["v8"], x["exps"], x["bt"],
                                        x["seq_lens"], out=x["out"], out_dtype=S.SPARROW_OUT_BF16)
    return S.sparse_decode_attn_e4m3(x["q"], x["k8"], x["v8"], x["exps"], x["bt"], x["seq_lens"],
                                     x["n"], x["idx"], out=x["out"], out_dtype=S.SPARROW_OUT_BF16)


def _plain(x):
    kind = x["kind"]
    if kind == "rope":
        a = x["pos"].double()[:, None] * x["inv_freq"]
        c, s = a.cos().float()[:, None], a.sin().float()[:, None]
        return _norm_rotate(x["q"], x["wq"], c, s), _norm_rotate(x["k"], x["wk"], c, s)
    if kind == "rope_grad":
        a = x["pos"].double()[:, None] * x["inv_freq"]
        c, s = a.cos().float()[:, None], a.sin().float()[:, None]
        dq, dwq = _norm_rotate_grad(x["dq"], x["q"], x["wq"], c, s)
        dk, dwk = _norm_rotate_grad(x["dk"], x["k"], x["wk"], c, s)
        return dq, dk, dwq, dwk
    if kind == "append":
        return _append(x)
    if kind == "read":
        phys, slot = _places(x)
        e = x["exps"][phys, :, slot // 4, :, slot % 4]           # [T][Hkv][2]
        rows = [(c.view(torch.uint8)[phys, :, slot].view(torch.float8_e4m3fn).float() *
                 _pow2(e[:, :, j, None])).to(torch.bfloat16)
                for j, c in enumerate((x["k8"], x["v8"]))]
        return rows[0], rows[1]
    return _attend(x)


def _norm_rotate(x, w, c, s):
    x = x.float()
    n = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * w.float()
    lo, hi = n[..., :D // 2], n[..., D // 2:]
    return torch.cat([lo * c - hi * s, hi * c + lo * s], -1).to(torch.bfloat16)


def _norm_rotate_grad(dy, x, w, c, s):
    x, dy = x.float(), dy.float()
    r = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
    lo, hi = dy[..., :D // 2], dy[..., D // 2:]
    g = torch.cat([lo * c + hi * s, hi * c - lo * s], -1)       # the rotation by the other angle
    xn = x * r
    u = g * w.float()
    dx = r * (u - xn * (u * xn).mean(-1, keepdim=True))
    return dx.to(torch.bfloat16), (g * xn).sum((0, 1))


def _pow2(byte):
    """2^(byte - 127) as float32, from its bits."""
    return (byte.int() << 23).view(torch.float32)


def _quantise(x):
    """(e4m3 codes, biased exponents) of rows [..., 128]."""
    x = x.float()
    m, e = torch.frexp(x.abs().amax(-1))                         # amax = m 2^e, m in [1/2, 1)
    e = torch.where(m <= 0.875, e - 9, e - 8)
    e = torch.where(m == 0, E_MIN, e).clamp(E_MIN, E_MAX)
    x = x * _pow2(127 - e)[..., None]
    return x.clamp(-448, 448).to(torch.float8_e4m3fn), (e + 127).to(torch.uint8)


def _places(x):
    """Physical page and slot of every new token's row."""
    lens, bt = x["seq_lens"].long(), x["bt"].long()
    cu = x["cu"]
    if cu is None:
        b, pos = torch.arange(len(lens), device="cuda"), lens - 1
    else:
        row = torch.arange(x["T"], device="cuda", dtype=torch.int32)
        b = torch.searchsorted(cu, row, right=True) - 1
        pos = lens[b] - (cu[b + 1] - row)
    ps = x["k8"].shape[2]
    return bt[b, pos // ps], pos % ps


def _append(x):
    phys, slot = _places(x)
    (ck, ek), (cv, ev) = _quantise(x["k"]), _quantise(x["v"])
    x["k8"].view(torch.uint8)[phys, :, slot] = ck.view(torch.uint8)
    x["v8"].view(torch.uint8)[phys, :, slot] = cv.view(torch.uint8)
    x["exps"][phys, :, slot // 4, :, slot % 4] = torch.stack([ek, ev], -1)
    key = ck.float() * _pow2(ek[..., None])
    lo, hi = x["meta"][:, :, 0].float(), x["meta"][:, :, 1].float()
    fresh = phys[slot == 0]                                      # pages that begin here
    lo[fresh], hi[fresh] = math.inf, -math.inf
    lo.index_reduce_(0, phys, key, "amin")
    hi.index_reduce_(0, phys, key, "amax")
    x["meta"].copy_(torch.stack([lo, hi], 2))
    return x["k8"], x["v8"], x["exps"], x["meta"]


def _attend(x):
    q, ps = x["q"], x["k8"].shape[2]
    B, Hq, _ = q.shape
    Hkv = x["k8"].shape[1]
    lens = x["seq_lens"].long()
    if x["kind"] == "dense":
        page = torch.arange(x["bt"].shape[1], device="cuda").expand(B, Hkv, -1)
    else:
        page = x["idx"].long()
    at = page.clamp_min(0)
    phys = torch.gather(x["bt"].long(), 1, at.flatten(1)).view_as(at)
    pos = at[..., None] * ps + torch.arange(ps, device="cuda")
    seen = ((page >= 0)[..., None] & (pos < lens[:, None, None, None])).flatten(2)   # [B][Hkv][n]
    head = torch.arange(Hkv, device="cuda")[None, :, None]
    e = x["exps"][phys, head]                                    # [B][Hkv][pages][ps/4][2][4]
    qg = q.float().view(B, Hkv, Hq // Hkv, D)
    k = x["k8"].view(torch.uint8)[phys, head].view(torch.float8_e4m3fn).float().flatten(2, 3)
    z = qg @ k.transpose(2, 3).contiguous()
    del k
    z = z * (_pow2(e[..., 0, :]).flatten(2)[:, :, None] / math.sqrt(D))
    z = z.masked_fill(~seen[:, :, None], -math.inf)
    p = torch.exp(z - z.amax(-1, keepdim=True))
    p = p / p.sum(-1, keepdim=True) * _pow2(e[..., 1, :]).flatten(2)[:, :, None]
    v = x["v8"].view(torch.uint8)[phys, head].view(torch.float8_e4m3fn).float().flatten(2, 3)
    return (p @ v).view(B, Hq, D).to(torch.bfloat16)


# ---------------------------------------------------------------------------------- in 64 bits
def exact(case, seed):
    x = prepare(case, seed)
    kind = case["kind"]
    if kind in ("rope", "rope_grad"):
        turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"),
                           x["pos"].double()[:, None, None] * x["inv_freq"])
        if kind == "rope":
            return tuple(_complex(turn * _pairs(_normed(x[a].double(), x[w].double())))
                         for a, w in (("q", "wq"), ("k", "wk")))
        got = []
        for a, d, w in (("q", "dq", "wq"), ("k", "dk", "wk")):
            xs, ws = x[a].double(), x[w].double()
            g = _complex(turn.conj() * _pairs(x[d].double()))
            ms = xs.pow(2).sum(-1, keepdim=True) / D + EPS
            # d/dx of w x ms^(-1/2): the direct part, and through ms
            through = (g * ws * xs).sum(-1, keepdim=True) * xs / D
            got.append((g * ws / ms.sqrt() - through / ms.pow(1.5),
                        (g * xs / ms.sqrt()).reshape(-1, D).sum(0)))
        return got[0][0], got[1][0], got[0][1], got[1][1]
    if kind == "append":
        return _exact_append(x, case)
    if kind == "read":
        value = [_exact_values(x["k8"], x["exps"], 0), _exact_values(x["v8"], x["exps"], 1)]
        lens, bt, cu = (x[n].cpu().numpy() for n in ("seq_lens", "bt", "cu"))
        rows = ([], [])
        for b in range(len(lens)):
            pos = np.arange(lens[b] - (cu[b + 1] - cu[b]), lens[b])
            at = torch.from_numpy(bt[b, pos // case["ps"]].astype(np.int64)).cuda()
            slot = torch.from_numpy(pos % case["ps"]).cuda()
            for j in (0, 1):
                rows[j].append(value[j][at, :, slot])
        return torch.cat(rows[0]), torch.cat(rows[1])
    return _exact_attend(x, case)


def _exp2(e):
    """2^e for whole float64 e, from its bits."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _pairs(x):
    return torch.complex(x[..., :D // 2], x[..., D // 2:])


def _complex(z):
    return torch.cat([z.real, z.imag], -1)


def _normed(x, w):
    return x / (x.pow(2).sum(-1, keepdim=True) / D + EPS).sqrt() * w


def _exact_values(codes, exps, j):
    """float64 values of a cache (or of some pages of it)."""
    e = exps[..., j, :].flatten(-2).double() - 127
    return codes.double() * _exp2(e)[..., None]


def _exact_append(x, case):
    ps, T = case["ps"], x["T"]
    lens, bt = x["seq_lens"].cpu().numpy(), x["bt"].cpu().numpy()
    cu = np.arange(len(lens) + 1) if x["cu"] is None else x["cu"].cpu().numpy()
    phys, slot = np.zeros(T, np.int64), np.zeros(T, np.int64)
    for b in range(len(lens)):
        pos = np.arange(lens[b] - (cu[b + 1] - cu[b]), lens[b])
        phys[cu[b]:cu[b + 1]], slot[cu[b]:cu[b + 1]] = bt[b, pos // ps], pos % ps
    got, key = [], None
    at = torch.from_numpy(phys).cuda(), torch.from_numpy(slot).cuda()
    for name, codes in (("k", x["k8"]), ("v", x["v8"])):
        rows = x[name].double()
        top = rows.abs().amax(-1, keepdim=True)
        # the least power of two that brings the row within 448
        scale = _exp2(torch.ceil(torch.log2(top / 448)).clamp(E_MIN, E_MAX))
        y = rows / scale
        grid = _exp2(torch.floor(torch.log2(y.abs().clamp_min(2.0 ** -6)))) / 8
        y = torch.round(y / grid) * grid                         # three bits behind the leading one
        whole = codes.double()
        whole[at[0], :, at[1]] = y
        got.append(whole)
        key = y * scale if key is None else key
    meta = x["meta"].double()
    new = torch.full((meta.shape[0], ps) + meta.shape[1:2] + (D,), math.nan, dtype=torch.float64,
                     device="cuda")
    new[at[0], at[1]] = key
    some = ~new.isnan().all(1)
    keep = torch.ones(meta.shape[0], dtype=torch.bool, device="cuda")
    keep[at[0][at[1] == 0]] = False
    for j, (reduce, none) in enumerate(((torch.amin, math.inf), (torch.amax, -math.inf))):
        n = reduce(torch.where(new.isnan(), none, new), 1)
        o = torch.where(keep[:, None, None], meta[:, :, j], none)
        both = torch.minimum(n, o) if j == 0 else torch.maximum(n, o)
        meta[:, :, j] = torch.where(some, both, meta[:, :, j])
    return got[0], got[1], None, meta


def _exact_attend(x, case):
    ps, B, Hq, Hkv = case["ps"], case["batch"], case["hq"], case["hkv"]
    lens = x["seq_lens"].cpu().numpy()
    out = torch.zeros((B, Hq, D), dtype=torch.float64, device="cuda")
    heads = torch.arange(Hkv, device="cuda")[:, None]
    for b in range(B):
        n = -(-int(lens[b]) // ps)
        if case["kind"] == "dense":
            pages = torch.arange(n, device="cuda").expand(Hkv, n)
        else:
            pages = x["idx"][b, :, :int(x["n"][b])].long()
        phys = x["bt"][b].long()[pages]
        pos = (pages[..., None] * ps + torch.arange(ps, device="cuda")).flatten(1)
        e = x["exps"][phys, heads]
        k, v = (_exact_values(c.view(torch.uint8)[phys, heads].view(torch.float8_e4m3fn), e, j)
                .flatten(1, 2) for j, c in enumerate((x["k8"], x["v8"])))
        q = x["q"][b].double().view(Hkv, Hq // Hkv, D)
        z = torch.matmul(q, k.transpose(1, 2).contiguous()) / math.sqrt(D)
        z = torch.where((pos < int(lens[b]))[:, None], z, -math.inf)
        out[b] = torch.matmul(torch.softmax(z, -1), v).view(Hq, D)
    return out
