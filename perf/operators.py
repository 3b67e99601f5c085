"""The paged operators as a serving program calls them, one layer of a model with many requests.

Kinds of cases, each with its plain form (elementary torch operations in 32 bits) and the framework's call:
  plan     one serving step's bookkeeping: finished requests give their pages back, new tokens get pages, slots and positions
  append   norms of queries and keys per head, rotary positions, queries out, keys and values into their pages
  decode   attention of one new token per request over its pages
  prefill  causal attention of a ragged batch of chunks over pages that hold them already, with or without a sliding window

Head layouts are those of `synth.WORKLOADS`, of the tests and of bench.py; pages of 16 to 128 units.
"""
import math
import random

import torch

own = False

DEV = "cuda:0"

LLAMA = dict(h=32, h_kv=8, d=128)
PHI3 = dict(h=32, h_kv=32, d=96)
NARROW = dict(h=32, h_kv=8, d=64)
SMALL = dict(h=8, h_kv=2, d=64)

DEFAULTS = dict(kind="decode", dtype="bf16", page=64, h=8, h_kv=2, d=64, shape=0, n_req=1, longest=1, window=0, sink=0,
                T=1, longest_new=1, far=4096, norm=False, rot=0, interleaved=False, theta=10000.0, stretch=1.0)


def _case(name=None, **kw):
    c = dict(DEFAULTS, **kw)
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # One generated token for each of 48 running requests: the bookkeeping of a decode step.
        _case("plan_step", kind="plan", n_req=48, longest=8192, longest_new=1, page=64),
        # Prompts of a large batch arriving beside running requests, small pages: some 100 thousand tokens.
        _case("plan_prompts", kind="plan", n_req=512, longest=16384, longest_new=1024, page=16),
        # A decode step of 48 requests far into their contexts, frequencies scaled for long contexts.
        _case("append_step", kind="append", **LLAMA, T=48, far=131072, rot=128, theta=500000.0, stretch=8.0),
        # The prompt chunks of a batch, with norms of queries and keys.
        _case("append_prompts", kind="append", **LLAMA, T=8192, far=32768, norm=True, rot=128, theta=500000.0, page=128),
        # A float32 layer, part of the head rotated in interleaved pairs, an odd number of tokens.
        _case("append_f32", kind="append", dtype="f32", h=32, h_kv=32, d=96, T=1111, far=4096, norm=True, rot=48, interleaved=True, page=16),
        # Generation for a single request on a 16K cache: latency.
        _case("decode_single", **LLAMA, n_req=1, longest=16421, page=64, shape=1),
        # A full batch of requests of very different lengths.
        _case("decode_batch", **LLAMA, n_req=64, longest=32768, page=64, shape=2),
        # Many KV heads, sliding window with a few first units kept.
        _case("decode_window", **PHI3, n_req=40, longest=12000, window=2048, sink=4, page=32, shape=3),
        # A float32 layer, a handful of short requests.
        _case("decode_f32", dtype="f32", **SMALL, n_req=6, longest=1500, page=16, shape=4),
        # A chunk of a long prompt on what is cached of it.
        _case("prefill_chunk", kind="prefill", **LLAMA, n_req=1, longest=16384, longest_new=4096, page=64, shape=5),
        # Short prompts and continued ones together, window and sinks, small pages.
        _case("prefill_ragged", kind="prefill", **NARROW, n_req=12, longest=5000, longest_new=700, window=1024, sink=4, page=16, shape=6),
        # A float32 layer's prompts.
        _case("prefill_f32", kind="prefill", dtype="f32", **SMALL, n_req=3, longest=900, longest_new=400, page=32, shape=7),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: sizes spread over what the listed cases stand for, odd ones among them."""
    kind = rng.choice(["plan", "append", "append", "decode", "decode", "decode", "prefill", "prefill", "prefill"])
    c = dict(kind=kind, page=rng.choice([16, 32, 64, 128]), shape=rng.randrange(8, 1 << 20))
    if kind == "plan":
        c.update(n_req=_log(rng, 1, 512), longest=_log(rng, 200, 16384))
        c["longest_new"] = rng.choice([1, _log(rng, 1, 1024)])
        return _case(**c)
    c["dtype"] = "f32" if rng.random() < 0.2 else "bf16"
    c.update(rng.choice([LLAMA, LLAMA, PHI3, NARROW, SMALL, dict(h=16, h_kv=4, d=128), dict(h=12, h_kv=2, d=32)]))
    if kind == "append":
        c.update(T=_log(rng, 1, 8192), far=_log(rng, 8192, 1 << 20), norm=rng.random() < 0.5, interleaved=rng.random() < 0.3,
                 rot=rng.choice([c["d"], c["d"], c["d"] // 2]), theta=rng.choice([10000.0, 500000.0]), stretch=rng.choice([1.0, 1.0, 4.0, 8.0]))
        if c["dtype"] == "f32":
            c["T"] = max(1, c["T"] // 4)
        return _case(**c)
    if rng.random() < 0.35:
        c.update(window=_log(rng, 64, 4096), sink=rng.choice([0, 1, 4, 64]))
    if kind == "decode":
        c["n_req"] = _log(rng, 1, 64)
        c["longest"] = _log(rng, 64, min(32768, (1 << 31) // (c["n_req"] * c["h_kv"] * c["d"] * 2)))
        return _case(**c)
    c["n_req"] = _log(rng, 1, 16)
    c["longest_new"] = _log(rng, 16, 4096 // c["n_req"])
    c["longest"] = max(c["longest_new"], _log(rng, 32, 16384 // c["n_req"]))
    if c["dtype"] == "f32":
        c["longest_new"] = min(c["longest_new"], 400)
        c["longest"] = max(c["longest_new"], min(c["longest"], 2000))
    return _case(**c)


# ---- the inputs ------------------------------------------------------------------------------------------------------
def _lens(c):
    """(units in the cache after the step, new tokens among them) of every request: ragged, the first one the longest."""
    r = random.Random(c["shape"])
    lens, new = [], []
    for i in range(c["n_req"]):
        n = c["longest"] if i == 0 else _log(r, max(1, c["longest"] // 16), c["longest"])
        k = 1 if c["kind"] == "decode" else min(n, c["longest_new"] if i == 0 else _log(r, max(1, c["longest_new"] // 16), c["longest_new"]))
        lens.append(n)
        new.append(k)
    return lens, new


def _type(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def _frequencies(c):
    """Radians a position of every rotated pair; `stretch` > 1 slows the low ones down, as contexts are extended (bands: wavelengths
    up to 2048 positions stay, those from 8192 on are `stretch` times as long, in between the two are mixed)."""
    f = []
    for i in range(c["rot"] // 2):
        x = c["theta"] ** (-2.0 * i / c["rot"])
        wave = 2 * math.pi / x
        s = 1.0 if c["stretch"] == 1.0 else min(1.0, max(0.0, (8192.0 / wave - 1.0) / 3.0))
        f.append((1 - s) * x / c["stretch"] + s * x)
    return f


def prepare(case, seed):
    c = _case(**case)
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    ints = dict(dtype=torch.int32, device=DEV)
    t, page, h, h_kv, d = _type(c), c["page"], c["h"], c["h_kv"], c["d"]

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=DEV, dtype=torch.float32).to(t)

    s = {"case": c}
    if c["kind"] == "plan":
        n = c["n_req"]
        s["max_pages"] = (c["longest"] + c["longest_new"] + page - 1) // page
        lens = (c["longest"] * torch.rand(n, generator=g, device=DEV)).to(torch.int32)
        new = 1 + (c["longest_new"] * torch.rand(n, generator=g, device=DEV)).to(torch.int32).clamp(max=c["longest_new"] - 1)
        fate = torch.rand(n, generator=g, device=DEV)
        lens = torch.where(fate < 0.1, 0, lens)                        # prompts that begin
        new = torch.where((fate > 0.9) & (fate < 0.95), -1, new)       # finished requests
        new = torch.where(fate >= 0.95, 0, new)                        # requests that wait
        held = (lens + page - 1) // page
        s["n_pages"] = n * s["max_pages"] + 1
        order = torch.randperm(s["n_pages"], generator=g, device=DEV).to(torch.int32)
        first = torch.cumsum(held, 0) - held
        p = torch.arange(s["max_pages"], **ints)
        s["table"] = torch.where(p < held[:, None], order[(first[:, None] + p).clamp(max=s["n_pages"] - 1).long()], -1).to(torch.int32)
        total = held.sum()
        s["n_free"] = (s["n_pages"] - total).to(torch.int32).reshape(1)
        s["free"] = order.roll(-int(total)).contiguous()
        s["lens"], s["new"] = lens.to(torch.int32), new.to(torch.int32)
        s["max_tokens"] = n * c["longest_new"]
        s["out"] = dict(lens=torch.empty(n, **ints), n_free=torch.empty(1, **ints), cu=torch.empty(n + 1, **ints),
                        slots=torch.empty(s["max_tokens"], **ints), positions=torch.empty(s["max_tokens"], **ints))
    elif c["kind"] == "append":
        T = c["T"]
        s["n_pages"] = 2 * T // page + 2
        # queries, keys and values lie beside each other, as one product with the three weights leaves them
        qkv = normal(T, (h + 2 * h_kv) * d) * 1.5
        s["q"], s["k"], s["v"] = (x.unflatten(1, (-1, d)) for x in qkv.split([h * d, h_kv * d, h_kv * d], 1))
        s["positions"] = (c["far"] * torch.rand(T, generator=g, device=DEV)).to(torch.int32)
        slots = torch.randperm(s["n_pages"] * page, generator=g, device=DEV)[:T]
        s["slots"] = torch.where(torch.rand(T, generator=g, device=DEV) < 0.02, -1, slots).to(torch.int32)   # padding of the batch
        s["freq"] = torch.tensor(_frequencies(c), dtype=torch.float64, device=DEV)
        s["wq"] = 1 + 0.2 * torch.randn(d, generator=g, device=DEV) if c["norm"] else None
        s["wk"] = 1 + 0.2 * torch.randn(d, generator=g, device=DEV) if c["norm"] else None
        s["K"], s["V"] = normal(s["n_pages"] + 1, h_kv, page, d), normal(s["n_pages"] + 1, h_kv, page, d)    # the last page: the plain form's
        s["out"] = torch.empty(T, h, d, dtype=t, device=DEV)
    else:
        lens, new = _lens(c)
        s["max_pages"] = (max(lens) + page - 1) // page
        held = [(n + page - 1) // page for n in lens]
        s["n_pages"] = sum(held) + 3
        order = torch.randperm(s["n_pages"], generator=g, device=DEV).to(torch.int32)
        first = torch.tensor([sum(held[:i]) for i in range(len(held))], device=DEV)
        at = (first[:, None] + torch.arange(s["max_pages"], device=DEV)).clamp(max=s["n_pages"] - 1)
        s["table"] = order[at].contiguous()
        s["lens"] = torch.tensor(lens, **ints)
        s["K"], s["V"] = normal(s["n_pages"], h_kv, page, d), normal(s["n_pages"], h_kv, page, d)
        T = sum(new)
        s["q"] = normal(T, h, d) * 2
        s["longest"], s["longest_new"], s["T"] = max(lens), max(new), T
        s["cu"] = torch.tensor([sum(new[:i]) for i in range(len(new) + 1)], **ints)
        s["out"] = torch.empty(T, h, d, dtype=t, device=DEV)
        s["lse"] = torch.empty(T, h, dtype=torch.float32, device=DEV)
    if own:
        from paper_2410_01805_amd import binding as B
        s["cfg"] = B.locret_paged_config(h, h_kv, d, B.LOCRET_F32 if c["dtype"] == "f32" else B.LOCRET_BF16, page, s["n_pages"],
                                         c["n_req"], s.get("max_pages", 1), c["window"], c["sink"], 0.0)
        s["work"] = torch.empty(B.locret_paged_workspace_bytes(s["cfg"]), dtype=torch.uint8, device=DEV)
    return s


# ---- one pass --------------------------------------------------------------------------------------------------------
def run(s):
    kind = s["case"]["kind"]
    if own:
        return _run_own(s, kind)
    return {"plan": _plan, "append": _append, "decode": _decode, "prefill": _prefill}[kind](s)


def _run_own(s, kind):
    from paper_2410_01805_amd import binding as B
    c, o = s["case"], s["out"]
    if kind == "plan":
        B.locret_paged_plan(s["cfg"], c["n_req"], s["lens"], s["new"], o["lens"], s["table"], s["free"], s["n_free"], o["n_free"],
                            s["max_tokens"], o["cu"], o["slots"], o["positions"])
        return dict(o, table=s["table"], free=s["free"])
    if kind == "append":
        B.locret_paged_append(s["cfg"], c["T"], s["q"], s["k"], s["v"], s["positions"], s["slots"], s["freq"], c["rot"],
                              c["interleaved"], 1.0, s["wq"], s["wk"], 1e-6, o, s["K"], s["V"])
        return dict(q=o, K=s["K"][:-1], V=s["V"][:-1])
    if kind == "decode":
        B.locret_paged_decode(s["cfg"], c["n_req"], s["q"], s["K"], s["V"], s["table"], s["lens"], o, s["lse"], s["work"])
    else:
        B.locret_paged_prefill(s["cfg"], c["n_req"], s["T"], s["q"], s["K"], s["V"], s["table"], s["lens"], s["cu"], o, s["lse"], s["work"])
    return dict(out=o, lse=s["lse"])


def _plan(s):
    """All in whole numbers.  Requests are served in their order, their pages come from the end of the list of free ones; the pages of
    finished requests join that list first.  (In these cases every request's pages are there.)"""
    page = s["case"]["page"]
    lens, new, table = s["lens"].long(), s["new"].long(), s["table"]
    p = torch.arange(s["max_pages"], device=DEV)
    held = (lens + page - 1) // page
    done = new < 0
    back = torch.where(done, held, 0)
    at = s["n_free"].long() + (torch.cumsum(back, 0) - back)[:, None] + p
    free = torch.cat([s["free"], s["free"][:1]])                      # one entry more: where what is not given back goes
    at = torch.where(p < back[:, None], at, s["n_pages"])
    free = free.scatter(0, at.flatten(), table.flatten())[:-1]
    n_free = s["n_free"].long() + back.sum()
    new = torch.where(done, 0, new)
    after = torch.where(done, 0, lens) + new
    want = torch.where(done, 0, (after + page - 1) // page - held)
    i = n_free - 1 - ((torch.cumsum(want, 0) - want)[:, None] + p - held[:, None])
    takes = (p >= held[:, None]) & (p < (held + want)[:, None])
    table = torch.where(takes, free[i.clamp(0, s["n_pages"] - 1)], table)
    cu = torch.cat([torch.zeros(1, dtype=torch.long, device=DEV), torch.cumsum(new, 0)])
    t = torch.arange(s["max_tokens"], device=DEV)
    r = (torch.searchsorted(cu, t, right=True) - 1).clamp(max=len(lens) - 1)
    pos = (lens[r] + t - cu[r])
    slot = table[r, (pos // page).clamp(0, s["max_pages"] - 1)] * page + pos % page
    inside = t < cu[-1]
    w = torch.int32
    return dict(lens=after.to(w), n_free=(n_free - want.sum()).to(w), cu=cu.to(w), slots=torch.where(inside, slot, -1).to(w),
                positions=torch.where(inside, pos, 0).to(w), table=table, free=free)


def _append(s):
    c = s["case"]
    rot, page = c["rot"], c["page"]
    angle = s["positions"].double()[:, None] * s["freq"]
    cos, sin = (f(angle).float()[:, None] for f in (torch.cos, torch.sin))

    def turned(x, w):
        x = x.float()
        if w is not None:
            x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6) * w
        y, rest = x[..., :rot], x[..., rot:]
        if c["interleaved"]:
            a, b = y[..., 0::2], y[..., 1::2]
            y = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
        else:
            a, b = y[..., : rot // 2], y[..., rot // 2:]
            y = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
        return torch.cat([y, rest], -1).to(_type(c))

    slot = torch.where(s["slots"] >= 0, s["slots"], s["n_pages"] * page).long()     # what has no slot goes to the spare page
    at, row = slot // page, slot % page
    s["K"][at, :, row] = turned(s["k"], s["wk"])
    s["V"][at, :, row] = s["v"]
    return dict(q=turned(s["q"], s["wq"]), K=s["K"][:-1], V=s["V"][:-1])


def _pages(s, X):
    """[request][KV head][unit][dim] in 32 bits."""
    R, P = s["table"].shape
    x = X[s["table"].long()]                                          # [R][P][h_kv][page][d]
    return x.transpose(1, 2).reshape(R, X.shape[1], P * X.shape[2], X.shape[3]).float()


def _seen(s, pos):
    """Which units each position sees: pos [request][...], -> [request][...][unit]."""
    c = s["case"]
    j = torch.arange(s["max_pages"] * c["page"], device=DEV)
    p = pos[..., None]
    see = j <= p
    if c["window"]:
        see = see & ((p - j < c["window"]) | (j < c["sink"]))
    return see


def _attend(s, q, see):
    """q [R][h_kv][rows][d], see [R][1][rows][units] -> (outputs, log sums of the exponentials)."""
    x = torch.matmul(q * (1.0 / math.sqrt(q.shape[-1])), _pages(s, s["K"]).transpose(2, 3).contiguous())
    x.masked_fill_(~see, -math.inf)
    top = x.amax(-1, keepdim=True)
    x.sub_(top).exp_()
    total = x.sum(-1, keepdim=True)
    return torch.matmul(x, _pages(s, s["V"])) / total, (top + total.log())[..., 0]


def _decode(s):
    c = s["case"]
    R, h, h_kv = c["n_req"], c["h"], c["h_kv"]
    out, lse = _attend(s, s["q"].float().view(R, h_kv, h // h_kv, c["d"]), _seen(s, s["lens"][:, None] - 1)[:, None])
    return dict(out=out.reshape(R, h, c["d"]).to(_type(c)), lse=lse.reshape(R, h))


def _prefill(s):
    c = s["case"]
    R, h, h_kv, d = c["n_req"], c["h"], c["h_kv"], c["d"]
    g, n = h // h_kv, s["longest_new"]
    cu = s["cu"].long()
    t = torch.arange(s["T"], device=DEV)
    r = torch.searchsorted(cu, t, right=True) - 1
    i = t - cu[r]
    q = torch.zeros(R, n, h, d, device=DEV)
    q[r, i] = s["q"].float()
    pos = (s["lens"] - s["cu"].diff())[:, None] + torch.arange(n, device=DEV)
    see = _seen(s, pos)[:, None]                                       # [R][1][n][units]
    q = q.view(R, n, h_kv, g, d).permute(0, 2, 3, 1, 4).reshape(R, h_kv, g * n, d)
    out, lse = _attend(s, q, see.repeat(1, 1, g, 1))
    out = out.view(R, h_kv, g, n, d).permute(0, 3, 1, 2, 4).reshape(R, n, h, d)
    lse = lse.view(R, h_kv, g, n).permute(0, 3, 1, 2).reshape(R, n, h)
    return dict(out=out[r, i].to(_type(c)), lse=lse[r, i].contiguous())


# ---- what a pass cannot do without -----------------------------------------------------------------------------------
def _visible(c, p):
    """Units that position p sees."""
    if not c["window"] or p < c["window"]:
        return p + 1
    return c["window"] + min(c["sink"], p + 1 - c["window"])


def work(case):
    c = _case(**case)
    h, h_kv, d, es = c["h"], c["h_kv"], c["d"], 4 if c["dtype"] == "f32" else 2
    if c["kind"] == "plan":
        tokens = c["n_req"] * (1 + c["longest_new"]) / 2
        return {"bytes": c["n_req"] * 16 + 8 * tokens / c["page"] + 8 * c["n_req"] * c["longest_new"], "flops": 0}
    if c["kind"] == "append":
        return {"bytes": c["T"] * (2 * (h + 2 * h_kv) * d * es + 8), "flops": c["T"] * (h + h_kv) * (3 * c["rot"] + (4 * d if c["norm"] else 0))}
    lens, new = _lens(c)
    pairs = sum(_visible(c, p) for n, k in zip(lens, new) for p in range(n - k, n))
    if c["window"]:
        units = sum(min(n, c["sink"] + c["window"] + k - 1) for n, k in zip(lens, new))
    else:
        units = sum(lens)
    return {"bytes": units * h_kv * d * 2 * es + sum(new) * h * (2 * d * es + 4) + 4 * units / c["page"], "flops": 4 * pairs * h * d}


# ---- the definitions in 64 bits ----------------------------------------------------------------------------------------
def exact(case, seed):
    c = _case(**case)
    if c["kind"] == "plan":
        return None                                                    # whole numbers
    s = prepare(case, seed)
    if c["kind"] == "append":
        T, d, rot, page = c["T"], c["d"], c["rot"], c["page"]
        turn = torch.polar(torch.ones(1, dtype=torch.float64, device=DEV), s["positions"].double()[:, None, None] * s["freq"])

        def made(x, w):
            x = x.double()
            if w is not None:
                x = x / (x.square().sum(-1, keepdim=True) / d + 1e-6).sqrt() * w.double()
            pairs = x[..., :rot].unflatten(-1, (rot // 2, 2) if c["interleaved"] else (2, rot // 2))
            if not c["interleaved"]:
                pairs = pairs.transpose(-1, -2)
            z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
            if not c["interleaved"]:
                z = z.transpose(-1, -2)
            return torch.cat([z.flatten(-2), x[..., rot:]], -1)

        K, V = s["K"][:-1].double(), s["V"][:-1].double()
        has = (s["slots"] >= 0).nonzero()[:, 0]
        at, row = s["slots"][has].long() // page, s["slots"][has].long() % page
        K[at, :, row] = made(s["k"], s["wk"])[has]
        V[at, :, row] = s["v"].double()[has]
        return dict(q=made(s["q"], s["wq"]), K=K, V=V)
    lens, new = _lens(c)
    h, h_kv, d, page = c["h"], c["h_kv"], c["d"], c["page"]
    if sum(n * k for n, k in zip(lens, new)) * h * d * 4 > 4e12:
        return None
    outs, sums = [], []
    first = 0
    for r, (n, k) in enumerate(zip(lens, new)):
        pages = s["table"][r, : (n + page - 1) // page].long()
        j = torch.arange(n, device=DEV)
        o, l = [], []
        for m in range(h_kv):
            K, V = (X[pages, m].reshape(-1, d)[:n].double() for X in (s["K"], s["V"]))
            for head in range(m * (h // h_kv), (m + 1) * (h // h_kv)):
                x = s["q"][first: first + k, head].double() @ K.t().contiguous() / math.sqrt(d)
                p = torch.arange(n - k, n, device=DEV)[:, None]
                hidden = j > p
                if c["window"]:
                    hidden = hidden | ((p - j >= c["window"]) & (j >= c["sink"]))
                x[hidden] = -math.inf
                l.append(torch.logsumexp(x, -1))
                o.append(torch.softmax(x, -1) @ V)
        outs.append(torch.stack(o, 1))
        sums.append(torch.stack(l, 1))
        first += k
    return dict(out=torch.cat(outs), lse=torch.cat(sums))
