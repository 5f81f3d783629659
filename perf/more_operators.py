"""The operators of a paged cache, as timed cases.

What a serving program uses for requests whose keys and values lie in pages, each beside the one before:

  rotate  infllm_rotate         per-head norms of the queries and keys and the rotation to their positions, one pass
  append  infllm_paged_append   the new tokens' keys and values into their pages, normed and rotated on the way, and the
                                queries rotated with them
  attend  infllm_paged_attend   causal attention of the new tokens over their sequences' pages: single tokens, chunks, and
                                both in one batch
  scored  infllm_paged_attend   the same with capped scores, a bias by distance, or a window beside the initial tokens

A case is one call on one layer.  Where `own` is false `run` computes the same in elementary torch operations, in
32 bits (angles in 64), rounded once at the end.
"""
from __future__ import annotations

import math

import torch

own = False

# the layer of the repository's workloads: 32 query and 8 kv heads of 128 dims; rotary base 500,000
_LAYER = dict(dtype="bf16", hq=32, hkv=8, d=128, base=500000.0, eps=1e-5, page=64, order="heads",
              rot=128, pairs="half", norm=False, scaled="", cap=0.0, slopes=False, window=0, init=0)


def _case(**kw):
    return dict(_LAYER, **kw)


def _text(xs):
    return ",".join(str(x) for x in xs)


def _spread(n, longest, shortest):
    return _text(longest - (longest - shortest) * i // max(1, n - 1) for i in range(n))


def listed():
    return [
        # sixteen sequences that decode, far into their streams: the smallest call
        _case(name="rotate_step", kind="rotate", pairs="interleaved", tokens=16, far=1000000),
        # a long prompt of a model with normed heads and frequencies scaled for long contexts
        _case(name="rotate_prompt", kind="rotate", norm=True, scaled="parts", tokens=16000, far=16000),
        # thirty-two sequences that decode
        _case(name="append_step", kind="append", norm=True, page=16, news=_text([1] * 32), pasts=_spread(32, 120000, 37)),
        # a prefill batch of a server, half of each head rotated
        _case(name="append_prompts", kind="append", rot=64,
              news="1,17,64,65,129,250,251,300,512,640,777,901,1024,1031,1300,1501,1777,2048,2100,2999", pasts=_text([0] * 20)),
        # one answer: the smallest decoding step
        _case(name="attend_step_1x2k", kind="attend", page=16, news="1", pasts="2011"),
        # a decoding batch of every length
        _case(name="attend_step_48", kind="attend", page=16, news=_text([1] * 48), pasts=_spread(48, 20000, 90)),
        # a batch in flight: a chunk of a long prompt, a fresh short one, and sequences that decode
        _case(name="attend_mixed", kind="attend", order="tokens", news=_text([512, 300] + [1] * 30),
              pasts="7500,0," + _spread(30, 9000, 200)),
        # a large chunk of one long prompt
        _case(name="attend_chunk_64k", kind="attend", page=128, news="2048", pasts="64000"),
        # the accuracy path: float32, a smaller layer, pages that end inside every tile
        _case(name="attend_f32", kind="attend", dtype="f32", hq=8, hkv=2, d=64, page=24, news="1,40,200,389,7", pasts="900,0,1000,33,2600"),
        # capped scores and a window, as alternating layers have: chunks of prompts
        _case(name="scored_cap_window", kind="scored", cap=50.0, window=4096, news="700,1500,64", pasts="9000,0,5000"),
        # a bias by distance: chunks and answers
        _case(name="scored_bias", kind="scored", slopes=True, news="300,1,1,800,25", pasts="2000,4100,700,6000,12000"),
        # a decoding batch that sees its initial tokens and a window, scores capped
        _case(name="scored_step_window", kind="scored", cap=30.0, window=4096, init=128, page=32, news=_text([1] * 32), pasts=_spread(32, 20000, 90)),
    ]


def draw(rng):
    """One more case of these ranges."""
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(("rotate", "append", "attend", "attend", "attend", "scored", "scored"))
    dtype = rng.choice(("bf16", "bf16", "bf16", "f32"))
    d = rng.choice((64, 128, 128))
    hkv = rng.choice((1, 2, 4, 8)) if dtype == "bf16" else rng.choice((1, 2, 4))
    hq = hkv * rng.choice((1, 2, 3, 4, 4, 5, 8)) if dtype == "bf16" else hkv * rng.choice((1, 2, 3, 4))
    common = dict(dtype=dtype, d=d, hkv=hkv, hq=hq, order=rng.choice(("heads", "tokens")),
                  page=rng.choice((1, 8, 16, 16, 24, 32, 50, 64, 64, 128, 256)))
    turned = dict(rot=rng.choice((d, d, d // 2, d // 4, 20)), pairs=rng.choice(("half", "interleaved")), norm=rng.random() < 0.5,
                  scaled=rng.choice(("", "linear", "parts")))
    if kind == "rotate":
        return _case(kind="rotate", tokens=log_int(1, 16000), far=log_int(16000, 1000000), **common, **turned)
    if kind == "append":
        n = log_int(1, 64)
        longest = log_int(1, 3000)
        news = [1] * n if rng.random() < 0.4 else [rng.randint(0, longest) for _ in range(n)]
        while sum(news) > 16000:
            news.pop()
        news = news or [1]
        return _case(kind="append", news=_text(news), pasts=_text(rng.randint(0, 120000) for _ in news), **common, **turned)
    n = log_int(1, 48)
    longest = log_int(20, 24000 if dtype == "bf16" else 4000)
    pasts = [rng.choice((0, rng.randint(0, longest), longest)) for _ in range(n)]
    shape = rng.choice(("steps", "chunks", "mixed"))
    most = log_int(2, 2048 if dtype == "bf16" else 400)
    news = [1 if shape == "steps" or shape == "mixed" and rng.random() < 0.8 else rng.randint(0, most) for _ in range(n)]
    budget = (8e10 if dtype == "bf16" else 8e9) / (hq * d)  # (query, key) pairs
    while len(news) > 1 and (sum(a * (a + b) for a, b in zip(news, pasts)) > budget or sum(pasts) > 400000):
        news.pop()
        pasts.pop()
    if sum(news) == 0:
        news[0] = 1
    extra = {}
    if kind == "scored":
        form = rng.choice(("cap", "bias", "window", "cap window", "bias window"))
        extra = dict(cap=rng.choice((15.0, 30.0, 50.0)) if "cap" in form else 0.0, slopes="bias" in form)
        if "window" in form:
            extra.update(window=log_int(1, 6000), init=rng.choice((0, 4, 64, 128)))
    return _case(kind=kind, news=_text(news), pasts=_text(pasts), **common, **extra)


# ------------------------------------------------------------------ geometry of a case
def _ints(text):
    return [int(x) for x in str(text).split(",")]


def _esize(c):
    return 2 if c["dtype"] == "bf16" else 4


def _dtype(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _frequencies(c):
    """The rotary frequencies (a list) and the factor of their cosines and sines."""
    theta = [c["base"] ** (-2.0 * i / c["rot"]) for i in range(c["rot"] // 2)]
    if c["scaled"] == "linear":
        return [t / 4.0 for t in theta], 1.0
    if c["scaled"] == "parts":
        # turns within the trained 8,192 tokens: fewer than 1 slowed by the factor, more than 32 kept
        out = []
        for t in theta:
            keep = min(1.0, max(0.0, (8192 * t / (2 * math.pi) - 1.0) / (32.0 - 1.0)))
            out.append(t * keep + t / 8.0 * (1.0 - keep))
        return out, 0.1 * math.log(8.0) + 1.0
    return theta, 1.0


def _pages_of(c, lens):
    return [(n + c["page"] - 1) // c["page"] for n in lens]


# ------------------------------------------------------------------ inputs
def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def normal(*shape, dtype=None, scale=1.0):
        return torch.randn(shape, generator=gen, device="cuda").mul_(scale).to(dtype or _dtype(c))

    s = {"case": c, "scale": c["d"] ** -0.5}
    d, hq, hkv, page = c["d"], c["hq"], c["hkv"], c["page"]
    if c["kind"] in ("rotate", "append"):
        s["theta"], s["magnitude"] = _frequencies(c)
        s["q_weight"] = normal(d, scale=0.2).add_(1.0)
        s["k_weight"] = normal(d, scale=0.2).add_(1.0)
        total = c["tokens"] if c["kind"] == "rotate" else sum(_ints(c["news"]))
        # the fused projection of all heads, token by token
        s["qkv"] = normal(max(1, total), (hq + 2 * hkv) * d)[:total]
    if c["kind"] == "rotate":
        # every token at a position of its own: decoding sequences, or a prompt's in their order
        s["at"] = (torch.randint(0, c["far"], (total,), generator=gen, device="cuda") if c["far"] > total
                   else torch.arange(total, device="cuda"))
        return s
    s["news"], s["pasts"] = _ints(c["news"]), _ints(c["pasts"])
    counts = _pages_of(c, [a + b for a, b in zip(s["news"], s["pasts"])])
    width = max(1, max(counts))
    table = torch.full((len(counts), width), -1, dtype=torch.int32)
    host = torch.Generator()
    host.manual_seed(seed)
    if c["kind"] == "append":
        # pages of their own for the new tokens; what lies before is not touched by the call
        first = [b // page for b in s["pasts"]]
        n_pages = sum(n - f for n, f in zip(counts, first)) + 3
    else:
        first = [0] * len(counts)
        n_pages = sum(counts) + 3
    order, at = torch.randperm(n_pages, generator=host).to(torch.int32), 0
    for i, (n, f) in enumerate(zip(counts, first)):
        table[i, :f] = int(order[-1])
        table[i, f:n] = order[at:at + n - f]
        at += n - f
    s["table"] = table.cuda()
    shape = (n_pages, hkv, page, d) if c["order"] == "heads" else (n_pages, page, hkv, d)
    s["k"], s["v"] = normal(*shape), normal(*shape)
    if c["kind"] == "append":
        return s
    s["q"] = normal(sum(s["news"]), hq, d)
    if c["cap"]:
        s["q"].mul_(c["cap"] / 5)  # scores that reach the cap
    if c["slopes"]:
        s["slopes"] = torch.tensor([2.0 ** (-8.0 * (h + 1) / hq) for h in range(hq)], dtype=torch.float32, device="cuda")
    return s


# ------------------------------------------------------------------ the framework's calls
def _plan(s):
    """What a program keeps for a layer: its parameters, structs and workspace."""
    if "plan" in s:
        return s["plan"]
    from paper_2402_04617_amd import infllm as F
    c = s["case"]
    d, hkv, page = c["d"], c["hkv"], c["page"]
    plan = {"F": F, "p": F.params(c["hq"], hkv, d, 0, 1, 1, 1, 0, dtype=c["dtype"], sm_scale=s["scale"])}
    if c["kind"] in ("rotate", "append"):
        plan["rot"] = F.rotary(s["theta"], interleaved=c["pairs"] == "interleaved", magnitude=s["magnitude"], norm=c["norm"],
                               q_weight=s["q_weight"], k_weight=s["k_weight"], eps=c["eps"])
    if c["kind"] != "rotate":
        heads = c["order"] == "heads"
        plan["pages"] = F.pages(s["k"], s["v"], page, page_stride=hkv * page * d, token_stride=d if heads else hkv * d,
                                head_stride=page * d if heads else d)
    if c["kind"] in ("attend", "scored"):
        plan["score"] = F.score(softcap=c["cap"], window=c["window"], n_init=c["init"], slopes=s.get("slopes")) if c["kind"] == "scored" else None
        size = F.infllm_paged_workspace_bytes(plan["p"], plan["pages"], s["news"], s["pasts"], plan["score"])
        plan["ws"] = torch.empty(max(256, size), dtype=torch.uint8, device="cuda")
    s["plan"] = plan
    return plan


def _run_own(s):
    c, plan = s["case"], _plan(s)
    F, p = plan["F"], plan["p"]
    d, hq, hkv = c["d"], c["hq"], c["hkv"]
    if c["kind"] in ("rotate", "append"):
        qkv = s["qkv"]
        total, row = qkv.shape[0], (hq + 2 * hkv) * d
        q, k, v = qkv, qkv[:, hq * d:], qkv[:, (hq + hkv) * d:]
        q_out = torch.empty((total, hq, d), dtype=qkv.dtype, device=qkv.device)
    if c["kind"] == "rotate":
        k_out = torch.empty((total, hkv, d), dtype=qkv.dtype, device=qkv.device)
        F.infllm_rotate(p, plan["rot"], total, s["at"], q, (row, d), q_out, (hq * d, d), k, (row, d), k_out, (hkv * d, d))
        return {"q": q_out, "k": k_out}
    if c["kind"] == "append":
        F.infllm_paged_append(p, plan["rot"], plan["pages"], s["news"], s["pasts"], s["table"], q, (row, d), q_out, (hq * d, d),
                              k, v, (row, d))
        return {"q": q_out, "k": s["k"], "v": s["v"]}
    out = torch.empty_like(s["q"])
    lse = torch.empty((hq, out.shape[0]), dtype=torch.float32, device="cuda")
    F.infllm_paged_attend(p, plan["pages"], s["news"], s["pasts"], s["table"], plan["score"], s["q"], (hq * d, d), out, (hq * d, d),
                          lse, plan["ws"])
    return {"out": out, "lse": lse}


# ------------------------------------------------------------------ the plain forms
def _turn(c, x, weight, theta, magnitude, at):
    """x [token][head][d] float32: normed, its first dims turned to the positions `at`."""
    if c["norm"]:
        x = x * torch.rsqrt((x * x).mean(dim=-1, keepdim=True) + c["eps"]) * weight.float()
    angle = at.double()[:, None] * torch.tensor(theta, dtype=torch.float64, device=x.device)
    cos, sin = (angle.cos() * magnitude).float()[:, None], (angle.sin() * magnitude).float()[:, None]
    r = c["rot"]
    if c["pairs"] == "half":
        a, b = x[..., :r // 2], x[..., r // 2:r]
        return torch.cat([a * cos - b * sin, a * sin + b * cos, x[..., r:]], dim=-1)
    a, b = x[..., :r:2], x[..., 1:r:2]
    return torch.cat([torch.stack([a * cos - b * sin, a * sin + b * cos], dim=-1).flatten(-2), x[..., r:]], dim=-1)


def _plain_turned(s, at):
    c = s["case"]
    d, hq, hkv = c["d"], c["hq"], c["hkv"]
    q, k, v = s["qkv"].view(-1, hq + 2 * hkv, d).split((hq, hkv, hkv), dim=1)
    q = _turn(c, q.float(), s["q_weight"], s["theta"], s["magnitude"], at)
    k = _turn(c, k.float(), s["k_weight"], s["theta"], s["magnitude"], at)
    return q.to(_dtype(c)), k.to(_dtype(c)), v


def _plain_append(s):
    c, page, dev = s["case"], s["case"]["page"], s["qkv"].device
    at = torch.cat([torch.arange(b, b + a, device=dev) for a, b in zip(s["news"], s["pasts"])])
    seq = torch.repeat_interleave(torch.arange(len(s["news"]), device=dev), torch.tensor(s["news"], device=dev))
    q, k, v = _plain_turned(s, at)
    where = s["table"][seq, at // page].long()
    for cache, rows in ((s["k"], k), (s["v"], v)):
        if c["order"] == "heads":
            cache[where, :, at % page] = rows
        else:
            cache[where, at % page] = rows
    return {"q": q, "k": s["k"], "v": s["v"]}


def _plain_attend(s):
    c = s["case"]
    d, hkv, page = c["d"], c["hkv"], c["page"]
    g, dev = c["hq"] // hkv, s["q"].device
    out = torch.empty_like(s["q"])
    lse = torch.empty((c["hq"], out.shape[0]), dtype=torch.float32, device=dev)
    first = 0
    for i, (new, past) in enumerate(zip(s["news"], s["pasts"])):
        if new == 0:
            continue
        end = past + new
        t = torch.arange(end, device=dev)
        pos = torch.arange(past, end, device=dev)
        seen = t[None, :] <= pos[:, None]
        if c["window"]:
            seen &= (t[None, :] > pos[:, None] - c["window"]) | (t[None, :] < c["init"])
        held = s["table"][i, :(end + page - 1) // page].long()
        x = s["q"][first:first + new].float().view(new, hkv, g, d)
        # all kv heads at once where the scores are few
        step = hkv if c["hq"] * new * end < 1 << 28 else 1
        for h in range(0, hkv, step):
            if c["order"] == "heads":
                k, v = (y[held, h:h + step].float().transpose(0, 1).reshape(step, -1, d)[:, :end] for y in (s["k"], s["v"]))
            else:
                k, v = (y[held, :, h:h + step].float().reshape(-1, step, d)[:end].transpose(0, 1).contiguous() for y in (s["k"], s["v"]))
            z = torch.matmul(x[:, h:h + step].permute(1, 2, 0, 3).reshape(step, g * new, d), k.transpose(-1, -2)).mul_(s["scale"])
            z = z.view(step, g, new, end)
            if c["cap"]:
                z = z.div_(c["cap"]).tanh_().mul_(c["cap"])
            if c["slopes"]:
                z -= s["slopes"].view(hkv, g, 1, 1)[h:h + step] * (pos[:, None] - t[None, :]).float()
            z.masked_fill_(~seen, -math.inf)
            top = z.amax(dim=-1, keepdim=True)
            e = z.sub_(top).exp_()
            total = e.sum(dim=-1, keepdim=True)
            o = torch.matmul(e.view(step, g * new, end), v).view(step, g, new, d) / total
            out[first:first + new, h * g:(h + step) * g] = o.permute(2, 0, 1, 3).reshape(new, step * g, d).to(out.dtype)
            lse[h * g:(h + step) * g, first:first + new] = (top + total.log()).view(step * g, new)
        first += new
    return {"out": out, "lse": lse}


def run(state):
    if own:
        return _run_own(state)
    kind = state["case"]["kind"]
    if kind == "rotate":
        q, k, _ = _plain_turned(state, state["at"])
        return {"q": q, "k": k}
    return _plain_append(state) if kind == "append" else _plain_attend(state)


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    c, e = case, _esize(case)
    d, hq, hkv = c["d"], c["hq"], c["hkv"]
    if c["kind"] == "rotate":
        return {"bytes": c["tokens"] * (2 * (hq + hkv) * d * e + 8), "flops": c["tokens"] * (hq + hkv) * 3 * c["rot"]}
    news, pasts = _ints(c["news"]), _ints(c["pasts"])
    if c["kind"] == "append":
        return {"bytes": sum(news) * 2 * (hq + 2 * hkv) * d * e, "flops": sum(news) * (hq + hkv) * 3 * c["rot"]}
    pairs = keys = 0
    for new, past in zip(news, pasts):
        if new == 0:
            continue
        if not c["window"]:
            pairs += new * past + new * (new + 1) // 2
            keys += past + new
            continue
        for p in range(past, past + new):
            low = max(0, p + 1 - c["window"])
            pairs += p + 1 - low + min(low, c["init"])
        low = max(0, past + 1 - c["window"])
        keys += past + new - low + min(low, c["init"])
    return {"bytes": keys * hkv * 2 * d * e + sum(news) * hq * (2 * d * e + 4) + 4 * sum(_pages_of(c, [a + b for a, b in zip(news, pasts)])),
            "flops": 4 * d * hq * pairs}


# ------------------------------------------------------------------ the definition in 64 bits
def _exact_turn(c, s, x, weight, at):
    """Rows x [token][head][d] in 64 bits: the norm, and each pair as a complex number times magnitude e^{i p theta}."""
    if c["norm"]:
        x = x / ((x ** 2).sum(-1, keepdim=True) / c["d"] + c["eps"]).sqrt() * weight.double()
    theta = torch.tensor(s["theta"], dtype=torch.float64, device=x.device)
    phase = torch.polar(torch.full_like(theta, s["magnitude"]).expand(len(at), -1).contiguous(), at.double()[:, None] * theta)
    n = c["rot"] // 2
    first = torch.arange(n, device=x.device) * (2 if c["pairs"] == "interleaved" else 1)
    second = first + (1 if c["pairs"] == "interleaved" else n)
    turned = torch.complex(x[..., first], x[..., second]) * phase[:, None]
    y = x.clone()
    y[..., first], y[..., second] = turned.real, turned.imag
    return y


def exact(case, seed):
    c = case
    d, hq, hkv, page = c["d"], c["hq"], c["hkv"], c["page"]
    g = hq // hkv
    s = prepare(case, seed)
    if c["kind"] == "rotate":
        x = s["qkv"].double().view(-1, hq + 2 * hkv, d)
        return {"q": _exact_turn(c, s, x[:, :hq], s["q_weight"], s["at"]), "k": _exact_turn(c, s, x[:, hq:hq + hkv], s["k_weight"], s["at"])}
    if c["kind"] == "append":
        x = s["qkv"].double().view(-1, hq + 2 * hkv, d)
        at = torch.tensor([b + j for a, b in zip(s["news"], s["pasts"]) for j in range(a)], device=x.device)
        k = _exact_turn(c, s, x[:, hq:hq + hkv], s["k_weight"], at)
        cache, row, table = s["k"].double(), 0, s["table"].cpu()
        for i, (new, past) in enumerate(zip(s["news"], s["pasts"])):
            done = 0
            while done < new:  # the run of tokens that one page takes
                t = past + done
                n = min(new - done, page - t % page)
                rows = k[row:row + n]
                slot = cache[int(table[i, t // page])]
                if c["order"] == "heads":
                    slot[:, t % page:t % page + n] = rows.transpose(0, 1)
                else:
                    slot[t % page:t % page + n] = rows
                done, row = done + n, row + n
        return {"q": _exact_turn(c, s, x[:, :hq], s["q_weight"], at), "k": cache, "v": None}
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros((hq, out.shape[0]), dtype=torch.float64, device="cuda")
    row = 0
    for i, (new, past) in enumerate(zip(s["news"], s["pasts"])):
        if new == 0:
            continue
        end = past + new
        distance = torch.arange(past, end, device="cuda")[:, None] - torch.arange(end, device="cuda")
        hidden = distance < 0
        if c["window"]:
            hidden |= (distance >= c["window"]) & (torch.arange(end, device="cuda") >= c["init"])
        at = s["table"][i].long().repeat_interleave(page)[:end]
        within = torch.arange(end, device="cuda") % page
        for h in range(hkv):
            k, v = ((y[at, h, within] if c["order"] == "heads" else y[at, within, h]).double() for y in (s["k"], s["v"]))
            for j in range(h * g, (h + 1) * g):
                z = s["q"][row:row + new, j].double() @ k.T * s["scale"]
                if c["cap"]:
                    z = c["cap"] * torch.tanh(z / c["cap"])
                if c["slopes"]:
                    z = z - s["slopes"][j].double() * distance
                z[hidden] = -math.inf
                lse[j, row:row + new] = torch.logsumexp(z, dim=-1)
                out[row:row + new, j] = torch.softmax(z, dim=-1) @ v
        row += new
    return {"out": out, "lse": lse}
