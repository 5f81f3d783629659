"""The operators of a batch that shares a document, as timed cases.

Four operators, which a program that serves many requests over long documents uses together:

  prompt  infllm_prompt_attend    causal attention of whole prompts of different lengths, packed one after another
  score   infllm_prefix_score     the relevance of a shared document's memory units to every continuation of it
  prefix  infllm_prefix_attend    attention of the continuations over the shared document (its keys read once for
                                  all of them), each one's looked-up units and its own tokens
  copy    infllm_copy_sequences   a layer's context memory forked to other batch slots, or compacted

A case is one call on one layer.  Where `own` is false `run` computes the same in elementary torch operations, in
32 bits, rounded once at the end.
"""
from __future__ import annotations

import math

import torch

own = False

# the layer of the repository's workloads: 32 query and 8 kv heads of 128 dims, 128 initial tokens, a 4K window,
# 128-token units, 4 representatives
_LAYER = dict(dtype="bf16", hq=32, hkv=8, d=128, init=128, local=4096, block=128, repr=4, topk=32)


def _case(**kw):
    return dict(_LAYER, **kw)


def listed():
    return [
        # one short question, nothing before it: the smallest call
        _case(name="prompt_short", kind="prompt", lens="45", order="heads"),
        # a prefill batch of a server: questions and passages of every length, projections token by token
        _case(name="prompt_packed", kind="prompt", order="tokens",
              lens="1,17,64,65,129,250,251,300,512,640,777,901,1024,1031,1300,1501,1777,2048,2100,2999"),
        # one long prompt, whole
        _case(name="prompt_16k", kind="prompt", lens="16000", order="tokens"),
        # the accuracy path: float32, a smaller layer
        _case(name="prompt_f32", kind="prompt", dtype="f32", hq=8, hkv=2, d=64, order="heads", lens="3,200,389,1000,1600"),
        # four continuations of a 32K document, a unit table of 217 units
        _case(name="score_4x32k", kind="score", batch=4, n=1, units=217),
        # sixteen continuations of a 1M document
        _case(name="score_16x1m", kind="score", batch=16, n=1, units=8155),
        # four answers sampled from one question about a 32K document: the smallest decoding step
        _case(name="prefix_4x32k", kind="prefix", batch=4, n=1, length=31999, topk=16, own=200, spread=180),
        # thirty-two users of one long prompt that is attended as a whole (a window as long as the prompt)
        _case(name="prefix_32x64k_whole", kind="prefix", batch=32, n=1, length=65536, local=65536, topk=0, own=700, spread=690),
        # verification of eight guessed tokens in eight continuations of a 128K document
        _case(name="prefix_8x128k_verify", kind="prefix", batch=8, n=8, length=130048, own=1500, spread=1400),
        # the accuracy path: float32, a smaller layer
        _case(name="prefix_f32", kind="prefix", dtype="f32", hq=8, hkv=2, d=64, batch=6, n=3, length=16001, init=64, local=1024,
              block=64, topk=16, own=333, spread=300),
        # a 128K document's memory forked to four slots, to be continued apart
        _case(name="copy_fork_128k", kind="copy", batch=4, slots=1, pairs="0>0,0>1,0>2,0>3", lens="131072", same=False),
        # a batch of eight from which some have finished, closed up in place
        _case(name="copy_compact", kind="copy", batch=8, slots=8, pairs="7>1,6>2,5>4", lens="1500,4097,9001", same=True),
    ]


def draw(rng):
    """One more case of these ranges."""
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(("prompt", "prompt", "prompt", "prefix", "prefix", "prefix", "score", "copy"))
    dtype = rng.choice(("bf16", "bf16", "bf16", "f32"))
    d = rng.choice((64, 128, 128))
    hkv = rng.choice((1, 2, 4, 8)) if dtype == "bf16" else rng.choice((1, 2, 4))
    hq = hkv * rng.choice((1, 2, 4, 4, 8)) if dtype == "bf16" else hkv * rng.choice((1, 2, 4))
    block = rng.choice((64, 128, 128, 256))
    common = dict(dtype=dtype, d=d, hkv=hkv, hq=hq, block=block)
    if kind == "prompt":
        longest = log_int(1, 8000 if dtype == "bf16" else 2000)
        most = max(1, min(64, (16000 ** 2 * 32 // (2 if dtype == "bf16" else 16)) // (hq * longest * longest)))
        lens = [longest] + [rng.randint(1, longest) for _ in range(log_int(1, most) - 1)]
        rng.shuffle(lens)
        return _case(kind="prompt", order=rng.choice(("heads", "tokens")), lens=",".join(map(str, lens)), **common)
    if kind == "score":
        return _case(kind="score", batch=log_int(1, 32), n=rng.choice((1, 1, log_int(2, 24))), units=log_int(1, 8155), **common)
    if kind == "copy":
        slots = rng.randint(2, 8)
        moved = rng.randint(1, slots // 2)
        lens = [log_int(1, 60000 if dtype == "bf16" else 20000) for _ in range(moved)]
        places = rng.sample(range(slots), 2 * moved)
        return _case(kind="copy", batch=slots, slots=slots, same=True, lens=",".join(map(str, lens)),
                     pairs=",".join("%d>%d" % (places[2 * i], places[2 * i + 1]) for i in range(moved)), **common)
    batch = log_int(1, 32)
    whole = rng.random() < 0.4
    length = log_int(100, 60000 if dtype == "bf16" else 8000)
    n = rng.choice((1, 1, 1, log_int(2, 12)))
    ahead = log_int(1, 2000)
    return _case(kind="prefix", batch=batch, n=n, length=length, local=max(length, 1) if whole else 4096 if dtype == "bf16" else 1024,
                 topk=0 if whole else min(rng.choice((8, 16, 32, 48)), 8192 // block), own=ahead, spread=rng.randint(0, ahead), **common)


# ------------------------------------------------------------------ geometry of a case
def _ints(text):
    return [int(x) for x in text.split(",")]


def _units(c, length):
    return max(0, (length - c["init"] - c["local"]) // c["block"])


def _own_lens(c):
    """Tokens of each continuation before the step."""
    return [c["own"] - (c["spread"] * b) // max(1, c["batch"] - 1) for b in range(c["batch"])]


def _pairs(c):
    """(source slot, destination slot, length, units built) of a copy."""
    lens = _ints(c["lens"])
    pairs = [tuple(map(int, x.split(">"))) for x in c["pairs"].split(",")]
    return [(s, t, lens[i % len(lens)], _units(c, lens[i % len(lens)])) for i, (s, t) in enumerate(pairs)]


def _esize(c):
    return 2 if c["dtype"] == "bf16" else 4


def _dtype(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


# ------------------------------------------------------------------ inputs
def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def normal(*shape, dtype=None, scale=1.0):
        return torch.randn(shape, generator=gen, device="cuda").mul_(scale).to(dtype or _dtype(c))

    s = {"case": c, "scale": c["d"] ** -0.5}
    if c["kind"] == "prompt":
        lens = _ints(c["lens"])
        total = sum(lens)
        s["lens"] = lens
        heads = [(total, h, c["d"]) if c["order"] == "tokens" else (h, total, c["d"]) for h in (c["hq"], c["hkv"], c["hkv"])]
        s["q"], s["k"], s["v"] = (normal(*shape) for shape in heads)
        return s
    if c["kind"] == "score":
        s["q"] = normal(c["batch"], c["hq"], c["n"], c["d"])
        s["ksum"] = normal(1, c["hkv"], c["d"] // 4, c["units"], 4, dtype=torch.float32, scale=2.0)
        return s
    if c["kind"] == "prefix":
        length, batch, n = c["length"], c["batch"], c["n"]
        room = c["own"] + n + 5
        s["q"] = normal(batch, c["hq"], n, c["d"])
        s["x_k"], s["x_v"] = normal(batch, c["hkv"], n, c["d"]), normal(batch, c["hkv"], n, c["d"])
        s["k"], s["v"] = normal(1, c["hkv"], length, c["d"]), normal(1, c["hkv"], length, c["d"])
        s["own_k"], s["own_v"] = normal(batch, c["hkv"], room, c["d"]), normal(batch, c["hkv"], room, c["d"])
        s["own_lens"] = _own_lens(c)
        units = _units(c, length)
        k = min(c["topk"], units)
        s["idx"] = None
        if c["topk"] > 0:
            # distinct units in ascending order and -1 behind them, as the lookup gives them
            s["idx"] = torch.full((batch, c["hkv"], c["topk"]), -1, dtype=torch.int32, device="cuda")
            score = torch.rand((batch, c["hkv"], max(units, 1)), generator=gen, device="cuda")
            s["idx"][..., :k] = score.topk(k, dim=-1).indices.sort(dim=-1).values.to(torch.int32)
        return s
    # copy: the memory of a layer, every part of it
    longest = max(x[2] for x in _pairs(c))
    units = max(1, _units(c, longest))
    ring = c["local"] + c["block"] + 2 * 512 + 1

    def memory(batch):
        return {"k": normal(batch, c["hkv"], longest, c["d"]), "v": normal(batch, c["hkv"], longest, c["d"]),
                "repr_idx": torch.randint(0, c["block"], (batch, c["hkv"], units, c["repr"]), generator=gen, device="cuda", dtype=torch.int32),
                "unit_ksum": normal(batch, c["hkv"], c["d"] // 4, units, 4, dtype=torch.float32),
                "qprefix": normal(batch, c["hkv"], ring, c["d"], dtype=torch.float64),
                "rpart": normal(batch, c["hkv"], c["d"] // 8, ring, dtype=torch.float64)}

    s["ring"], s["capacity"], s["units"] = ring, longest, units
    s["dst"] = memory(c["batch"])
    s["src"] = s["dst"] if c["same"] else memory(c["slots"])
    return s


# ------------------------------------------------------------------ the framework's calls
def _params(c, F):
    return F.params(c["hq"], c["hkv"], c["d"], c["init"], c["local"], c["block"], c["repr"], c["topk"], dtype=c["dtype"],
                    sm_scale=c["d"] ** -0.5)


def _plan(s):
    """What a program keeps for a layer: its parameters, memory structs and workspace."""
    if "plan" in s:
        return s["plan"]
    from paper_2402_04617_amd import infllm as F
    c = s["case"]
    p = _params(c, F)
    plan = {"F": F, "p": p}

    def struct(batch, capacity, units=0, ring=0, **tensors):
        m = F.Memory(batch=batch, capacity=capacity, max_units=units, ring=ring)
        for name, t in tensors.items():
            setattr(m, name, t.data_ptr())
        return m

    def workspace(size):
        return torch.empty(max(256, size), dtype=torch.uint8, device="cuda")

    if c["kind"] == "prompt":
        plan["ws"] = workspace(F.infllm_prompt_workspace_bytes(p, s["lens"]))
    elif c["kind"] == "score":
        plan["m"] = struct(1, 1, units=c["units"], unit_ksum=s["ksum"])
        plan["ws"] = workspace(F.infllm_prefix_workspace_bytes(p, c["batch"], c["n"], 0, 0))
    elif c["kind"] == "prefix":
        plan["m"] = struct(1, c["length"], k=s["k"], v=s["v"])
        plan["own"] = struct(c["batch"], s["own_k"].shape[2], k=s["own_k"], v=s["own_v"])
        plan["ws"] = workspace(F.infllm_prefix_workspace_bytes(p, c["batch"], c["n"], c["length"], s["own_k"].shape[2]))
    else:
        plan["dst"], plan["src"] = (struct(b, s["capacity"], units=s["units"], ring=s["ring"], **s[m])
                                    for m, b in (("dst", c["batch"]), ("src", c["slots"])))
        plan["pairs"] = tuple(zip(*_pairs(c)))
    s["plan"] = plan
    return plan


def _run_own(s):
    c, plan = s["case"], _plan(s)
    F, p = plan["F"], plan["p"]
    d = c["d"]
    if c["kind"] == "prompt":
        out = torch.empty_like(s["q"])
        tokens = c["order"] == "tokens"
        total = s["q"].shape[0 if tokens else 1]
        lse = torch.empty((c["hq"], total), dtype=torch.float32, device="cuda")
        q_st, kv_st = ((c["hq"] * d, d), (c["hkv"] * d, d)) if tokens else ((d, total * d), (d, total * d))
        F.infllm_prompt_attend(p, s["lens"], s["q"], q_st, s["k"], s["v"], kv_st, out, q_st, lse, plan["ws"])
        return {"out": out, "lse": lse}
    if c["kind"] == "score":
        scores = torch.empty((c["batch"], c["hkv"], c["units"]), dtype=torch.float32, device="cuda")
        F.infllm_prefix_score(p, plan["m"], c["batch"], s["q"], c["n"] * d, c["n"], c["units"], scores, plan["ws"])
        return {"scores": scores}
    if c["kind"] == "prefix":
        out = torch.empty_like(s["q"])
        lse = torch.empty(s["q"].shape[:3], dtype=torch.float32, device="cuda")
        F.infllm_prefix_attend(p, plan["m"], c["length"], plan["own"], s["own_lens"], s["q"], c["n"] * d, s["x_k"], s["x_v"],
                               c["n"] * d, c["n"], s["idx"], c["topk"], out, c["n"] * d, lse, plan["ws"])
        return {"out": out, "lse": lse, "own_k": s["own_k"], "own_v": s["own_v"]}
    src, dst, lens, built = plan["pairs"]
    F.infllm_copy_sequences(p, plan["dst"], plan["src"], dst, src, lens, built)
    return s["dst"]


# ------------------------------------------------------------------ the plain forms
def _softmax_parts(logits):
    """exp(logits - row maximum), the row's sum and its log-sum-exp; rows without a visible key give 0, 0 and -inf."""
    top = logits.amax(dim=-1, keepdim=True)
    top = torch.where(torch.isinf(top), torch.zeros_like(top), top)
    e = logits.sub_(top).exp_()
    total = e.sum(dim=-1, keepdim=True)
    return e, total, (top + total.log()).squeeze(-1)


def _plain_prompt(s):
    c, lens = s["case"], s["lens"]
    g, d, hkv = c["hq"] // c["hkv"], c["d"], c["hkv"]
    tokens = c["order"] == "tokens"
    q, k, v = (x.float() if tokens else x.float().transpose(0, 1) for x in (s["q"], s["k"], s["v"]))
    n, longest = len(lens), max(lens)
    length = torch.tensor(lens, device=q.device)
    at = torch.arange(longest, device=q.device)
    there = at < length[:, None]                                        # [n][longest]
    row = ((length.cumsum(0) - length)[:, None] + at).clamp(max=q.shape[0] - 1)
    qp = q[row].view(n, longest, hkv, g, d).permute(0, 2, 3, 1, 4).reshape(n, hkv, g * longest, d)
    kp, vp = (x[row].permute(0, 2, 1, 3) for x in (k, v))               # [n][hkv][longest][d]
    logits = torch.matmul(qp, kp.transpose(-1, -2)).mul_(s["scale"]).view(n, hkv, g, longest, longest)
    seen = (at[None, :] <= at[:, None]) & there[:, None, :]             # [n][query][key]
    logits.masked_fill_(~seen[:, None, None], -math.inf)
    e, total, lse = _softmax_parts(logits)
    out = torch.matmul(e.view(n, hkv, g * longest, longest), vp).view(n, hkv, g, longest, d) / total
    out = out.permute(0, 3, 1, 2, 4).reshape(n, longest, hkv * g, d)[there]  # [total][hq][d]
    lse = lse.permute(0, 3, 1, 2).reshape(n, longest, hkv * g)[there]
    out = out if tokens else out.transpose(0, 1)
    return {"out": out.to(_dtype(c)).contiguous(), "lse": lse.transpose(0, 1).contiguous()}


def _plain_score(s):
    c = s["case"]
    g = c["hq"] // c["hkv"]
    q = s["q"].float().view(c["batch"], c["hkv"], g * c["n"], c["d"]).sum(dim=2)
    ksum = s["ksum"][0].permute(0, 1, 3, 2).reshape(c["hkv"], c["d"], c["units"])
    return {"scores": torch.matmul(q.transpose(0, 1), ksum).transpose(0, 1).contiguous()}


def _plain_prefix(s):
    c, n, d, hkv, batch = s["case"], s["case"]["n"], s["case"]["d"], s["case"]["hkv"], s["case"]["batch"]
    g, length = c["hq"] // hkv, c["length"]
    dev = s["q"].device
    before = torch.tensor(s["own_lens"], device=dev)
    # the step's own keys and values join the continuation's
    b_at = torch.arange(batch, device=dev)[:, None]
    t_at = before[:, None] + torch.arange(n, device=dev)
    s["own_k"][b_at, :, t_at] = s["x_k"].transpose(1, 2)
    s["own_v"][b_at, :, t_at] = s["x_v"].transpose(1, 2)
    q = s["q"].float().view(batch, hkv, g, n, d).mul(s["scale"])
    units = _units(c, length)
    first = min(c["init"], length)
    shared = torch.cat([torch.arange(first, device=dev), torch.arange(first + units * c["block"], length, device=dev)])
    ks, vs = s["k"][0][:, shared].float(), s["v"][0][:, shared].float()  # [hkv][keys][d], once for all
    qs = q.transpose(0, 1).reshape(hkv, batch * g * n, d)
    logits = [torch.matmul(qs, ks.transpose(-1, -2)).view(hkv, batch, g * n, -1).transpose(0, 1)]
    qb = q.reshape(batch, hkv, g * n, d)
    kv = []
    if c["topk"] > 0 and units > 0:
        idx = s["idx"][..., :min(c["topk"], units)].long()
        pos = (c["init"] + idx[..., None] * c["block"] + torch.arange(c["block"], device=dev)).flatten(2)  # [batch][hkv][keys]
        h_at = torch.arange(hkv, device=dev)[None, :, None]
        ku, vu = s["k"][0][h_at, pos].float(), s["v"][0][h_at, pos].float()
        logits.append(torch.matmul(qb, ku.transpose(-1, -2)))
        kv.append(vu)
    ko, vo = s["own_k"].float(), s["own_v"].float()
    seen = torch.arange(ko.shape[2], device=dev) <= t_at[:, :, None]     # [batch][n][keys]
    lo = torch.matmul(qb, ko.transpose(-1, -2)).view(batch, hkv, g, n, -1)
    logits.append(lo.masked_fill_(~seen[:, None, None], -math.inf).view(batch, hkv, g * n, -1))
    kv.append(vo)
    sizes = [x.shape[-1] for x in logits]
    e, total, lse = _softmax_parts(torch.cat(logits, dim=-1))
    parts = e.split(sizes, dim=-1)
    out = torch.matmul(parts[0].transpose(0, 1).reshape(hkv, batch * g * n, -1), vs).view(hkv, batch, g * n, d).transpose(0, 1)
    out = out + torch.matmul(parts[-1], kv[-1])
    if len(parts) > 2:
        out = out + torch.matmul(parts[1], kv[0])
    return {"out": (out / total).reshape(batch, c["hq"], n, d).to(_dtype(c)), "lse": lse.reshape(batch, c["hq"], n),
            "own_k": s["own_k"], "own_v": s["own_v"]}


def _plain_copy(s):
    src, dst, ring = s["src"], s["dst"], s["ring"]
    for a, b, length, built in _pairs(s["case"]):  # whole runs at a time
        held = min(length, ring)  # (of shorter sequences the first slots)
        dst["k"][b, :, :length] = src["k"][a, :, :length]
        dst["v"][b, :, :length] = src["v"][a, :, :length]
        dst["repr_idx"][b, :, :built] = src["repr_idx"][a, :, :built]
        dst["unit_ksum"][b, :, :, :built] = src["unit_ksum"][a, :, :, :built]
        dst["qprefix"][b, :, :held] = src["qprefix"][a, :, :held]
        dst["rpart"][b, :, :, :held] = src["rpart"][a, :, :, :held]
    return dst


def run(state):
    if own:
        return _run_own(state)
    return {"prompt": _plain_prompt, "score": _plain_score, "prefix": _plain_prefix, "copy": _plain_copy}[state["case"]["kind"]](state)


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    c, e = case, _esize(case)
    d, hq, hkv = c["d"], c["hq"], c["hkv"]
    if c["kind"] == "prompt":
        lens = _ints(c["lens"])
        total = sum(lens)
        return {"bytes": total * (2 * hq + 2 * hkv) * d * e + total * hq * 4, "flops": sum(4 * d * hq * n * (n + 1) // 2 for n in lens)}
    if c["kind"] == "score":
        return {"bytes": hkv * d * c["units"] * 4 + c["batch"] * (hq * c["n"] * d * e + hkv * c["units"] * 4),
                "flops": 2 * c["batch"] * hkv * c["units"] * d}
    if c["kind"] == "prefix":
        units = _units(c, c["length"])
        looked = min(c["topk"], units) * c["block"]
        shared = c["length"] - units * c["block"]
        keys = min(c["batch"] * looked, units * c["block"]) + shared + sum(_own_lens(c))  # K and V rows of a kv head
        rows = c["batch"] * c["n"]
        return {"bytes": (keys + 2 * rows) * hkv * 2 * d * e + rows * hq * (2 * d * e + 4),
                "flops": sum(4 * d * hq * (c["n"] * (shared + looked + b) + c["n"] * (c["n"] + 1) // 2) for b in _own_lens(c))}
    ring = c["local"] + c["block"] + 2 * 512 + 1
    size = lambda n, u: hkv * (n * d * e * 2 + u * (c["repr"] * 4 + d * 4) + min(n, ring) * (d * 8 + d // 8 * 8))  # noqa: E731
    read = {a: size(n, u) for a, _, n, u in _pairs(c)}  # a source of several copies once
    return {"bytes": sum(read.values()) + sum(size(n, u) for _, _, n, u in _pairs(c)), "flops": 0}


# ------------------------------------------------------------------ the definition in 64 bits
def _attend64(q, k, v, scale, seen=None):
    """One softmax of scale * q . k over the rows of k; (output, log-sum-exp)."""
    z = (q @ k.T) * scale
    if seen is not None:
        z[~seen] = -math.inf
    lse = torch.logsumexp(z, dim=-1)
    return torch.exp(z - lse[:, None]) @ v, lse


def exact(case, seed):
    c = case
    if c["kind"] == "copy":
        return None
    s = prepare(case, seed)
    d, g = c["d"], c["hq"] // c["hkv"]
    scale = d ** -0.5
    if c["kind"] == "score":
        q, ks = s["q"].double(), s["ksum"][0].double().permute(0, 2, 1, 3).flatten(2)  # [hkv][units][d]
        by_group = q.view(c["batch"], c["hkv"], g, c["n"], d)
        return {"scores": torch.stack([torch.stack([(by_group[b, h].reshape(-1, d) @ ks[h].T).sum(0) for h in range(c["hkv"])])
                                       for b in range(c["batch"])])}
    if c["kind"] == "prompt":
        q, k, v = ((x.transpose(0, 1) if c["order"] == "tokens" else x) for x in (s["q"], s["k"], s["v"]))  # [head][token][d]
        out, lse = torch.zeros(q.shape, dtype=torch.float64, device=q.device), torch.zeros(q.shape[:2], dtype=torch.float64, device=q.device)
        at = 0
        for n in s["lens"]:
            seen = torch.ones((n, n), dtype=torch.bool, device=q.device).tril()
            for h in range(c["hq"]):
                o, l = _attend64(q[h, at:at + n].double(), k[h // g, at:at + n].double(), v[h // g, at:at + n].double(), scale, seen)
                out[h, at:at + n], lse[h, at:at + n] = o, l
            at += n
        return {"out": out.transpose(0, 1).contiguous() if c["order"] == "tokens" else out, "lse": lse}
    # prefix: the keys of every continuation, gathered, and the step's behind them
    dev, n, length = s["q"].device, c["n"], c["length"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=dev)
    lse = torch.zeros(s["q"].shape[:3], dtype=torch.float64, device=dev)
    units = _units(c, length)
    first = min(c["init"], length)
    for b, held in enumerate(s["own_lens"]):
        for h in range(c["hkv"]):
            at = list(range(first))
            if c["topk"] > 0 and units > 0:
                for u in s["idx"][b, h].tolist():
                    at += range(c["init"] + u * c["block"], c["init"] + (u + 1) * c["block"]) if u >= 0 else ()
            at = torch.tensor(at + list(range(first + units * c["block"], length)), dtype=torch.long, device=dev)
            keys, values = (torch.cat([s[x][0, h][at], s["own_" + x][b, h, :held], s["x_" + x][b, h]]).double() for x in ("k", "v"))
            seen = torch.ones((n, len(keys)), dtype=torch.bool, device=dev).tril(diagonal=len(keys) - n)
            for i in range(g):
                out[b, h * g + i], lse[b, h * g + i] = _attend64(s["q"][b, h * g + i].double(), keys, values, scale, seen)
    return {"out": out, "lse": lse, "own_k": None, "own_v": None}
