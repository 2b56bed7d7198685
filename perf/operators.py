"""Performance cases of decoding from a paged key/value cache: the four calls of a decode step that are not linears.

A case is a dict of plain values.  `kind` names the call:

    append   per-head norm + rotary embedding of new rows, keys and values into the pages of the cache (zo_cache_append)
    attend   attention of new rows over the paged cache (zo_attention_paged)
    sample   temperature, top-k, top-p and min-p from given uniforms (zo_sample)
    embed    embedding rows of tokens, with learned positions where the model has them (zo_embed_rows)

With `own` false, `run` computes the same outputs from elementary torch operations.  Both sides work on the same tensors:
a pool of pages [page][kv head][slot][head dim] for keys and one for values, a page table [sequence][page], the number of
positions of every sequence once this call's rows are in, and packed rows whose bounds are `cu`.
"""
import math
import random

import numpy as np
import torch

own = False

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


# ---- the cases ------------------------------------------------------------------------------------------------------

def listed():
    return [
        # one new token for each of 16 co-served sequences of a Qwen3-8B layer (q/k norm, rotary): what a decode step does
        dict(name="append_step", kind="append", dtype="bf16", heads=32, kv=8, dh=128, page=16, seqs=16, lo=1, hi=1,
             past=512, norm=True, theta=1e6, lens=1),
        # the prompts of a ragged batch of 32 probe pairs entering an empty cache
        dict(name="append_prompts", kind="append", dtype="bf16", heads=32, kv=8, dh=128, page=64, seqs=64, lo=16, hi=512,
             past=0, norm=True, theta=1e6, lens=2),
        # the fp32 path: prompts of a small model without q/k norm behind a cached prefix
        dict(name="append_f32", kind="append", dtype="f32", heads=8, kv=4, dh=64, page=16, seqs=24, lo=16, hi=48,
             past=100, norm=False, theta=1e4, lens=3),
        # a small fp32 model answering a few short prompts: the smallest call
        dict(name="attend_f32_small", kind="attend", dtype="f32", heads=8, kv=4, dh=64, page=16, seqs=6, rows=1,
             lo=16, hi=300, lens=4),
        # rollouts: 32 probe pairs and 16 foreground sequences of a Qwen3-8B layer, a prompt and what was answered so far
        dict(name="attend_rollouts", kind="attend", dtype="bf16", heads=32, kv=8, dh=128, page=16, seqs=80, rows=1,
             lo=64, hi=1024, lens=5),
        # OPT-13B (40 heads of their own) at its full context of 2048 tokens
        dict(name="attend_documents", kind="attend", dtype="bf16", heads=40, kv=40, dh=128, page=64, seqs=32, rows=1,
             lo=2048, hi=2048, lens=6),
        # one probe pair over a long document: few rows, a long cache, the largest call
        dict(name="attend_long_pair", kind="attend", dtype="bf16", heads=32, kv=8, dh=128, page=64, seqs=2, rows=1,
             lo=131072, hi=131072, lens=7),
        # the answers of four short prompts, OPT's vocabulary, bf16 logits, top-k and temperature
        dict(name="sample_few", kind="sample", dtype="bf16", rows=4, vocab=50272, mode="topk", std=2.5, banned=0.0),
        # a decode step of 64 rollouts over Qwen3's vocabulary, every request with settings of its own
        dict(name="sample_mixed", kind="sample", dtype="f32", rows=64, vocab=151936, mode="mixed", std=2.5, banned=0.02),
        # nucleus sampling of a large group of rollouts
        dict(name="sample_nucleus", kind="sample", dtype="f32", rows=256, vocab=151936, mode="topp", std=2.5, banned=0.0),
        # the next rows of 64 rollouts, positions advanced
        dict(name="embed_step", kind="embed", dtype="bf16", rows=64, vocab=151936, d=4096, positions=0),
        # all tokens of a batch of prompts of a model with learned positions
        dict(name="embed_prompts", kind="embed", dtype="bf16", rows=16384, vocab=50272, d=5120, positions=2050),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    top = max(work(c)["bytes"] for c in listed())
    while True:
        case = _draw(rng)
        if work(case)["bytes"] <= 0.9 * top:
            return case


def _draw(rng):
    kind = rng.choice(["append", "append", "attend", "attend", "attend", "sample", "sample", "sample", "embed"])
    dtype = "bf16" if rng.random() < 0.7 else "f32"
    c = dict(kind=kind, dtype=dtype)
    if kind in ("append", "attend"):
        heads, kv = rng.choice([(32, 8), (40, 40), (8, 4), (16, 2), (12, 1), (32, 1), (5, 5)])
        dh = rng.choice([128, 128, 128, 64, 256] if dtype == "bf16" else [128, 64, 80, 256, 32])
        c.update(heads=heads, kv=kv, dh=dh, page=rng.choice([16, 16, 32, 64, 128, 256]), lens=rng.randrange(1 << 30))
    if kind == "append":
        hi = rng.choice([1, 1, _log(rng, 2, 600)])
        c.update(seqs=_log(rng, 1, 128), hi=hi, lo=max(1, hi // rng.choice([1, 2, 16])), past=rng.choice([0, _log(rng, 1, 3000)]),
                 norm=rng.random() < 0.5, theta=rng.choice([0.0, 1e4, 1e6]))
    elif kind == "attend":
        hi = _log(rng, 1, 30000)
        c.update(seqs=max(1, _log(rng, 1, 256) * 2000 // (2000 + hi)), rows=rng.choice([1, 1, 1, 1, 3]), hi=hi,
                 lo=max(1, hi // rng.choice([1, 2, 8, 64])))
    elif kind == "sample":
        c.update(rows=_log(rng, 1, 256), vocab=rng.choice([50272, 151936, 32000, _log(rng, 300, 150000)]),
                 mode=rng.choice(["greedy", "plain", "topk", "topp", "minp", "mixed", "mixed"]),
                 std=rng.choice([0.5, 1.5, 2.5, 4.0]), banned=rng.choice([0.0, 0.0, 0.05, 0.9]))
    else:
        c.update(rows=_log(rng, 1, 16384), vocab=rng.choice([50272, 151936, 32000]), d=8 * _log(rng, 16, 700),
                 positions=rng.choice([0, 0, 2050]))
    return c


# ---- inputs ---------------------------------------------------------------------------------------------------------

def _lengths(case):
    """(rows of every sequence, positions of every sequence once they are in): part of the case, not of the seed."""
    rnd = random.Random(case["lens"])
    if case["kind"] == "append":
        rows = [rnd.randint(case["lo"], case["hi"]) for _ in range(case["seqs"])]
        return rows, [r + (rnd.randint(case["past"] // 2, case["past"]) if case["past"] else 0) for r in rows]
    kv = [max(case["rows"], rnd.randint(case["lo"], case["hi"])) for _ in range(case["seqs"])]
    return [case["rows"]] * case["seqs"], kv


class _Source:
    """Seeded random tensors on the GPU."""

    def __init__(self, seed):
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(int(seed))

    def normal(self, shape, std=1.0, dtype=torch.float32):
        return torch.randn(shape, device="cuda", dtype=dtype, generator=self.g).mul_(std)

    def uniform(self, n, lo=0.0, hi=1.0):
        return torch.rand(n, device="cuda", generator=self.g) * (hi - lo) + lo

    def whole(self, n, lo, hi):
        return torch.randint(lo, hi, (n,), device="cuda", generator=self.g).to(torch.int32)


def _cache(case, s, st):
    """Pools, a page table whose pages lie anywhere in the pools, lengths and row bounds."""
    rows, kv = _lengths(case)
    P = case["page"]
    st["max_pages"] = max(-(-n // P) for n in kv)
    n_pages = st["n_pages"] = sum(-(-n // P) for n in kv) + 3
    shape = (n_pages, case["kv"], P, case["dh"])
    st["Kp"], st["Vp"] = s.normal(shape, 1.0, DT[case["dtype"]]), s.normal(shape, 1.0, DT[case["dtype"]])
    perm = torch.randperm(n_pages, device="cuda", generator=s.g).to(torch.int32)
    used = torch.tensor([-(-n // P) for n in kv], device="cuda")
    slot = torch.arange(st["max_pages"], device="cuda")[None, :]
    first = (torch.cumsum(used, 0) - used)[:, None]
    st["table"] = torch.where(slot < used[:, None], perm[(first + slot).clamp(max=n_pages - 1)], torch.full_like(perm[:1], -1)).contiguous()
    st["kv_len"] = torch.tensor(kv, device="cuda", dtype=torch.int32)
    cu = np.zeros(len(rows) + 1, np.int32)
    cu[1:] = np.cumsum(rows)
    st["host_cu"], st["T"], st["S"], st["longest"] = cu, int(cu[-1]), len(rows), max(kv)
    st["cu"] = torch.from_numpy(cu).cuda()


def prepare(case, seed):
    s, dt, kind = _Source(seed), DT[case["dtype"]], case["kind"]
    st = {"case": case}
    if kind in ("append", "attend"):
        _cache(case, s, st)
        H, G, dh = case["heads"], case["kv"], case["dh"]
    if kind == "append":
        st["qkv"] = s.normal((st["T"], (H + 2 * G) * dh), 1.0, dt)
        st["gq"] = 1 + s.normal((dh,), 0.1) if case["norm"] else None
        st["gk"] = 1 + s.normal((dh,), 0.1) if case["norm"] else None
    elif kind == "attend":
        st["Q"] = s.normal((st["T"], H * dh), 1.0, dt)
    elif kind == "sample":
        T, V, mode = case["rows"], case["vocab"], case["mode"]
        z = s.normal((T, V), case["std"])
        if case["banned"]:   # tokens that a request does not allow
            z.masked_fill_(torch.rand((T, V), device="cuda", generator=s.g) < case["banned"], -math.inf)
        st["logits"] = z.to(dt)
        st["temperature"], st["u"] = s.uniform(T, 0.5, 1.2), s.uniform(T)
        st["top_k"], st["top_p"], st["min_p"] = s.whole(T, 1, 200), s.uniform(T, 0.5, 0.99), s.uniform(T, 0.0, 0.2)
        if mode == "mixed":   # each filter off for some rows, some rows greedy
            st["temperature"][s.uniform(T) < 0.1] = 0.0
            st["top_k"][s.uniform(T) < 0.5] = 0
            st["top_p"][s.uniform(T) < 0.3] = 1.0
            st["min_p"][s.uniform(T) < 0.5] = 0.0
        else:
            st["top_k"] = st["top_k"] if mode == "topk" else None
            st["top_p"] = st["top_p"] if mode == "topp" else None
            st["min_p"] = st["min_p"] if mode == "minp" else None
            if mode == "greedy":
                st["temperature"].zero_()
    else:
        T, V, d = case["rows"], case["vocab"], case["d"]
        st["E"] = s.normal((V, d), 0.02, dt)
        st["Epos"] = s.normal((case["positions"], d), 0.02, dt) if case["positions"] else None
        st["tokens"] = s.whole(T, 0, V)
        st["pos"] = s.whole(T, 0, case["positions"] or 4096)
    return st


# ---- one pass -------------------------------------------------------------------------------------------------------

def run(st):
    return (_own if own else _plain)[st["case"]["kind"]](st)


def _rows_at(st):
    """Sequence and position of every packed row."""
    t = torch.arange(st["T"], device="cuda")
    cu = st["cu"].long()
    seq = torch.searchsorted(cu[1:].contiguous(), t, right=True)
    return seq, st["kv_len"].long()[seq] - (cu[seq + 1] - t)


def _plain_append(st):
    c = st["case"]
    H, G, dh, T, P = c["heads"], c["kv"], c["dh"], st["T"], c["page"]
    seq, pos = _rows_at(st)
    x = st["qkv"].float().view(T, H + 2 * G, dh)
    q, k, v = x[:, :H], x[:, H:H + G], st["qkv"].view(T, H + 2 * G, dh)[:, H + G:]
    if st["gq"] is not None:
        q = q / torch.sqrt((q * q).mean(-1, keepdim=True) + 1e-6) * st["gq"]
        k = k / torch.sqrt((k * k).mean(-1, keepdim=True) + 1e-6) * st["gk"]
    if c["theta"] > 0:
        i = torch.arange(dh // 2, device="cuda", dtype=torch.float64)
        angle = pos.double()[:, None] * torch.exp(-2.0 * i / dh * math.log(c["theta"]))
        cs, sn = angle.cos().float()[:, None], angle.sin().float()[:, None]
        turn = lambda y: torch.cat([y[..., :dh // 2] * cs - y[..., dh // 2:] * sn, y[..., dh // 2:] * cs + y[..., :dh // 2] * sn], -1)
        q, k = turn(q), turn(k)
    page = st["table"][seq, pos // P].long()
    st["Kp"][page, :, pos % P] = k.to(st["Kp"].dtype)
    st["Vp"][page, :, pos % P] = v
    return {"Q": q.reshape(T, H * dh).to(st["qkv"].dtype), "K": st["Kp"], "V": st["Vp"]}


def _plain_attend(st):
    c = st["case"]
    H, G, dh, T, P = c["heads"], c["kv"], c["dh"], st["T"], c["page"]
    seq, pos = _rows_at(st)
    page = st["table"][seq].clamp(min=0).long()                       # [T, pages]
    n = page.shape[1] * P
    k = st["Kp"][page].transpose(1, 2).reshape(T, G, n, dh).float()   # [T, G, n, dh]
    q = st["Q"].float().view(T, G, H // G, dh)
    z = torch.matmul(q, k.transpose(2, 3).contiguous()) * dh ** -0.5
    del k
    z = z.masked_fill(torch.arange(n, device="cuda")[None, None, None, :] > pos[:, None, None, None], -math.inf)
    p = torch.exp(z - z.amax(-1, keepdim=True))
    v = st["Vp"][page].transpose(1, 2).reshape(T, G, n, dh).float()
    o = torch.matmul(p, v) / p.sum(-1, keepdim=True)
    return {"O": o.reshape(T, H * dh).to(st["Q"].dtype)}


def _plain_sample(st):
    z = st["logits"].double()
    T, V = z.shape
    t = st["temperature"].double()[:, None]
    greedy = ~(t > 0)
    order, index = torch.sort(z, dim=1, descending=True, stable=True)   # equal logits: the lowest index first
    w = torch.exp((order - order[:, :1]) / torch.where(greedy, torch.ones_like(t), t))
    place = torch.arange(V, device="cuda")[None, :]
    n = (order > -math.inf).sum(1, keepdim=True)
    if st["top_k"] is not None:
        k = st["top_k"].long()[:, None]
        n = torch.where(k > 0, torch.minimum(n, k), n)
    if st["top_p"] is not None:
        p = st["top_p"].double()[:, None]
        mass = torch.cumsum(torch.where(place < n, w, torch.zeros_like(w)), 1)
        n = torch.where(p < 1, torch.minimum(n, (mass - w < p * mass[:, -1:]).sum(1, keepdim=True)), n)
    if st["min_p"] is not None:
        m = st["min_p"].double()[:, None]
        n = torch.where(m > 0, torch.minimum(n, (w >= m).sum(1, keepdim=True)), n)
    n = torch.where(greedy, torch.ones_like(n), n.clamp(min=1))
    kept = torch.zeros_like(w).scatter_(1, index, torch.where(place < n, w, torch.zeros_like(w)))   # by token
    cum = torch.cumsum(kept, 1)
    total = cum[:, -1:]
    token = torch.searchsorted(cum, st["u"].double()[:, None] * total, right=True).clamp(max=V - 1)
    return {"token": token[:, 0].to(torch.int32), "prob": (kept.gather(1, token) / total)[:, 0].float(),
            "kept": n[:, 0].to(torch.int32)}


def _plain_embed(st):
    x = st["E"][st["tokens"].long()]
    if st["Epos"] is not None:
        x = (x.float() + st["Epos"][st["pos"].long()].float()).to(x.dtype)
    return {"X": x, "pos": st["pos"] + 1}


_plain = {"append": _plain_append, "attend": _plain_attend, "sample": _plain_sample, "embed": _plain_embed}


def _kit(st):
    """What a program makes once and keeps for its calls: the batch and cache structs, outputs, workspace."""
    if "kit" in st:
        return st["kit"]
    from paper_2605_28760_amd import binding as zb
    c, kit = st["case"], {"zb": zb}
    empty = lambda shape, dt: torch.empty(shape, device="cuda", dtype=dt)
    kit["dt"] = zb.ZO_BF16 if c["dtype"] == "bf16" else zb.ZO_F32
    if c["kind"] in ("append", "attend"):
        none = torch.full((st["S"],), -1, device="cuda", dtype=torch.int32)
        kit["batch"] = zb.make_batch(st["T"], st["cu"], none, None, None, None, st["host_cu"], n_seqs=st["S"], n_cands=0,
                                     n_dirs=0)
        kit["cache"] = zb.make_cache(st["Kp"], st["Vp"], kit["dt"], st["table"], st["kv_len"])
        kit["out"] = empty((st["T"], c["heads"] * c["dh"]), DT[c["dtype"]])
    ws = 0
    if c["kind"] == "attend":
        ws = zb.zo_attention_paged_workspace_bytes(st["T"], c["heads"], c["dh"], st["max_pages"] * c["page"], kit["dt"])
    elif c["kind"] == "sample":
        T = c["rows"]
        ws = zb.zo_sample_workspace_bytes(T, c["vocab"], kit["dt"])
        kit["token"], kit["prob"], kit["kept"] = empty(T, torch.int32), empty(T, torch.float32), empty(T, torch.int32)
    elif c["kind"] == "embed":
        kit["X"], kit["pos"] = empty((c["rows"], c["d"]), DT[c["dtype"]]), empty(c["rows"], torch.int32)
    kit["ws_bytes"], kit["ws"] = ws, empty(max(ws, 256), torch.uint8)
    st["kit"] = kit
    return kit


def _own_append(st):
    c, k = st["case"], _kit(st)
    nq, nkv = c["heads"] * c["dh"], c["kv"] * c["dh"]
    x, ld = st["qkv"], st["qkv"].stride(0)
    k["zb"].zo_cache_append(k["batch"], x, ld, x[:, nq:], ld, x[:, nq + nkv:], ld, c["heads"], st["gq"], st["gk"], 1e-6,
                            c["theta"], k["cache"], k["out"], nq)
    return {"Q": k["out"], "K": st["Kp"], "V": st["Vp"]}


def _own_attend(st):
    c, k = st["case"], _kit(st)
    n = c["heads"] * c["dh"]
    k["zb"].zo_attention_paged(k["batch"], st["Q"], n, c["heads"], c["dh"] ** -0.5, k["cache"], k["out"], n, k["ws"],
                               k["ws_bytes"])
    return {"O": k["out"]}


def _own_sample(st):
    c, k = st["case"], _kit(st)
    k["zb"].zo_sample(st["logits"], c["vocab"], c["rows"], c["vocab"], k["dt"], st["temperature"], st["top_k"], st["top_p"],
                      st["min_p"], st["u"], k["token"], k["prob"], k["kept"], k["ws"], k["ws_bytes"])
    return {"token": k["token"], "prob": k["prob"], "kept": k["kept"]}


def _own_embed(st):
    c, k = st["case"], _kit(st)
    k["zb"].zo_embed_rows(st["tokens"], st["pos"], c["rows"], st["E"], c["d"], c["vocab"], st["Epos"], c["d"],
                          c["positions"], c["d"], k["dt"], k["X"], c["d"], k["pos"])
    return {"X": k["X"], "pos": k["pos"]}


_own = {"append": _own_append, "attend": _own_attend, "sample": _own_sample, "embed": _own_embed}


# ---- what a pass cannot do without ----------------------------------------------------------------------------------

def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    if case["kind"] == "append":
        T = sum(_lengths(case)[0])
        wide = T * (case["heads"] + 2 * case["kv"]) * case["dh"]
        return {"bytes": 2 * wide * size + 4 * T, "flops": 8 * wide}
    if case["kind"] == "attend":
        rows, kv = _lengths(case)
        r, H, dh = case["rows"], case["heads"], case["dh"]
        pages = sum(-(-n // case["page"]) for n in kv)
        seen = sum(r * n - r * (r - 1) // 2 for n in kv)
        return {"bytes": 2 * sum(kv) * case["kv"] * dh * size + 2 * sum(rows) * H * dh * size + 4 * pages,
                "flops": 4 * seen * H * dh}
    if case["kind"] == "sample":
        return {"bytes": case["rows"] * (case["vocab"] * size + 28), "flops": 4 * case["rows"] * case["vocab"]}
    T, d = case["rows"], case["d"]
    return {"bytes": 2 * T * d * size + min(T, case["positions"]) * d * size + 12 * T, "flops": T * d if case["positions"] else 0}


# ---- the definition in 64 bits --------------------------------------------------------------------------------------

def exact(case, seed):
    st = prepare(case, seed)
    return {"append": _exact_append, "attend": _exact_attend, "sample": _exact_sample, "embed": _exact_embed}[case["kind"]](case, st)


def _places(case, st, i):
    """Rows of sequence i, their positions, and the page of each position that the sequence has."""
    a, b = int(st["host_cu"][i]), int(st["host_cu"][i + 1])
    n = int(st["kv_len"][i])
    at = np.arange(n)
    pages = st["table"][i].cpu().numpy()
    return a, b, np.arange(n - (b - a), n), pages[at // case["page"]].astype(np.int64), at % case["page"]


def _exact_append(case, st):
    H, G, dh = case["heads"], case["kv"], case["dh"]
    x = st["qkv"].double().cpu().numpy().reshape(st["T"], H + 2 * G, dh)
    K, V = st["Kp"].double(), st["Vp"].double()
    freq = np.array([case["theta"] ** (-2.0 * j / dh) for j in range(dh // 2)]) if case["theta"] > 0 else np.zeros(dh // 2)

    def turned(rows, gain, pos):
        if gain is not None:
            rows = rows * gain.double().cpu().numpy() / np.sqrt(np.square(rows).mean(-1, keepdims=True) + 1e-6)
        z = (rows[..., :dh // 2] + 1j * rows[..., dh // 2:]) * np.exp(1j * np.multiply.outer(pos.astype(np.float64), freq))[:, None]
        return np.concatenate([z.real, z.imag], -1)

    q = np.empty((st["T"], H, dh))
    for i in range(st["S"]):
        a, b, pos, pages, slots = _places(case, st, i)
        q[a:b] = turned(x[a:b, :H], st["gq"], pos)
        k = torch.from_numpy(turned(x[a:b, H:H + G], st["gk"], pos)).cuda()
        pg, sl = torch.from_numpy(pages[pos]).cuda(), torch.from_numpy(slots[pos]).cuda()
        K[pg, :, sl] = k
        V[pg, :, sl] = torch.from_numpy(x[a:b, H + G:]).cuda()
    return {"Q": torch.from_numpy(q.reshape(st["T"], H * dh)), "K": K, "V": V}


def _exact_attend(case, st):
    H, G, dh = case["heads"], case["kv"], case["dh"]
    out = torch.empty((st["T"], H, dh), dtype=torch.float64, device="cuda")
    for i in range(st["S"]):
        a, b, pos, pages, slots = _places(case, st, i)
        pg, sl = torch.from_numpy(pages).cuda(), torch.from_numpy(slots).cuda()
        for g in range(G):
            k, v = st["Kp"][pg, g, sl].double(), st["Vp"][pg, g, sl].double()
            for t in range(a, b):
                n = int(pos[t - a]) + 1
                q = st["Q"][t].double().view(H, dh)[g * (H // G):(g + 1) * (H // G)]
                out[t, g * (H // G):(g + 1) * (H // G)] = torch.softmax(q @ k[:n].T / math.sqrt(dh), -1) @ v[:n]
    return {"O": out.reshape(st["T"], H * dh)}


def _exact_sample(case, st):
    T, V = case["rows"], case["vocab"]
    z = st["logits"].double().cpu().numpy()
    get = lambda name, off: np.full(T, off) if st[name] is None else st[name].double().cpu().numpy()
    temp, k, p, m, u = get("temperature", 1.0), get("top_k", 0), get("top_p", 1.0), get("min_p", 0.0), get("u", 0.0)
    token, prob, kept = np.zeros(T, np.int32), np.zeros(T), np.zeros(T, np.int32)
    for t in range(T):
        if temp[t] <= 0:
            token[t], prob[t], kept[t] = int(np.argmax(z[t])), 1.0, 1
            continue
        order = np.argsort(-z[t], kind="stable")
        order = order[:int((z[t] > -np.inf).sum())]
        w = np.exp((z[t][order] - z[t][order[0]]) / temp[t])
        if k[t] > 0:
            order, w = order[:int(k[t])], w[:int(k[t])]
        n = len(w)
        if p[t] < 1:
            n = min(n, 1 + int(np.searchsorted(np.cumsum(w)[:-1], p[t] * w.sum(), side="left")))
        if m[t] > 0:
            n = min(n, int((w >= m[t]).sum()))
        n = max(n, 1)
        mine = np.argsort(order[:n])
        cum = np.cumsum(w[:n][mine])
        at = min(int(np.searchsorted(cum, u[t] * cum[-1], side="right")), n - 1)
        token[t], prob[t], kept[t] = order[:n][mine[at]], w[:n][mine[at]] / cum[-1], n
    return {"token": torch.from_numpy(token), "prob": torch.from_numpy(prob), "kept": torch.from_numpy(kept)}


def _exact_embed(case, st):
    tok, pos = st["tokens"].cpu().numpy(), st["pos"].cpu().numpy()
    x = st["E"].cpu().double().numpy()[tok]
    if st["Epos"] is not None:
        x = x + st["Epos"].cpu().double().numpy()[pos]
    return {"X": torch.from_numpy(x), "pos": torch.from_numpy(pos + 1)}
