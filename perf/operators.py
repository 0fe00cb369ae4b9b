"""The operators around a served model's key-value cache, as cases that can be timed and compared.

A case is a dict of plain values; `op` names the operator:

  "window"  causal attention with a sliding window of `window` positions and the first `sinks` ones always visible; `Lq` <= L
            queries, the last positions of the context
  "paged"   attention of one new token per sequence over a paged key-value cache (window 0: the whole context), with
            `accumulate` also adding every key's softmax weights to the cache's own sums
  "write"   the last `T` positions of every sequence into the pages, with their starting weights where `weighted`
  "weights" the softmax weights that every key gets from the last `Lq` queries, summed over the queries and a group's heads
  "evict"   a cache's positions by accumulated weight, down to `keep` with the first `sinks` and the last `recent` among them,
            into other pages

  batch, L, Hq, Hkv, d, dtype               as in include/rr_attn.h; L of a cache case is its longest sequence
  shortest                                  cache cases: lengths of the batch lie between this and L
  page                                      positions to a page
"""
import math

import torch

own = False
DEVICE = "cuda:0"


def _case(name, op, **more):
    c = dict(op=op, batch=1, Hq=32, Hkv=8, d=128, dtype="bf16", **more)
    return dict(name=name, **c) if name else c


def listed():
    return [
        # a local layer's share of a 32K prompt, 32 / 8 heads: the largest
        _case("window_32k", "window", L=32768, Lq=32768, window=4096, sinks=4),
        # the same operator in fp32 at a width and length that are multiples of nothing: a reference run, the smallest prompt
        dict(_case("window_ragged_f32", "window", L=1511, Lq=1511, window=200, sinks=5), Hq=8, Hkv=2, d=80, dtype="f32"),
        # one decoded token of a local layer against a contiguous 64K context
        _case("window_step_64k", "window", L=65536, Lq=1, window=8192, sinks=128),
        # one token against 128K in pages
        _case("paged_128k", "paged", L=131072, shortest=131072, page=64, window=0, sinks=0, accumulate=False),
        # a serving batch of uneven lengths whose cache is evicted from by weight
        dict(_case("paged_batch64_weights", "paged", L=16384, shortest=200, page=16, window=0, sinks=0, accumulate=True), batch=64),
        # a few short sequences in fp32: launches and host work
        dict(_case("paged_small_f32", "paged", L=300, shortest=1, page=16, window=128, sinks=4, accumulate=False), batch=4, Hq=8,
             Hkv=2, d=64, dtype="f32"),
        # the new token of every sequence of a batch
        dict(_case("write_step64", "write", L=8192, shortest=100, T=1, page=16, weighted=False), batch=64),
        # a prompt into its pages, with the weights it starts with
        _case("write_prompt_16k", "write", L=16384, shortest=16384, T=16384, page=64, weighted=True),
        # weights of a 64K prompt's keys as its last 64 queries see them
        _case("weights_last64_64k", "weights", L=65536, Lq=64),
        # the same from every query of an 8K prompt, 28 / 4 heads
        dict(_case("weights_prompt_8k", "weights", L=8192, Lq=8192), Hq=28, Hkv=4),
        # a batch that has outgrown its 2048 positions by a few pages
        dict(_case("evict_batch16", "evict", L=2304, shortest=2049, page=16, keep=2048, sinks=4, recent=256), batch=16),
        # a long context halved
        _case("evict_128k", "evict", L=131072, shortest=131072, page=64, keep=65536, sinks=4, recent=4096),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["window", "window", "paged", "paged", "paged", "write", "weights", "evict"])
    heads = rng.choice([(32, 8, 128), (32, 8, 128), (28, 4, 128), (64, 8, 128), (8, 2, 128), (16, 4, 64), (6, 3, 80), (8, 8, 40)])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    page = rng.choice([16, 16, 32, 48, 64, 128])
    common = dict(Hq=heads[0], Hkv=heads[1], d=heads[2], dtype=dtype)
    plain = dtype == "f32" or heads[2] != 128
    if op == "window":
        L = _log(rng, 64, 6000 if plain else 24576)
        Lq = rng.choice([L, L, L, _log(rng, 1, L)])
        return dict(_case(None, op, L=L, Lq=Lq, window=_log(rng, 16, 4096), sinks=rng.choice([0, 1, 4, 33, 128, 200])), **common)
    if op == "weights":
        L = _log(rng, 64, 3000 if plain else 8192)
        return dict(_case(None, op, L=L, Lq=rng.choice([L, _log(rng, 1, min(L, 512))])), **common)
    batch = rng.choice([1, 1, 2, 5, 16, 40])
    L = _log(rng, 16, 131072 // batch)
    shortest = rng.choice([1, max(1, L // 20), L])
    if op == "paged":
        window = rng.choice([0, 0, 0, _log(rng, 16, 4096)])
        return dict(_case(None, op, L=L, shortest=shortest, page=page, window=window, sinks=rng.choice([0, 4, 100]) if window else 0,
                          accumulate=rng.choice([False, True])), **common, batch=batch)
    if op == "write":
        T = rng.choice([1, _log(rng, 1, L)])
        return dict(_case(None, op, L=L, shortest=max(T, shortest), T=T, page=page, weighted=rng.choice([False, True])), **common,
                    batch=batch)
    keep = max(8, int(L * rng.uniform(0.1, 0.98)))
    return dict(_case(None, op, L=L, shortest=shortest, page=page, keep=keep, sinks=rng.choice([0, min(4, keep // 4)]),
                      recent=int(keep * rng.uniform(0.0, 0.5))), **common, batch=batch)


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def prepare(case, seed):
    b, L, Hq, Hkv, d, op = (case[k] for k in ("batch", "L", "Hq", "Hkv", "d", "op"))
    dt = _dtype(case)
    g = torch.Generator(device=DEVICE).manual_seed(int(seed))

    def normal(*shape, by=1.0):
        return (torch.randn(*shape, generator=g, device=DEVICE) * by).to(dt)

    def log_sums(Q, K):
        """Log of the causal softmax's denominators, one KV head's queries at a time."""
        Lq, G = case["Lq"], Hq // Hkv
        hidden = torch.arange(L, device=DEVICE)[None] > torch.arange(L - Lq, L, device=DEVICE)[:, None]
        out = torch.empty(b, Hq, Lq, dtype=torch.float32, device=DEVICE)
        for i in range(b):
            for kv in range(Hkv):
                heads = slice(kv * G, kv * G + G)
                x = (Q[i, heads].float().reshape(-1, d) @ K[i, kv].float().T).reshape(G, Lq, L) / math.sqrt(d)
                out[i, heads] = x.masked_fill(hidden, -math.inf).logsumexp(-1)
        return out

    s = dict(case=case)
    if op in ("window", "weights"):
        # scores of deviation 2: a few keys in a hundred carry most of a row, as trained heads have it
        s["Q"], s["K"] = normal(b, Hq, case["Lq"], d, by=2.0), normal(b, Hkv, L, d)
        if op == "window":
            s["V"] = normal(b, Hkv, L, d)
            s["lse"] = torch.empty(b, Hq, case["Lq"], dtype=torch.float32, device=DEVICE)
        else:
            # what the attention before it has written beside its outputs
            s["lse"] = log_sums(s["Q"], s["K"])
        return s
    page = case["page"]
    width = -(-L // page)
    pages = b * width + 3
    at = torch.randint(case["shortest"], L + 1, (b,), generator=g, device=DEVICE)
    at[0] = L
    s["length"] = at.int()
    order = torch.randperm(pages, generator=g, device=DEVICE)[: b * width].reshape(b, width).int()
    # a page that a sequence does not reach has no entry
    s["table"] = torch.where(torch.arange(width, device=DEVICE)[None] * page < s["length"][:, None], order, -1).contiguous()
    if op != "evict":
        s["K"], s["V"] = normal(pages, Hkv, page, d), normal(pages, Hkv, page, d)
    # accumulated weights: a few heavy positions and a long tail
    s["weight"] = torch.rand(pages, Hkv, page, generator=g, device=DEVICE).pow(8) * 50.0
    if op == "paged":
        s["Q"] = normal(b, Hq, 1, d, by=2.0)
        s["lse"] = torch.empty(b, Hq, 1, dtype=torch.float32, device=DEVICE)
    elif op == "write":
        s["newK"], s["newV"] = normal(b, Hkv, case["T"], d), normal(b, Hkv, case["T"], d)
        s["count"] = torch.randint(max(1, case["T"] // 2), case["T"] + 1, (b,), generator=g, device=DEVICE).int()
        s["first"] = torch.rand(b, Hkv, case["T"], generator=g, device=DEVICE) if case["weighted"] else None
    else:
        kept = -(-case["keep"] // page)
        s["K"], s["V"] = normal(pages + b * kept, Hkv, page, d), normal(pages + b * kept, Hkv, page, d)
        s["weight"] = torch.cat([s["weight"], torch.zeros(b * kept, Hkv, page, device=DEVICE)])
        s["to"] = (pages + torch.randperm(b * kept, generator=g, device=DEVICE)).reshape(b, kept).int()
        s["to_length"] = torch.zeros(b, dtype=torch.int32, device=DEVICE)
        s["kept"] = torch.empty(b, Hkv, case["keep"], dtype=torch.int32, device=DEVICE)
    return s


def run(s):
    case = s["case"]
    return _kernels(s, case) if own else _PLAIN[case["op"]](s, case)


def _kernels(s, case):
    import paper_2602_05853_amd as rr
    op = case["op"]
    if op == "window":
        if "ws" not in s:
            n = rr.rr_window_workspace_bytes(s["Q"], s["K"], case["window"], case["sinks"])
            s["ws"] = torch.empty(n, dtype=torch.uint8, device=DEVICE) if n else None
        O = rr.rr_window_attn(s["Q"], s["K"], s["V"], case["window"], case["sinks"], lse=s["lse"], workspace=s["ws"])
        return {"O": O, "lse": s["lse"]}
    if op == "weights":
        return {"weight": rr.rr_key_weights(s["Q"], s["K"], s["lse"])}
    if "cache" not in s:
        s["cache"] = rr.PagedCache(s["K"], s["V"], s["table"], s["length"], s["weight"])
    cache = s["cache"]
    if op == "paged":
        if "ws" not in s:
            n = rr.rr_paged_workspace_bytes(s["Q"], cache, case["window"], case["sinks"], accumulate=case["accumulate"])
            s["ws"] = torch.empty(n, dtype=torch.uint8, device=DEVICE)
        O = rr.rr_paged_attn(s["Q"], cache, case["window"], case["sinks"], accumulate=case["accumulate"], lse=s["lse"],
                             workspace=s["ws"])
        return {"O": O, "lse": s["lse"], **({"weight": s["weight"]} if case["accumulate"] else {})}
    if op == "write":
        rr.rr_paged_write(cache, s["newK"], s["newV"], count=s["count"], weight=s["first"])
        return {"K": s["K"], "V": s["V"], "weight": s["weight"]}
    rr.rr_cache_evict(cache, s["to"], case["keep"], case["sinks"], case["recent"], length=s["to_length"], kept=s["kept"])
    return {"kept": s["kept"], "length": s["to_length"], "K": s["K"], "V": s["V"], "weight": s["weight"]}


# ---- plain forms: 32 bits, elementary operations ----

def _plain_window(s, case):
    """Queries in bands of c: a band meets the c + W - 1 keys that any of its windows reaches, and the sinks apart."""
    Q, K, V = s["Q"].float(), s["K"].float(), s["V"].float()
    (b, Hq, Lq, d), (Hkv, L) = Q.shape, K.shape[1:3]
    G, W = Hq // Hkv, min(case["window"], L)
    c = max(1, min(Lq, max(64, W // 4)))
    n = -(-Lq // c)
    q0, span = L - Lq, c + W - 1
    q = torch.cat([Q, Q.new_zeros(b, Hq, n * c - Lq, d)], 2).reshape(b, Hkv, G, n, c, d).transpose(2, 3).reshape(b, Hkv, n, G * c, d)
    # key t of band m is position q0 + m c - (W - 1) + t
    lead, tail = q0 - (W - 1), q0 + n * c - L
    band = [torch.cat([x.new_zeros(b, Hkv, max(0, -lead), d), x[:, :, max(0, lead):], x.new_zeros(b, Hkv, tail, d)], 2)
            .unfold(2, span, c) for x in (K, V)]                                   # [b, Hkv, n, d, span]
    i = q0 + torch.arange(n * c, device=DEVICE).reshape(n, c, 1)
    j = lead + torch.arange(n, device=DEVICE)[:, None, None] * c + torch.arange(span, device=DEVICE)
    sinks = min(case["sinks"], L)
    far = torch.arange(sinks, device=DEVICE).expand(n, c, sinks)
    seen = torch.cat([(j >= 0) & (j <= i) & (j > i - W), far <= i - W], 2)         # (a sink inside the window is in the band)
    x = torch.cat([torch.matmul(q, band[0].contiguous()),
                   torch.matmul(q, K[:, :, None, :sinks].transpose(3, 4).contiguous())], 4) / math.sqrt(d)
    x = x.reshape(b, Hkv, n, G, c, span + sinks).masked_fill(~seen[:, None], -math.inf)
    top = x.amax(-1, keepdim=True)
    x = (x - top).exp()
    total = x.sum(-1, keepdim=True)
    lse = (top + total.log()).reshape(b, Hkv, n, G, c)
    x = (x / total).reshape(b, Hkv, n, G * c, span + sinks)
    O = torch.matmul(x[..., :span], band[1].transpose(3, 4).contiguous()) + torch.matmul(x[..., span:], V[:, :, None, :sinks])
    O = O.reshape(b, Hkv, n, G, c, d).transpose(2, 3).reshape(b, Hq, n * c, d)[:, :, :Lq]
    return {"O": O.to(s["Q"].dtype).contiguous(), "lse": lse.transpose(2, 3).reshape(b, Hq, n * c)[:, :, :Lq].contiguous()}


def _slots(table, position, page):
    """Page and slot of `position` [b, n] of every sequence; positions without a page come out as page 0."""
    width = table.shape[1]
    entry = table.long().gather(1, (position // page).clamp(0, width - 1))
    return entry.clamp(min=0), position % page


def _plain_paged(s, case):
    b, Hq, Hkv, d, L, page = (case[k] for k in ("batch", "Hq", "Hkv", "d", "L", "page"))
    t = torch.arange(L, device=DEVICE).expand(b, L)
    at, slot = _slots(s["table"], t, page)
    length = s["length"].long()[:, None]
    seen = t < length
    if case["window"]:
        seen = seen & ((t >= length - case["window"]) | (t < case["sinks"]))
    K = s["K"][at, :, slot].float().permute(0, 2, 1, 3)                            # [b, Hkv, L, d]
    V = s["V"][at, :, slot].float().permute(0, 2, 1, 3)
    q = s["Q"].float().reshape(b, Hkv, Hq // Hkv, d)
    x = torch.matmul(q, K.transpose(2, 3).contiguous()) / math.sqrt(d)
    x = x.masked_fill(~seen[:, None, None], -math.inf)
    top = x.amax(-1, keepdim=True)
    x = (x - top).exp()
    total = x.sum(-1, keepdim=True)
    x = x / total
    s["lse"].copy_((top + total.log()).reshape(b, Hq, 1))
    out = {"O": torch.matmul(x, V.contiguous()).to(s["Q"].dtype).reshape(b, Hq, 1, d), "lse": s["lse"]}
    if case["accumulate"]:
        # every page belongs to one sequence; positions nobody sees add nothing
        head = torch.arange(Hkv, device=DEVICE)[None, :, None]
        s["weight"].index_put_((at[:, None], head, slot[:, None]), x.sum(2), accumulate=True)
        out["weight"] = s["weight"]
    return out


def _plain_write(s, case):
    b, Hkv, T, page = (case[k] for k in ("batch", "Hkv", "T", "page"))
    t = torch.arange(T, device=DEVICE).expand(b, T)
    count = s["count"].long()[:, None]
    at, slot = _slots(s["table"], s["length"].long()[:, None] - count + t, page)
    new = t < count
    i, j, at, slot = t.new_tensor(range(b))[:, None].expand(b, T)[new], t[new], at[new], slot[new]
    s["K"][at, :, slot] = s["newK"][i, :, j]
    s["V"][at, :, slot] = s["newV"][i, :, j]
    s["weight"][at, :, slot] = s["first"][i, :, j] if s["first"] is not None else 0.0
    return {"K": s["K"], "V": s["V"], "weight": s["weight"]}


def _plain_weights(s, case):
    Q, K = s["Q"].float(), s["K"].float()
    (b, Hq, Lq, d), (Hkv, L) = Q.shape, K.shape[1:3]
    x = torch.matmul(Q.reshape(b, Hkv, Hq // Hkv * Lq, d), K.transpose(2, 3).contiguous()) / math.sqrt(d)
    x = (x - s["lse"].reshape(b, Hkv, Hq // Hkv * Lq, 1)).exp().reshape(b, Hkv, Hq // Hkv, Lq, L)
    hidden = torch.arange(L, device=DEVICE)[None] > torch.arange(L - Lq, L, device=DEVICE)[:, None]
    return {"weight": x.masked_fill(hidden, 0.0).sum((2, 3))}


def _plain_evict(s, case):
    b, Hkv, L, page, keep = (case[k] for k in ("batch", "Hkv", "L", "page", "keep"))
    t = torch.arange(L, device=DEVICE).expand(b, L)
    at, slot = _slots(s["table"], t, page)
    length = s["length"].long()[:, None]
    w = s["weight"][at, :, slot].transpose(1, 2)                                   # [b, Hkv, L]
    kept_anyway = (t < case["sinks"]) | (t >= length - case["recent"])
    w = w.masked_fill(kept_anyway[:, None], math.inf).masked_fill((t >= length)[:, None], -math.inf)
    order = w.sort(dim=2, descending=True, stable=True).indices[:, :, :keep]
    n = length.clamp(max=keep)[:, None]                                            # [b, 1, 1]
    real = torch.arange(order.shape[2], device=DEVICE) < n
    kept = torch.where(real, order, L).sort(dim=2).values
    s["kept"].fill_(-1)
    s["kept"][:, :, : order.shape[2]] = torch.where(real, kept, -1).int()
    s["to_length"].copy_(n.reshape(b))
    i, h, r = torch.where(real.expand(b, Hkv, order.shape[2]))
    src = kept[i, h, r]
    p, q = s["table"].long()[i, src // page], s["to"].long()[i, r // page]
    for name in ("K", "V", "weight"):
        s[name][q, h, r % page] = s[name][p, h, src % page]
    return {"kept": s["kept"], "length": s["to_length"], "K": s["K"], "V": s["V"], "weight": s["weight"]}


_PLAIN = {"window": _plain_window, "paged": _plain_paged, "write": _plain_write, "weights": _plain_weights, "evict": _plain_evict}


def _pairs(case):
    """(query, key) pairs a query head has."""
    L, Lq = case["L"], case["Lq"]
    W, sinks = case.get("window", L), case.get("sinks", 0)

    def below(n):                                    # pairs of the positions before n
        near = n * (n + 1) / 2 if n <= W else W * (W + 1) / 2 + (n - W) * W
        m = max(0, n - W)                            # positions W .. n - 1 see min(sinks, i - W + 1) keys in front of their window
        k = min(m, sinks)
        return near + k * (k + 1) / 2 + (m - k) * sinks
    return below(L) - below(L - Lq)


def work(case):
    b, L, Hq, Hkv, d, op = (case[k] for k in ("batch", "L", "Hq", "Hkv", "d", "op"))
    size = 2 if case["dtype"] == "bf16" else 4
    if op in ("window", "weights"):
        Lq = case["Lq"]
        seen = L if op == "weights" else min(L, Lq - 1 + case["window"] + case["sinks"])
        rows = b * Hq * Lq
        if op == "weights":
            return {"bytes": rows * (d * size + 4) + b * Hkv * seen * (d * size + 4), "flops": 2.0 * d * b * Hq * _pairs(case)}
        return {"bytes": rows * (2 * d * size + 4) + 2 * b * Hkv * seen * d * size, "flops": 4.0 * d * b * Hq * _pairs(case)}
    mean = L if b == 1 else (L + (b - 1) * (L + case["shortest"]) / 2) / b         # lengths are uniform in their range
    if op == "paged":
        seen = min(mean, case["window"] + case["sinks"]) if case["window"] else mean
        per = 2 * d * size + (8 if case["accumulate"] else 0)
        return {"bytes": b * Hkv * seen * per + b * Hq * (2 * d * size + 4), "flops": 4.0 * d * b * Hq * seen}
    if op == "write":
        new = b * Hkv * case["T"] * 0.75
        return {"bytes": new * (4 * d * size + (8 if case["weighted"] else 4)), "flops": 0}
    n = min(mean, case["keep"])
    return {"bytes": b * Hkv * (4 * mean + n * (4 * d * size + 4 + 4)), "flops": 0}


# ---- the definitions in 64 bits ----

def exact(case, seed):
    s = prepare(case, seed)
    b, L, Hq, Hkv, d, op = (case[k] for k in ("batch", "L", "Hq", "Hkv", "d", "op"))
    G = Hq // Hkv

    def attend(q, K, V, seen):
        """Rows q [n, d] over keys K, V [m, d] where `seen` [n, m] says so: outputs, log-sum-exp, probabilities."""
        score = torch.where(seen, q.double() @ K.double().T * d ** -0.5, -math.inf)
        lse = torch.logsumexp(score, 1)
        p = torch.exp(score - lse[:, None])
        return p @ V.double(), lse, p

    if op in ("window", "weights"):
        Lq = case["Lq"]
        O, lse = torch.empty(b, Hq, Lq, d, dtype=torch.float64, device=DEVICE), torch.empty(b, Hq, Lq, dtype=torch.float64, device=DEVICE)
        weight = torch.zeros(b, Hkv, L, dtype=torch.float64, device=DEVICE)
        key = torch.arange(L, device=DEVICE)[None]
        step = 2048
        for r in range(0, Lq, step):
            e = min(Lq, r + step)
            pos = torch.arange(L - Lq + r, L - Lq + e, device=DEVICE)[:, None]
            seen = key <= pos
            if op == "window":
                seen = seen & ((pos - key < case["window"]) | (key < case["sinks"]))
            for i in range(b):
                for h in range(Hq):
                    q, K = s["Q"][i, h, r:e], s["K"][i, h // G]
                    if op == "window":
                        O[i, h, r:e], lse[i, h, r:e], _ = attend(q, K, s["V"][i, h // G], seen)
                    else:
                        p = torch.exp(q.double() @ K.double().T * d ** -0.5 - s["lse"][i, h, r:e, None].double())
                        weight[i, h // G] += torch.where(seen, p, 0.0).sum(0)
        return {"O": O, "lse": lse} if op == "window" else {"weight": weight}
    if op != "paged":
        return None                                  # moved values and whole numbers: nothing is computed
    O, lse = torch.empty(b, Hq, 1, d, dtype=torch.float64, device=DEVICE), torch.empty(b, Hq, 1, dtype=torch.float64, device=DEVICE)
    weight = s["weight"].double()
    lengths, table = s["length"].tolist(), s["table"].tolist()
    for i, n in enumerate(lengths):
        used = table[i][: -(-n // case["page"])]
        key = torch.arange(n, device=DEVICE)
        seen = torch.ones(1, n, dtype=torch.bool, device=DEVICE)
        if case["window"]:
            seen = ((n - 1 - key < case["window"]) | (key < case["sinks"]))[None]
        for kv in range(Hkv):
            K, V = (s[x][used, kv].reshape(-1, d)[:n] for x in ("K", "V"))
            heads = slice(kv * G, kv * G + G)
            O[i, heads, 0], lse[i, heads, 0], p = attend(s["Q"][i, heads, 0], K, V, seen.expand(G, n))
            if case["accumulate"]:
                add = torch.zeros(len(used) * case["page"], dtype=torch.float64, device=DEVICE)
                add[:n] = p.sum(0)
                weight[used, kv] += add.reshape(len(used), -1)
    return {"O": O, "lse": lse, **({"weight": weight} if case["accumulate"] else {})}
