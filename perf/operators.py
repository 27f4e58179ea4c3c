"""Performance cases of the cache operators: attention of drafted tokens over the cache,
accumulated attention weights, eviction by them, and the compaction of the cache.

  tree      N drafted tokens a row attend the cached context (all of it, or the selected
            blocks and the window) and their ancestors in the draft (cobs_tree_decode).
            Without a draft the N queries attend the context alone.
  weights   the attention weights that N queries give each cached token, added up over
            queries and query heads (cobs_attention_weights).
  evict     which tokens a cache keeps: the first, the last and the heaviest between
            (cobs_evict).
  compact   the kept tokens' keys, values and weights, moved together in another cache
            (cobs_compact_cache).

A program holds the cache, its page tables and its output buffers, so prepare() makes
those and run() is the one call.  Keys are a block mean plus unit noise, queries unit
normal.  Drafts are random trees; the draft's keys stand in the cache behind the context.
"""

import math

import torch

own = False


def _case(name, op, **over):
    c = dict(op=op, B=1, Hkv=8, G=4, d=128, L=64, T=32741, N=1, s=-1, w=0, kv="bf16", io="f32", draft=True,
             ragged=False, paged=False, keep=0, sinks=4, recent=64)
    c.update(over)
    if name:
        c = dict(name=name, **c)
    return c


def listed():
    return [
        # the smallest call: one short fp32 conversation, one head, a draft of five
        _case("tree_1k_fp32", "tree", Hkv=1, G=1, d=64, T=1009, N=5, kv="f32"),
        # interactive speculation on one sequence of a 32-head GQA layer, a draft of eight
        _case("tree_4k", "tree", T=4001, N=8, io="bf16"),
        # a serving batch with rows of different lengths on pages, drafts of up to 32
        _case("tree_32k_ragged_paged", "tree", B=4, N=32, io="bf16", ragged=True, paged=True),
        # the sparse form: 85 selected blocks and a window of 512, drafts of 16
        _case("tree_32k_sparse", "tree", B=32, N=16, s=85, w=512),
        # the largest draft over the longest rows, eight query heads per KV head: bound by the matrix cores
        _case("tree_32k_64_drafts", "tree", B=8, G=8, T=32768, N=64, io="bf16"),
        # the weights of one decoded token a row (after a decode step), whole cache
        _case("weights_step_32k", "weights", B=4, draft=False),
        # an observation window: the last 64 prompt tokens over the prompt
        _case("weights_window_16k", "weights", B=2, T=16381, N=64, io="bf16"),
        # the weights of a verified draft over the selected blocks and the window, on pages
        _case("weights_sparse_64k", "weights", B=4, T=65501, N=16, s=64, w=512, paged=True),
        # eviction from a short cache
        _case("evict_4k", "evict", T=4093, keep=1024, sinks=4, recent=128),
        # eviction from a batch of the longest rows
        _case("evict_128k", "evict", B=8, T=131045, keep=32768, sinks=4, recent=1024),
        # a small fp32 cache of 64-element heads, from pages to pages
        _case("compact_2k_fp32_paged", "compact", Hkv=2, d=64, T=2011, keep=500, kv="f32", paged=True),
        # a quarter of a 32k batch kept, rows of different lengths
        _case("compact_32k", "compact", B=4, keep=8192, ragged=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["tree", "tree", "tree", "weights", "weights", "evict", "compact"])
    d = rng.choice([64, 128, 128])
    hkv = rng.choice([1, 2, 4, 8, 8])
    L = rng.choice([32, 64, 64, 64, 128])
    B = _log_int(rng, 1, 32)
    G = rng.choice([1, 2, 4, 4, 8, 16])
    kv = rng.choice(["bf16", "bf16", "bf16", "f32"])
    ragged, paged = B > 1 and rng.random() < 0.5, rng.random() < 0.4
    if op == "evict":
        T = _log_int(rng, 64, min(131072, (8 << 20) // (B * hkv)))
        keep = _log_int(rng, 16, T)
        recent = rng.randrange(0, min(keep // 2, 1024) + 1)
        return _case(None, op, B=B, Hkv=hkv, L=L, T=T, keep=keep, sinks=rng.randrange(0, min(8, keep - recent) + 1),
                     recent=recent, ragged=ragged)
    if op == "compact":
        T = _log_int(rng, 64, max(65, min(131072, (2 << 20) // (B * hkv))))
        return _case(None, op, B=B, Hkv=hkv, d=d, L=L, T=T, keep=_log_int(rng, 16, T), kv=kv, ragged=ragged, paged=paged)
    N = rng.choice([1, _log_int(rng, 1, 64), _log_int(rng, 4, 64)])
    # cache rows, scores and (fp32 caches, which the cores multiply at a sixteenth of the bf16 rate) products
    # within the largest listed cases
    most = min((4 << 20) // (B * hkv), (1 << 30) // (B * hkv * G * N))
    if kv == "f32":
        most = min(most, (1 << 26) // (B * hkv * G * N))
    T = _log_int(rng, 16, max(17, min(131072, most)))
    sparse = rng.random() < 0.4
    return _case(None, op, B=B, Hkv=hkv, G=G, d=d, L=L, T=T, N=N, s=_log_int(rng, 1, 96) if sparse else -1,
                 w=rng.randrange(0, 1025) if sparse else 0, kv=kv, io=rng.choice(["f32", "bf16"]),
                 draft=N > 1 or rng.random() < 0.5, ragged=ragged, paged=paged)


# ------------------------------------------------------------------ sizes --
def _lens(c):
    """Context tokens of every row."""
    if not c["ragged"]:
        return [c["T"]] * c["B"]
    return [c["T"] - (b * 7919) % (c["T"] // 2 + 1) for b in range(c["B"])]


def _drafts(c):
    """Drafted tokens of every row."""
    if not c["draft"]:
        return [0] * c["B"]
    return [c["N"] - (b * 7 % (c["N"] // 2 + 1) if c["ragged"] else 0) for b in range(c["B"])]


def _up(n, m):
    return -(-n // m) * m


def _capacity(c):
    return _up(c["T"] + (c["N"] if c["draft"] and c["op"] in ("tree", "weights") else 0), c["L"])


def _window_start(c, T):
    return max(0, T - c["w"])


def _torch_type(name):
    return {"f32": torch.float32, "bf16": torch.bfloat16}[name]


# ----------------------------------------------------------------- inputs --
def _device():
    return "cuda" if torch.cuda.is_available() else "cpu"


def _tree_bits(c, gen):
    """Ancestor bits (itself included) of a random tree in each row."""
    N, rows = c["N"], []
    for _ in range(c["B"]):
        back = torch.randint(0, 4, (N,), generator=gen).tolist()
        bits = []
        for i in range(N):
            parent = i - 1 - back[i]
            bits.append((1 << i) | (bits[parent] if parent >= 0 else 0))
        rows.append([x - (1 << 64) if x >= 1 << 63 else x for x in bits])
    return torch.tensor(rows, dtype=torch.int64)


def _cache(c, capacity, gen, dev, zeros=False):
    """Keys, values and, on pages, the table [B, capacity / L] of a shuffled pool with spare pages."""
    B, H, L, d, nb = c["B"], c["Hkv"], c["L"], c["d"], capacity // c["L"]
    pages = B * nb + 7 if c["paged"] else 0
    shape = (pages, H, L, d) if c["paged"] else (B, H, capacity, d)
    t = _torch_type(c["kv"])
    if zeros:
        k, v = torch.zeros(shape, dtype=t, device=dev), torch.zeros(shape, dtype=t, device=dev)
    else:
        k = torch.randn(shape, generator=gen, device=dev, dtype=t)
        v = torch.randn(shape, generator=gen, device=dev, dtype=t)
        mean = 0.3 * torch.randn((pages, H, 1, d) if c["paged"] else (B, H, nb, 1, d), generator=gen, device=dev, dtype=t)
        (k if c["paged"] else k.view(B, H, nb, L, d)).add_(mean)
    if not c["paged"]:
        return k, v, None
    table = torch.argsort(torch.rand(pages, generator=gen, device=dev))[:B * nb].to(torch.int32).view(B, nb)
    return k, v, table


def prepare(case, seed):
    c, dev = case, _device()
    gen, host = torch.Generator(device=dev), torch.Generator()
    gen.manual_seed(int(seed))
    host.manual_seed(int(seed))
    B, H, d, N, cap = c["B"], c["Hkv"], c["d"], c["N"], _capacity(c)
    lens = torch.tensor(_lens(c), dtype=torch.int32, device=dev)
    s = dict(case=c, seq_lens=lens, capacity=cap)
    if c["op"] in ("tree", "weights"):
        s["k"], s["v"], s["table"] = _cache(c, cap, gen, dev)
        s["q"] = torch.randn((B, N, H * c["G"], d), generator=gen, device=dev).to(_torch_type(c["io"]))
        s["draft_lens"] = s["bits"] = s["sel"] = None
        if c["draft"]:
            s["draft_lens"] = torch.tensor(_drafts(c), dtype=torch.int32, device=dev)
            s["bits"] = _tree_bits(c, host).to(dev)
        if c["s"] >= 0:
            # as many candidate blocks as the budget holds, ascending, then -1
            cand = -(-(lens.long() - c["w"]).clamp(min=0) // c["L"]).view(B, 1, 1)
            rank = torch.rand((B, H, cap // c["L"]), generator=gen, device=dev)
            at = torch.arange(cap // c["L"], device=dev)
            rank = torch.where(at < cand, rank, rank + 2.0)
            pick = torch.argsort(rank, -1)[..., :c["s"]]
            pick = torch.where(pick < cand, pick, torch.full_like(pick, 1 << 30)).sort(-1)[0]
            pick = torch.where(pick < 1 << 30, pick, torch.full_like(pick, -1))
            pad = torch.full((B, H, c["s"] - pick.shape[-1]), -1, dtype=pick.dtype, device=dev)
            s["sel"] = torch.cat([pick, pad], -1).to(torch.int32).contiguous()
        if c["op"] == "tree":
            s["out"], s["lse"] = torch.empty_like(s["q"]), torch.empty((B, N, H * c["G"]), device=dev)
        else:
            # the normaliser that the queries' attention returned, and the weights of earlier steps
            s["lse"] = _attend(s, False)[1].contiguous()
            s["prev"] = (8.0 * c["G"] * N / c["T"]) * torch.rand((B, H, cap), generator=gen, device=dev) ** 4
            s["weights"] = torch.zeros((B, H, cap), device=dev)
        return s
    # accumulated weights: a few heavy tokens, most light, some never attended to
    weights = torch.exp(2.0 * torch.randn((B, H, cap), generator=gen, device=dev) - 4.0)
    weights = torch.where(torch.rand((B, H, cap), generator=gen, device=dev) < 0.05, torch.zeros_like(weights), weights)
    s["weights"] = weights
    if c["op"] == "evict":
        s["kept"] = torch.empty((B, H, c["keep"]), dtype=torch.int32, device=dev)
        s["new_lens"] = torch.empty(B, dtype=torch.int32, device=dev)
        return s
    s["k"], s["v"], s["table"] = _cache(c, cap, gen, dev)
    s["out_capacity"] = _up(c["keep"], c["L"])
    s["k_out"], s["v_out"], s["out_table"] = _cache(c, s["out_capacity"], gen, dev, zeros=True)
    s["weights_out"] = torch.zeros((B, H, s["out_capacity"]), device=dev)
    # a random choice of each row's tokens, ascending, then -1
    rank = torch.rand((B, H, cap), generator=gen, device=dev)
    T = lens.long().view(B, 1, 1)
    rank = torch.where(torch.arange(cap, device=dev) < T, rank, rank + 2.0)
    pick = torch.argsort(rank, -1)[..., :c["keep"]]
    pick = torch.where(pick < T, pick, torch.full_like(pick, 1 << 30)).sort(-1)[0]
    s["kept"] = torch.where(pick < 1 << 30, pick, torch.full_like(pick, -1)).to(torch.int32).contiguous()
    return s


# ------------------------------------------------------------ plain forms --
def _rows(x, table, heads):
    """A cache as [B, Hkv, capacity, d]: itself, or its pages in order."""
    if table is None:
        return x
    B, nb = table.shape
    return x[table.long()].permute(0, 2, 1, 3, 4).reshape(B, heads, nb * x.shape[2], x.shape[3])


def _visible(s, t):
    """Which tokens `t` (positions) each query attends to: [B, Hkv or 1, N, len(t)]."""
    c = s["case"]
    T = s["seq_lens"].long().view(-1, 1, 1, 1)
    if s["sel"] is None:
        context = t < T
    else:
        # a block is selected or not: one flag per block, looked up by position
        flags = torch.zeros((c["B"], c["Hkv"], s["capacity"] // c["L"] + 1), dtype=torch.bool, device=t.device)
        flags.scatter_(2, torch.where(s["sel"] >= 0, s["sel"], torch.full_like(s["sel"], flags.shape[2] - 1)).long(), True)
        start = (T - c["w"]).clamp(min=0)
        picked = flags[:, :, t // c["L"]].unsqueeze(2) & (t // c["L"] < flags.shape[2] - 1)
        context = (t < T) & ((t >= start) | picked)
    context = context.expand(-1, -1, c["N"], -1)
    if s["bits"] is None:
        return context
    n = s["draft_lens"].long().view(-1, 1, 1, 1)
    j = t - T
    i = torch.arange(c["N"], device=t.device).view(1, 1, -1, 1)
    drafted = (j >= 0) & (j < n) & ((s["bits"].view(c["B"], 1, c["N"], 1) >> j.clamp(0, 63)) & 1).bool()
    return (context | drafted) & (i < n)


def _scores(s):
    """c q.k in 32 bits, -inf where a query does not attend: [B, Hkv, N, G, capacity]."""
    c = s["case"]
    B, H, G, N, d = c["B"], c["Hkv"], c["G"], c["N"], c["d"]
    k = _rows(s["k"], s["table"], H).float()
    q = s["q"].float().view(B, N, H, G, d).permute(0, 2, 1, 3, 4).reshape(B, H, N * G, d)
    x = torch.matmul(q, k.transpose(-1, -2)).mul_(1.0 / math.sqrt(d)).view(B, H, N, G, s["capacity"])
    seen = _visible(s, torch.arange(s["capacity"], device=k.device))
    return x.masked_fill_(~seen.unsqueeze(3), -math.inf)


def _attend(s, with_out=True):
    c = s["case"]
    B, H, G, N, d = c["B"], c["Hkv"], c["G"], c["N"], c["d"]
    x = _scores(s)
    top = x.amax(-1, keepdim=True)
    top = torch.where(top > -math.inf, top, torch.zeros_like(top))
    x = x.sub_(top).exp_()
    total = x.sum(-1, keepdim=True)
    lse = (total.log() + top).view(B, H, N, G).permute(0, 2, 1, 3).reshape(B, N, H * G)
    if not with_out:
        return None, lse
    out = torch.matmul(x.view(B, H, N * G, -1), _rows(s["v"], s["table"], H).float()).view(B, H, N, G, d)
    out = torch.where(total > 0, out / total, torch.zeros_like(out))
    return out.permute(0, 2, 1, 3, 4).reshape(B, N, H * G, d).to(s["q"].dtype), lse


def _plain_weights(s):
    c = s["case"]
    B, H, G, N = c["B"], c["Hkv"], c["G"], c["N"]
    lse = s["lse"].view(B, N, H, G).permute(0, 2, 1, 3).unsqueeze(-1)
    x = _scores(s)
    added = x.sub_(torch.where(lse > -math.inf, lse, torch.full_like(lse, math.inf))).exp_().sum((2, 3))
    held = s["seq_lens"].long() + (s["draft_lens"].long() if s["bits"] is not None else 0)
    t = torch.arange(s["capacity"], device=x.device)
    return torch.where(t < held.view(B, 1, 1), s["prev"] + added, s["weights"])


def _plain_evict(s):
    c, w = s["case"], s["weights"]
    keep, t = c["keep"], torch.arange(w.shape[-1], device=w.device)
    T = s["seq_lens"].long().view(-1, 1, 1)
    order = torch.sort(w.nan_to_num(nan=-math.inf, posinf=math.inf, neginf=-math.inf), dim=-1, descending=True, stable=True)[1]
    always = (t < c["sinks"]) | (t >= T - c["recent"])
    rank = torch.where(t < T, torch.where(always, 0, 1), 2).expand_as(w)
    order = order.gather(-1, torch.sort(rank.gather(-1, order), dim=-1, stable=True)[1])
    kept = order[..., :keep].sort(-1)[0]
    kept = torch.where(kept < T, kept, torch.full_like(kept, -1))
    return kept.to(torch.int32), s["seq_lens"].clamp(max=keep)


def _plain_compact(s):
    c = s["case"]
    B, H, n, L = c["B"], c["Hkv"], c["keep"], c["L"]
    at, valid = s["kept"].clamp(min=0).long(), s["kept"] >= 0
    got = []
    for x, out in ((s["k"], s["k_out"]), (s["v"], s["v_out"])):
        rows = _rows(x, s["table"], H).gather(2, at.unsqueeze(-1).expand(-1, -1, -1, c["d"]))
        if s["out_table"] is None:
            out[:, :, :n] = torch.where(valid.unsqueeze(-1), rows, out[:, :, :n])
        else:
            j = torch.arange(n, device=x.device)
            where = (s["out_table"][:, j // L].long().unsqueeze(1), torch.arange(H, device=x.device).view(1, -1, 1),
                     (j % L).view(1, 1, -1))
            out[where] = torch.where(valid.unsqueeze(-1), rows, out[where])
        got.append(out)
    s["weights_out"][:, :, :n] = torch.where(valid, s["weights"].gather(2, at), torch.zeros_like(s["weights_out"][:, :, :n]))
    return got + [s["weights_out"]]


# --------------------------------------------------------- the framework's --
def _plan(s):
    """The problem description and the workspace that a program keeps."""
    from paper_2607_09052_amd import cache, cobs
    if "plan" not in s:
        c = s["case"]
        cfg = cobs.Config(batch=c["B"], num_q_heads=c["Hkv"] * c["G"], num_kv_heads=c["Hkv"], head_dim=c["d"],
                          max_seq_len=s["capacity"], rank=0, budget=max(c["s"], 0), window=c["w"], kv_dtype=c["kv"],
                          block_size=c["L"])
        ws = None
        if c["op"] == "tree":
            ws = cache.new_tree_workspace(cfg, c["N"], s["q"].device)
        elif c["op"] == "evict":
            ws = cache.new_evict_workspace(cfg, s["weights"].device)
        s["plan"] = (cache, cfg, ws)
    return s["plan"]


def _own_run(s):
    cache, cfg, ws = _plan(s)
    c = s["case"]
    pages = {}
    if s.get("table") is not None:
        pages = dict(block_table=s["table"], num_pages=s["k"].shape[0])
    if c["op"] == "tree":
        cache.cobs_tree_decode(cfg, s["q"], s["k"], s["v"], s["seq_lens"], s["draft_lens"], s["bits"], s["out"], ws,
                               sel=s["sel"], lse=s["lse"], **pages)
        return s["out"], s["lse"]
    if c["op"] == "weights":
        cache.cobs_attention_weights(cfg, s["q"], s["k"], s["v"], s["seq_lens"], s["draft_lens"], s["bits"], s["lse"],
                                     s["weights"], prev=s["prev"], sel=s["sel"], **pages)
        return s["weights"]
    if c["op"] == "evict":
        cache.cobs_evict(cfg, s["weights"], s["seq_lens"], s["kept"], ws, sinks=c["sinks"], recent=c["recent"],
                         new_lens=s["new_lens"])
        return s["kept"], s["new_lens"]
    if s["out_table"] is not None:
        pages.update(out_block_table=s["out_table"], out_num_pages=s["k_out"].shape[0])
    cache.cobs_compact_cache(cfg, s["k"], s["v"], s["kept"], s["seq_lens"], k_out=s["k_out"], v_out=s["v_out"],
                             weights=s["weights"], weights_out=s["weights_out"], **pages)
    return [s["k_out"], s["v_out"], s["weights_out"]]


def run(state):
    if own:
        return _own_run(state)
    plain = dict(tree=_attend, weights=_plain_weights, evict=_plain_evict, compact=_plain_compact)
    return plain[state["case"]["op"]](state)


# ------------------------------------------------------------------- work --
def _selected(c, T):
    """Tokens of the context that one unit attends to."""
    if c["s"] < 0:
        return T
    start = _window_start(c, T)
    return min(start, c["s"] * c["L"]) + T - start


def work(case):
    c = case
    es, H, G, d = (4 if c["kv"] == "f32" else 2), c["Hkv"], c["G"], c["d"]
    nbytes = flops = 0
    for T, n in zip(_lens(c), _drafts(c)):
        if c["op"] == "evict":
            nbytes += H * 4 * (T + min(T, c["keep"]))
            flops += H * T
        elif c["op"] == "compact":
            m = min(T, c["keep"])
            nbytes += H * m * (2 * 2 * d * es + 2 * 4 + 4)
        else:
            q = n if c["draft"] else c["N"]
            seen = _selected(c, T)
            io = 2 if c["io"] == "bf16" else 4
            pairs = H * G * (q * seen + (q * (q + 1)) // 2 * c["draft"])   # a draft token sees at most its predecessors
            if c["op"] == "tree":
                nbytes += H * (seen + n) * 2 * d * es + H * G * q * (2 * d * io + 4)
                flops += 4 * d * pairs
            else:
                nbytes += H * (seen + n) * (d * es + 8) + H * G * q * (d * io + 4)
                flops += 2 * d * pairs
    return dict(bytes=nbytes, flops=flops)


# ------------------------------------------------------------- definition --
def _exact_attention(s):
    """out, lse and the weights' sums in 64 bits, one row after the other, from the definition."""
    c = s["case"]
    H, G, N, d, L = c["Hkv"], c["G"], c["N"], c["d"], c["L"]
    dev, cap = s["q"].device, s["capacity"]
    outs, lses, sums = [], [], []
    for b in range(c["B"]):
        T, n = _lens(c)[b], _drafts(c)[b]
        k, v = s["k"], s["v"]
        if s["table"] is None:
            k, v = k[b], v[b]
        else:
            page = s["table"][b].long()
            k, v = (x[page].transpose(0, 1).reshape(H, cap, d) for x in (k, v))
        see = torch.zeros((H, N, cap), dtype=torch.bool, device=dev)
        if s["sel"] is None:
            see[:, :, :T] = True
        else:
            see[:, :, _window_start(c, T):T] = True
            for h, blocks in enumerate(s["sel"][b].tolist()):
                for x in blocks:
                    if x >= 0:
                        see[h, :, x * L:min(x * L + L, T)] = True
        if c["draft"]:
            for i, bits in enumerate(s["bits"][b].tolist()):
                for j in range(n):
                    see[:, i, T + j] = bool((bits >> j) & 1)
            see[:, n:] = False
        out, lse, total = [], [], []
        for h in range(H):
            q = s["q"][b, :, h * G:(h + 1) * G].double().reshape(N * G, d)
            x = q @ k[h].double().T.contiguous() / math.sqrt(d)
            x = x.masked_fill(~see[h].repeat_interleave(G, 0), -math.inf)
            z = torch.logsumexp(x, -1)
            if c["op"] == "weights":
                z = s["lse"][b, :, h * G:(h + 1) * G].double().reshape(N * G)
                z = torch.where(torch.isfinite(z), z, torch.full_like(z, math.inf))
                total.append(torch.exp(x - z[:, None]).sum(0))
                continue
            p = torch.exp(x - torch.where(torch.isfinite(z), z, torch.zeros_like(z))[:, None])
            out.append((p @ v[h].double()).view(N, G, d))
            lse.append(z.view(N, G))
        if c["op"] == "weights":
            held = T + n
            total = torch.stack(total) + s["prev"][b].double()
            total[:, held:] = s["weights"][b, :, held:].double()
            sums.append(total)
        else:
            outs.append(torch.stack(out, 1).reshape(N, H * G, d))
            lses.append(torch.stack(lse, 1).reshape(N, H * G))
    if c["op"] == "weights":
        return torch.stack(sums)
    return torch.stack(outs), torch.stack(lses)


def _exact_compact(s):
    c = s["case"]
    L = c["L"]
    got = [x.double().clone() for x in (s["k_out"], s["v_out"], s["weights_out"])]
    for b in range(c["B"]):
        for h in range(c["Hkv"]):
            at = s["kept"][b, h].long()
            at = at[at >= 0]
            j = torch.arange(at.numel(), device=at.device)
            for x, out in ((s["k"], got[0]), (s["v"], got[1])):
                rows = x[b, h, at] if s["table"] is None else x[s["table"][b].long()[at // L], h, at % L]
                if s["out_table"] is None:
                    out[b, h, j] = rows.double()
                else:
                    out[s["out_table"][b].long()[j // L], h, j % L] = rows.double()
            got[2][b, h, j] = s["weights"][b, h, at].double()
    return got


def exact(case, seed):
    if case["op"] == "evict":
        return None                     # whole numbers
    s = prepare(case, seed)
    return _exact_compact(s) if case["op"] == "compact" else _exact_attention(s)
