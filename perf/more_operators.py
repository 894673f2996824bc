"""Operators around mixed attention over the paged KV cache, as cases that a timing program can run.

A case is one pass of one batch, one layer, on tensors that are already on the GPU:

  "rows"    the rows that the projections give become what attention works on: each head of q and k is divided by the root
            of its mean square (and multiplied by a weight for each element), then rotated by its position's angles.
            `append`: k goes on into the cache, v with it; else k comes back as rows, for a cache of another kind
  "window"  attention over the newest `window` tokens of each sequence and its `sinks` first ones
  "shared"  attention of sequences that begin with the same cached tokens

A batch is given by `chunk` (a prompt chunk as "tokens@offset", or nothing) and by `decodes` running requests whose
context lengths follow from `context` ("lognormal mean sigma low high" or "uniform low high") and `lengths` (the seed
of the draw); `groups` ("tokens:sequences tokens:sequences ..") says what the batch's sequences begin with, in their order,
offsets and lengths then count from there.  The seed given to prepare() makes tensors and block tables.

Layouts (B = 16 tokens to a block, D = head_dim):
  rows     [tokens][heads + 2 kv heads][D]   q, k and v of a token one after the other
  k pool   [blocks][kv heads][D/8][B][8]     d = 8 i + l of token t at [i][t][l]
  v pool   [blocks][kv heads][D][B]          token t at index t with bits 2 and 3 exchanged
"""
import math

import numpy as np
import torch

own = False

BLOCK = 16  # tokens per KV block
GPU = "cuda:0"
EPS = 1e-6
SLOT = [t & 3 | (t & 4) << 1 | (t & 8) >> 1 for t in range(BLOCK)]  # where token t lies in a row of a V block, and the other way round


def _case(name, kind, heads, kv_heads, head_dim, dtype, chunk, decodes, context, lengths, **more):
    return {"name": name, "kind": kind, "heads": heads, "kv_heads": kv_heads, "head_dim": head_dim, "dtype": dtype, "chunk": chunk,
            "decodes": decodes, "context": context, "lengths": lengths, **more}


def listed():
    return [
        # A handful of chat requests, a token each: the smallest call of a decode loop.
        _case("rows_few", "rows", 32, 8, 128, "bf16", "", 8, "lognormal 1024 0.8 64 4096", 1, append=True, rotary=128, pairs="halves", base=500000.0),
        # A full instance: a token of every request; half of each head is rotated, as adjacent pairs.
        _case("rows_decodes", "rows", 40, 8, 128, "fp16", "", 512, "uniform 16 512", 2, append=True, rotary=64, pairs="adjacent", base=10000.0),
        # A long prompt's later half arrives, a few decodes ride along.
        _case("rows_prompt", "rows", 64, 8, 128, "bf16", "8192@8192", 4, "uniform 500 1500", 3, append=True, rotary=128, pairs="halves", base=1000000.0),
        # Rows for a cache of another kind: a chunk of odd length of a model with a KV head for each query head.
        _case("rows_apart", "rows", 32, 32, 64, "bf16", "1234@1000", 16, "lognormal 1024 0.8 64 4096", 4, append=False, rotary=64, pairs="halves", base=10000.0),
        # Decode only at low load: launches and the chain of latencies.
        _case("window_few", "window", 32, 8, 128, "bf16", "", 8, "lognormal 4096 0.8 64 16384", 5, window=1024, sinks=4, gain=1.0),
        # Decode only at high load, some requests not yet as long as the window: bytes.
        _case("window_decodes", "window", 40, 8, 128, "fp16", "", 128, "uniform 512 8192", 6, window=2048, sinks=16, gain=2.0),
        # A mixed batch: a chunk in the middle of a prompt, some decodes, a window at no block's border.
        _case("window_mixed", "window", 32, 8, 128, "bf16", "2048@4096", 64, "lognormal 2048 0.8 64 8192", 7, window=1000, sinks=0, gain=1.0),
        # A long prompt in one chunk: matrix products.
        _case("window_prompt", "window", 64, 8, 128, "bf16", "8192@4100", 0, "uniform 1 1", 8, window=2048, sinks=4, gain=1.0),
        # Four requests behind one system prompt.
        _case("shared_few", "shared", 32, 8, 128, "bf16", "", 4, "lognormal 128 0.8 1 1024", 9, groups="2048:4", gain=1.0),
        # A long instruction that every request of a service begins with.
        _case("shared_decodes", "shared", 32, 8, 128, "bf16", "", 256, "uniform 64 1024", 10, groups="8192:256", gain=1.0),
        # Several services on one instance, and requests that share nothing; IEEE half, a small model.
        _case("shared_groups", "shared", 16, 2, 64, "fp16", "", 113, "uniform 1 700", 11, groups="4096:64 1008:33 0:16", gain=2.0),
        # Questions about one long document: a new one's prompt, and the answers under way.
        _case("shared_chunk", "shared", 64, 8, 128, "bf16", "512@100", 63, "uniform 100 900", 12, groups="16384:64", gain=1.0),
    ]


def _cost(case):
    w = work(case)
    return w["bytes"] / 5e12 + w["flops"] / 1e15


def draw(rng):
    """One more case of the same ranges: any operator, any load from one decode to a full instance, any chunk from none to the largest."""
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    heads, kv_heads = rng.choice([(32, 8), (32, 8), (40, 8), (64, 8), (8, 8), (32, 32), (16, 2)])
    kind, dim, dtype = rng.choice(["rows", "window", "window", "shared", "shared"]), rng.choice([128, 128, 64]), rng.choice(["bf16", "bf16", "fp16"])
    case = _case("", kind, heads, kv_heads, dim, dtype, "", 0, "", rng.randrange(1 << 20))
    del case["name"]
    most = 1.0e9 / (kv_heads * dim)  # tokens that the decodes may have, each as long as the longest may be: 2 GB of K
    mean = log(16, 8192 if kind == "window" else 2048 if kind == "shared" else 512)
    case["context"] = rng.choice(["lognormal %d 0.8 1 %d" % (mean, 2 * mean), "uniform %d %d" % (max(1, mean // 4), 2 * mean)])
    prefix = BLOCK * log(1, 1024)
    whole = 2 * mean + (prefix if kind == "shared" else 0)
    case["decodes"] = max(1, min(log(1, 512), int(most / whole)))
    if rng.random() < 0.6:
        case["chunk"] = "%d@%d" % (log(2, 8192), rng.choice([0, log(1, 16384)]))
        if kind != "shared" and rng.random() < 0.3:
            case["decodes"], case["context"] = 0, "uniform 1 1"
    if kind == "rows":
        case["append"], case["rotary"] = rng.random() < 0.7, rng.choice([dim, dim, dim // 2, 48])
        case["pairs"], case["base"] = rng.choice(["halves", "halves", "adjacent"]), rng.choice([10000.0, 500000.0])
    else:
        case["gain"] = rng.choice([1.0, 2.0, 3.0])
    if kind == "window":
        case["window"], case["sinks"] = log(1, 4096), rng.choice([0, 1, 4, log(1, 200)])
    if kind == "shared":
        n = case["decodes"] + bool(case["chunk"])
        a = rng.randint(0, n)
        b = rng.randint(a, n)
        case["groups"] = rng.choice(["%d:%d" % (prefix, n), "%d:%d" % (prefix, n), "%d:%d %d:%d 0:%d" % (prefix, a, BLOCK * log(1, prefix // BLOCK + 1), b - a, n - b)])
    # no more work than the largest listed call
    while case["chunk"] and (_cost(case) > 9e-4 or heads * _chunk(case)[0] * sum(_chunk(case)) > 64 * 8192 * 12292):
        tokens, offset = (int(x) for x in case["chunk"].split("@"))
        case["chunk"] = "%d@%d" % (max(2, tokens // 2), offset // 2)
    return case


def _groups(case):
    """What each sequence begins with: cached tokens that its group shares, and the group's number."""
    pairs = [g.split(":") for g in case.get("groups", "0:%d" % (case["decodes"] + bool(case["chunk"]))).split()]
    return np.repeat([int(p) for p, _ in pairs], [int(n) for _, n in pairs]), np.repeat(np.arange(len(pairs)), [int(n) for _, n in pairs])


def _chunk(case):
    """New tokens of the chunk and the tokens before them."""
    tokens, offset = (int(x) for x in case["chunk"].split("@"))
    return tokens, offset + int(_groups(case)[0][0])


def _lengths(case):
    """New tokens and cached tokens of every sequence: the chunk, then the decodes (their context counts the new token)."""
    rs = np.random.RandomState(case["lengths"] % (1 << 31))
    law, *num = case["context"].split()
    num = [float(x) for x in num]
    n = case["decodes"]
    if law == "lognormal":
        mean, sigma, lo, hi = num
        kv = np.clip(np.rint(np.exp(rs.normal(math.log(mean) - 0.5 * sigma * sigma, sigma, n))), lo, hi)
    else:
        kv = rs.randint(int(num[0]), int(num[1]) + 1, n)
    chunk = [tuple(int(x) for x in c.split("@")) for c in case["chunk"].split()]
    q_len = np.array([c[0] for c in chunk] + [1] * n, np.int64)
    ctx = np.array([c[1] for c in chunk] + [int(x) - 1 for x in kv], np.int64)
    return q_len, ctx + _groups(case)[0]


def prepare(case, seed):
    q_len, ctx = _lengths(case)
    dtype = torch.bfloat16 if case["dtype"] == "bf16" else torch.float16
    heads, kv_heads, dim, kind = case["heads"], case["kv_heads"], case["head_dim"], case["kind"]
    rs = np.random.RandomState((seed * 2 + 1) % (1 << 31))
    gen = torch.Generator(device=GPU).manual_seed(seed)
    kv_len = q_len + ctx
    pages = -(-kv_len // BLOCK)
    q_start = np.concatenate([[0], np.cumsum(q_len)]).astype(np.int32)
    tokens = int(q_start[-1])
    # block tables over a pool with a quarter of its blocks to spare, the blocks scattered as a running allocator leaves them
    blocks = int(pages.sum()) + max(4, int(pages.sum()) // 4)
    if kind == "shared":
        blocks = int((pages - _groups(case)[0] // BLOCK).sum()) + sum(int(g.split(":")[0]) // BLOCK for g in case["groups"].split())
        blocks += max(4, blocks // 4)
    prefix, group = _groups(case)
    table = np.zeros((len(kv_len), int(pages.max())), np.int32)
    first = np.unique(group, return_index=True)[1][np.searchsorted(np.unique(group), group)]  # of each sequence's group
    mine = np.arange(table.shape[1])[None, :] < pages[:, None]
    mine &= (np.arange(table.shape[1])[None, :] >= prefix[:, None] // BLOCK) | (first == np.arange(len(kv_len)))[:, None]
    table[mine] = rs.permutation(blocks).astype(np.int32)[:int(mine.sum())]
    table = np.where(np.arange(table.shape[1])[None, :] < prefix[:, None] // BLOCK, table[first], table)

    def normal(gain, *shape):
        return torch.empty(shape, dtype=dtype, device=GPU).normal_(0.0, gain, generator=gen)

    state = {"case": case, "q_len": q_len, "ctx": ctx, "table": table, "q_start": q_start, "scale": 1.0 / math.sqrt(dim)}
    if kind != "rows" or case["append"]:  # cached tokens, and leftovers of earlier requests in the free slots
        state["k_pool"] = normal(1.0, blocks, kv_heads, dim // 8, BLOCK, 8)
        state["v_pool"] = normal(1.0, blocks, kv_heads, dim, BLOCK)
    if kind == "rows":
        state["rows"] = normal(1.0, tokens, heads + 2 * kv_heads, dim)
        state["q_weight"], state["k_weight"] = (1.0 + normal(0.2, dim).float()).to(dtype), (1.0 + normal(0.2, dim).float()).to(dtype)
        state["freq"] = case["base"] ** (torch.arange(case["rotary"] // 2, dtype=torch.float64, device=GPU) * (-2.0 / case["rotary"]))
        state["q_out"] = torch.zeros((tokens, heads, dim), dtype=dtype, device=GPU)
        if not case["append"]:
            state["k_out"] = torch.zeros((tokens, kv_heads, dim), dtype=dtype, device=GPU)
    else:
        state["q"] = normal(case["gain"], tokens, heads, dim)
        state["out"] = torch.zeros((tokens, heads, dim), dtype=dtype, device=GPU)
    if own:
        import paper_2508_01989_amd as tc
        pool = tc.make_pool(heads, kv_heads, dim, blocks, state.get("k_pool"), state.get("v_pool"), dtype=tc.TC_BF16 if case["dtype"] == "bf16" else tc.TC_FP16)
        plan = state["plan"] = tc.Plan(pool, q_start, ctx.astype(np.int32), table)
        state["pool"] = pool
        if kind == "window":
            plan.set_window(case["window"], case["sinks"])
            state["workspace"] = torch.empty(max(16, plan.window_workspace_bytes), dtype=torch.uint8, device=GPU)
        if kind == "shared":
            counts = [int(g.split(":")[1]) for g in case["groups"].split()]
            some = [i for i, c in enumerate(counts) if c]
            starts = np.concatenate([[0], np.cumsum(counts)])
            plan.set_shared([int(starts[i]) for i in some] + [int(starts[-1])], [int(case["groups"].split()[i].split(":")[0]) for i in some])
            state["workspace"] = torch.empty(max(16, plan.shared_workspace_bytes), dtype=torch.uint8, device=GPU)
    # the same batch as the index tensors that a program without the library keeps for its iteration
    seq = np.repeat(np.arange(len(q_len)), q_len)
    at = np.arange(tokens) - q_start[seq] + ctx[seq]  # position of every new row
    state["position"] = torch.from_numpy(at).to(GPU)
    state["block"], state["slot"] = torch.from_numpy(table[seq, at // BLOCK].astype(np.int64)).to(GPU), torch.from_numpy(at % BLOCK).to(GPU)
    state["table_gpu"] = torch.from_numpy(table.astype(np.int64)).to(GPU)
    state["kv_len_gpu"] = torch.from_numpy(kv_len).to(GPU)
    state["v_slot"] = torch.tensor(SLOT, device=GPU)
    return state


# ---- the plain form: elementary operations in 32 bits

def _norm_rotate(x, weight, position, state):
    """Heads of rows, each divided by its root mean square, times the weight; then pairs of elements turned by position * frequency."""
    case, x = state["case"], x.float()
    x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * weight.float()
    n = case["rotary"]
    angle = (position.double()[:, None] * state["freq"])[:, None, :]
    cos, sin = angle.cos().float(), angle.sin().float()
    halves = case["pairs"] == "halves"
    a, b = (x[..., :n // 2], x[..., n // 2:n]) if halves else (x[..., 0:n:2], x[..., 1:n:2])
    turned = (a * cos - b * sin, b * cos + a * sin)
    turned = torch.cat(turned, -1) if halves else torch.stack(turned, -1).flatten(-2)
    return torch.cat([turned, x[..., n:]], -1).to(state["q_out"].dtype)


def _rows(state):
    heads, kv_heads, rows = state["case"]["heads"], state["case"]["kv_heads"], state["rows"]
    state["q_out"].copy_(_norm_rotate(rows[:, :heads], state["q_weight"], state["position"], state))
    k = _norm_rotate(rows[:, heads:heads + kv_heads], state["k_weight"], state["position"], state)
    if not state["case"]["append"]:
        state["k_out"].copy_(k)
        return
    state["k_pool"][state["block"], :, :, state["slot"]] = k.unflatten(-1, (-1, 8))
    state["v_pool"][state["block"], :, :, state["v_slot"][state["slot"]]] = rows[:, heads + kv_heads:]


def _cached(state, first, last, low, count):
    """K and V of the tokens low + 0 .. low + count - 1 of the sequences [first, last), float32 [n][kv heads][token][d].  `low`: of each sequence."""
    at = low[:, None] + torch.arange(count, device=GPU)
    ids = state["table_gpu"][first:last].gather(1, (at // BLOCK).clamp_max(state["table_gpu"].shape[1] - 1))
    k = state["k_pool"][ids, :, :, at % BLOCK].float().flatten(-2)
    v = state["v_pool"][ids, :, :, state["v_slot"][at % BLOCK]].float()
    return k.transpose(1, 2), v.transpose(1, 2), at


def _attend(state, first, last, window, sinks):
    """Rows of the sequences [first, last), all of them with as many new tokens as the first has.  Keys: from the first one in the first row's window on, and the sinks."""
    case, rows = state["case"], int(state["q_len"][first])
    heads, kv_heads, dim, n = case["heads"], case["kv_heads"], case["head_dim"], last - first
    a = int(state["q_start"][first])
    q = state["q"][a:a + n * rows].float().view(n, rows, kv_heads, heads // kv_heads, dim).permute(0, 2, 3, 1, 4).reshape(n, kv_heads, -1, dim)
    position = state["position"][a:a + n * rows].view(n, rows, 1)
    low = (position[:, 0, 0] - window + 1).clamp_min(0)
    ctx = state["ctx"][first:last]
    count = int((ctx + rows - np.maximum(ctx - window + 1, 0)).max())
    k, v, at = (torch.cat([x0, x], d) for x0, x, d in zip(_cached(state, first, last, low - low, sinks), _cached(state, first, last, low, count), (2, 2, 1)))
    in_window, at = torch.arange(sinks + count, device=GPU) >= sinks, at[:, None]
    sees = (at <= position) & torch.where(in_window, at > position - window, at <= position - window)  # a sink that is in the window counts there
    x = torch.matmul(q * state["scale"], k.transpose(2, 3)).view(n, heads, rows, -1)
    x = x.masked_fill_(~sees[:, None], -math.inf)
    x = x.sub_(x.amax(-1, keepdim=True)).exp_().view(n, kv_heads, -1, k.shape[2])
    v = v * (at[:, 0] < state["kv_len_gpu"][first:last, None])[:, None, :, None]  # what lies behind the last token may be anything
    o = torch.matmul(x, v) / x.sum(-1, keepdim=True)
    o = o.view(n, kv_heads, heads // kv_heads, rows, dim).permute(0, 3, 1, 2, 4).reshape(n * rows, heads, dim)
    state["out"][a:a + n * rows] = o.to(state["out"].dtype)


def _plain(state):
    case, chunks = state["case"], int(state["q_len"][0] > 1)
    if case["kind"] == "rows":
        return _rows(state)
    window, sinks = (case["window"], case["sinks"]) if case["kind"] == "window" else (1 << 31, 0)
    if chunks:
        _attend(state, 0, 1, window, sinks)
    if len(state["q_len"]) > chunks:
        _attend(state, chunks, len(state["q_len"]), window, sinks)


def run(state):
    case = state["case"]
    if own:
        import paper_2508_01989_amd as tc
        plan, pool = state["plan"], state["pool"]
        if case["kind"] == "rows":
            heads, kv_heads, rows = case["heads"], case["kv_heads"], state["rows"]
            rows = tc.make_qkv_rows(rows[:, :heads], rows[:, heads:heads + kv_heads], rows[:, heads + kv_heads:], q_weight=state["q_weight"], k_weight=state["k_weight"],
                                    eps=EPS, freq=state["freq"], rotary_dim=case["rotary"], adjacent=case["pairs"] == "adjacent")
            if case["append"]:
                tc.tc_qk_norm_rotate_append(plan, pool, rows, state["q_out"])
            else:
                tc.tc_qk_norm_rotate(plan, rows, state["q_out"], state["k_out"])
        elif case["kind"] == "window":
            tc.tc_window_attention(plan, pool, state["q"], state["out"], state["scale"], state["workspace"])
        else:
            tc.tc_shared_attention(plan, pool, state["q"], state["out"], state["scale"], state["workspace"])
    else:
        _plain(state)
    if case["kind"] != "rows":
        return state["out"]
    return (state["q_out"], state["k_pool"], state["v_pool"]) if case["append"] else (state["q_out"], state["k_out"])


def work(case):
    q, c = _lengths(case)
    heads, kv_heads, dim = case["heads"], case["kv_heads"], case["head_dim"]
    tokens, token = int(q.sum()), 4 * kv_heads * dim  # bytes of K and V of a token
    n_bytes = 2 * tokens * heads * dim * 2
    if case["kind"] == "rows":
        return {"bytes": n_bytes + (2 if case["append"] else 1) * tokens * token, "flops": 0}
    if case["kind"] == "window":
        w, s = case["window"], case["sinks"]
        low = np.maximum(c - w + 1, 0)
        n_bytes += int((c + q - low + np.minimum(low, s)).sum()) * token
        p = np.repeat(c, q) + np.arange(tokens) - np.repeat(np.cumsum(q) - q, q)  # positions
        pairs = int((np.minimum(p + 1, w) + np.clip(p + 1 - w, 0, s)).sum())
    else:
        prefix, group = _groups(case)
        once = prefix[np.unique(group, return_index=True)[1]].sum()
        n_bytes += int((q + c - prefix).sum() + once) * token
        pairs = int((q * c + q * (q + 1) // 2).sum())
    return {"bytes": n_bytes, "flops": 4 * dim * heads * pairs}


# ---- from the definition, in 64 bits

def _pool_index(dim):
    """Where element d of token t lies inside a block of one KV head, of K and of V, [token][d]."""
    t, d = torch.arange(BLOCK, device=GPU)[:, None], torch.arange(dim, device=GPU)[None, :]
    return (d // 8 * BLOCK + t) * 8 + d % 8, d * BLOCK + (t % 4 + 8 * (t // 4 % 2) + 4 * (t // 8))


def _exact_rows(x, weight, position, state):
    """Complex numbers: a head's pairs times exp(i position frequency)."""
    case, x = state["case"], x.double()
    x = x / torch.sqrt(x.pow(2).sum(-1, keepdim=True) / x.shape[-1] + EPS) * weight.double()
    n = case["rotary"]
    order = torch.arange(n, device=GPU).view(2, -1).t() if case["pairs"] == "halves" else torch.arange(n, device=GPU).view(-1, 2)
    z = torch.complex(x[..., order[:, 0]], x[..., order[:, 1]]) * torch.polar(torch.ones_like(state["freq"]), torch.outer(position.double(), state["freq"]))[:, None]
    x[..., order[:, 0]], x[..., order[:, 1]] = z.real, z.imag
    return x


def exact(case, seed):
    state = prepare(case, seed)
    heads, kv_heads, dim = case["heads"], case["kv_heads"], case["head_dim"]
    k_at, v_at = _pool_index(dim)
    group = heads // kv_heads
    position = torch.cat([torch.arange(c, c + n, device=GPU) for n, c in zip(state["q_len"].tolist(), state["ctx"].tolist())])
    if case["kind"] == "rows":
        rows = state["rows"]
        q, k = _exact_rows(rows[:, :heads], state["q_weight"], position, state), _exact_rows(rows[:, heads:heads + kv_heads], state["k_weight"], position, state)
        if not case["append"]:
            return q, k
        ks, vs = state["k_pool"].double(), state["v_pool"].double()
        shapes, ks, vs = (ks.shape, vs.shape), ks.view(ks.shape[0], kv_heads, -1), vs.view(vs.shape[0], kv_heads, -1)
        at = 0
        for s, (n, c) in enumerate(zip(state["q_len"].tolist(), state["ctx"].tolist())):
            p = torch.arange(c, c + n, device=GPU)
            ids = torch.from_numpy(state["table"][s].astype(np.int64)).to(GPU)[p // BLOCK]
            head = torch.arange(kv_heads, device=GPU)[None, :, None]
            ks[ids[:, None, None], head, k_at[p % BLOCK][:, None, :]] = k[at:at + n]
            vs[ids[:, None, None], head, v_at[p % BLOCK][:, None, :]] = rows[at:at + n, heads + kv_heads:].double()
            at += n
        return q, ks.view(shapes[0]), vs.view(shapes[1])
    out = torch.zeros(state["out"].shape, dtype=torch.float64, device=GPU)
    window, sinks = case.get("window", 1 << 40), case.get("sinks", 0)
    for s, (n, c) in enumerate(zip(state["q_len"].tolist(), state["ctx"].tolist())):
        ids = torch.from_numpy(state["table"][s, :-(-(c + n) // BLOCK)].astype(np.int64)).to(GPU)
        a = int(state["q_start"][s])
        k, v = ((state[name].view(state[name].shape[0], kv_heads, -1)[ids][:, :, at].view(-1, kv_heads, BLOCK, dim).permute(1, 0, 2, 3).reshape(kv_heads, -1, dim)[:, :c + n].double())
                for name, at in (("k_pool", k_at), ("v_pool", v_at)))
        step = max(1, (1 << 27) // (heads * (c + n)))  # query rows at a time: a gibibyte of scores
        for r in range(0, n, step):
            m = min(step, n - r)
            q = state["q"][a + r:a + r + m].double().view(m, kv_heads, group, dim).permute(1, 2, 0, 3).reshape(kv_heads, group * m, dim)
            x = torch.bmm(q, k.transpose(1, 2).contiguous()).mul_(state["scale"]).view(kv_heads, group, m, c + n)
            key, p = torch.arange(c + n, device=GPU)[None, :], c + r + torch.arange(m, device=GPU)[:, None]
            hidden = (key > p) | ((key <= p - window) & (key >= sinks))
            x = torch.softmax(x.masked_fill_(hidden, -math.inf), -1).view(kv_heads, group * m, c + n)
            out[a + r:a + r + m] = torch.bmm(x, v).view(kv_heads, group, m, dim).permute(2, 0, 1, 3).reshape(m, heads, dim)
    return out
