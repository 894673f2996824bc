"""The operators of the 8-bit KV cache, as cases that a timing program can run.

The cache holds K and V as E4M3 bytes with one power-of-two scale for each block of 16 tokens and KV head (K and V
apart).  A case is one pass of one batch, one layer, on tensors that are already on the GPU:

  "append"     the new rows of a batch are quantised into the cache as they are written
  "read"       whole requests are read back, in the type that attention computes in
  "attention"  mixed attention of a batch over the cache, the new rows in it already
  "step"       both in one call, as a serving loop has it for each layer

A batch is given by `chunk` (a prompt chunk as "tokens@offset", or nothing) and by `decodes` running requests whose
context lengths follow from `context` ("lognormal mean sigma low high" or "uniform low high") and `lengths` (the seed
of the draw); the seed given to prepare() makes tensors and block tables.

Layouts (B = 16 tokens to a block, D = head_dim):
  k pool  [blocks][kv heads][D/16][B][16]           bytes of d = 16 i + l of token t at [i][t][l]
  v pool  [blocks][kv heads][2][B/4][16][D/32][4]   bytes of d = 32 c + 16 h + j of token 4 g + t at [h][g][j][c][t]
  scales  [blocks][kv heads][2]                     exponent + 127 of the K block's and of the V block's scale
"""
import math

import numpy as np
import torch

own = False

BLOCK = 16  # tokens per KV block
GPU = "cuda:0"
E4M3_MAX = 448.0
# The exponents a scale may have: as wide as keeps what the bytes stand for exact and finite in the type of q.
EXPONENTS = {"bf16": (-117, 120), "fp16": (-15, 8)}


def _case(name, kind, heads, kv_heads, head_dim, dtype, chunk, decodes, context, lengths, gain=1.0):
    return {"name": name, "kind": kind, "heads": heads, "kv_heads": kv_heads, "head_dim": head_dim, "dtype": dtype, "chunk": chunk,
            "decodes": decodes, "context": context, "lengths": lengths, "gain": gain}


def listed():
    return [
        # A handful of chat requests, a token each: the smallest call of a decode loop.
        _case("append_few", "append", 32, 8, 128, "bf16", "", 8, "lognormal 1024 0.8 64 8192", 1),
        # A full instance: a token of every request, each into a block of its own that has older tokens in it.
        _case("append_decodes", "append", 40, 8, 128, "fp16", "", 512, "lognormal 1024 1.0 16 16384", 2),
        # A long prompt arrives, a few decodes ride along.
        _case("append_prompt", "append", 32, 8, 128, "bf16", "8192@0", 4, "uniform 500 1500", 3),
        # One request leaves for an instance whose cache has 16 bits.
        _case("read_one", "read", 40, 8, 128, "fp16", "", 1, "uniform 1500 1600", 4),
        # Sixteen leave at once.
        _case("read_batch", "read", 32, 8, 128, "bf16", "", 16, "lognormal 2048 1.0 16 16384", 5),
        # The smallest mixed batch: a short first chunk and four decodes of a small model.
        _case("attention_tiny", "attention", 8, 8, 64, "bf16", "64@0", 4, "uniform 37 128", 6),
        # The prefill-heavy kind of instance: a large chunk in the middle of a prompt, some decodes.
        _case("attention_prefill_heavy", "attention", 32, 8, 128, "bf16", "2048@4096", 64, "lognormal 1024 0.8 64 8192", 7),
        # The decode-heavy kind: a small chunk at an odd offset, many decodes; five query heads to a KV head, IEEE half.
        _case("attention_decode_heavy", "attention", 40, 8, 128, "fp16", "256@1234", 256, "uniform 512 4096", 8, 2.0),
        # Decode only at low load: launches and the chain of latencies.
        _case("step_few", "step", 32, 8, 128, "bf16", "", 8, "lognormal 1024 0.8 64 8192", 9),
        # Two users with long documents: few sequences, long contexts.
        _case("step_long_context", "step", 64, 8, 128, "bf16", "", 2, "uniform 16384 32768", 10),
        # Decode only, at the number of requests that a cache of half the size lets in.
        _case("step_pure_decode", "step", 32, 8, 128, "bf16", "", 512, "uniform 1000 3000", 11),
        # The largest call: a long document's later half in one chunk, with decodes of other documents.
        _case("step_long_prompt", "step", 64, 8, 128, "bf16", "8192@8192", 8, "uniform 1024 16384", 12),
    ]


def draw(rng):
    """One more case of the same ranges: any operator, any load from one decode to a full instance, any chunk from none to the largest."""
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    heads, kv_heads = rng.choice([(32, 8), (32, 8), (40, 8), (64, 8), (8, 8), (32, 32), (16, 2)])
    kind = rng.choice(["append", "read", "attention", "attention", "step", "step"])
    case = _case("", kind, heads, kv_heads, rng.choice([128, 128, 64]), rng.choice(["bf16", "bf16", "fp16"]), "", 0, "", rng.randrange(1 << 20),
                 rng.choice([1.0, 2.0, 3.0]))
    del case["name"]
    mean = log(64, 8192)
    case["context"] = rng.choice(["lognormal %d 0.8 16 %d" % (mean, 2 * mean), "uniform %d %d" % (max(1, mean // 4), 2 * mean)])
    budget = 1.0e9 if kind != "read" else 2.0e8  # elements of K of the decodes, each as long as the longest may be
    case["decodes"] = max(1, min(log(1, 512), int(budget / (2 * mean * kv_heads * case["head_dim"]))))
    if kind != "read" and rng.random() < 0.7:
        tokens, offset = log(2, 8192), rng.choice([0, log(1, 16384)])
        # no more work than the largest listed chunk
        while heads * tokens * (offset + tokens) > 64 * 8192 * 16384 * (1.0 if case["head_dim"] == 128 else 0.5):
            tokens, offset = (tokens + 1) // 2, offset // 2
        case["chunk"] = "%d@%d" % (max(2, tokens), offset)
        if rng.random() < 0.2:
            case["decodes"], case["context"] = 0, "uniform 1 1"
    return case


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
    return q_len, ctx


def prepare(case, seed):
    q_len, ctx = _lengths(case)
    dtype = torch.bfloat16 if case["dtype"] == "bf16" else torch.float16
    heads, kv_heads, dim = case["heads"], case["kv_heads"], case["head_dim"]
    rs = np.random.RandomState((seed * 2 + 1) % (1 << 31))
    gen = torch.Generator(device=GPU).manual_seed(seed)
    kv_len = q_len + ctx
    pages = -(-kv_len // BLOCK)
    q_start = np.concatenate([[0], np.cumsum(q_len)]).astype(np.int32)
    tokens = int(q_start[-1])
    # block tables over a pool with a quarter of its blocks to spare, the blocks scattered as a running allocator leaves them
    blocks = int(pages.sum()) + max(4, int(pages.sum()) // 4)
    ids = rs.permutation(blocks).astype(np.int32)
    table = np.zeros((len(kv_len), int(pages.max())), np.int32)
    table[np.arange(table.shape[1])[None, :] < pages[:, None]] = ids[:int(pages.sum())]

    def normal(gain, *shape):
        return torch.empty(shape, dtype=dtype, device=GPU).normal_(0.0, gain, generator=gen)

    def cached():  # what appended rows of a normal distribution leave, and leftovers of earlier requests in the free slots
        x = torch.empty((blocks, kv_heads, BLOCK * dim), dtype=torch.float32, device=GPU).normal_(0.0, 128.0, generator=gen)
        return x.clamp_(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)

    state = {"case": case, "k": cached(), "v": cached(), "scale": 1.0 / math.sqrt(dim), "q_len": q_len, "ctx": ctx, "table": table, "q_start": q_start}
    state["scales"] = torch.randint(119, 122, (blocks, kv_heads, 2), dtype=torch.uint8, device=GPU, generator=gen)
    if case["kind"] == "read":
        state["k_out"] = torch.zeros((int(kv_len.sum()), kv_heads, dim), dtype=dtype, device=GPU)
        state["v_out"] = torch.zeros_like(state["k_out"])
    else:
        state["k_new"], state["v_new"] = normal(1.0, tokens, kv_heads, dim), normal(1.0, tokens, kv_heads, dim)
    if case["kind"] in ("attention", "step"):
        state["q"] = normal(case["gain"], tokens, heads, dim)
        state["out"] = torch.zeros((tokens, heads, dim), dtype=dtype, device=GPU)
    if own:
        import paper_2508_01989_amd as tc
        pool = tc.make_kvq_pool(heads, kv_heads, dim, blocks, state["k"], state["v"], state["scales"],
                                dtype=tc.TC_BF16 if case["dtype"] == "bf16" else tc.TC_FP16)
        state["pool"], state["plan"] = pool, tc.Plan(pool, q_start, ctx.astype(np.int32), table)
        state["workspace"] = torch.empty(max(16, state["plan"].workspace_bytes), dtype=torch.uint8, device=GPU)
    # the same batch as the index tensors that a program without the library keeps for its iteration
    seq = np.repeat(np.arange(len(q_len)), q_len)
    at = np.arange(tokens) - q_start[seq] + ctx[seq]  # position of every new row
    block = table[seq, at // BLOCK]
    written, segment = np.unique(block, return_inverse=True)
    first = np.full(len(written), BLOCK, np.int64)
    np.minimum.at(first, segment, at % BLOCK)
    state["segment"], state["slot"] = torch.from_numpy(segment).to(GPU), torch.from_numpy(at % BLOCK).to(GPU)
    state["written"], state["older"] = torch.from_numpy(written.astype(np.int64)).to(GPU), torch.from_numpy(first).to(GPU)
    state["table_gpu"] = torch.from_numpy(table.astype(np.int64)).to(GPU)
    state["kv_len_gpu"] = torch.from_numpy(kv_len).to(GPU)
    return state


# ---- the plain form: elementary operations in 32 bits

def _blocks(cache, ids):
    return cache.view(torch.uint8)[ids].view(torch.float8_e4m3fn)


def _values(k8, v8):
    """The bytes of blocks [n][kv heads][...] as numbers, float32 [n][kv heads][token][d]."""
    n, heads, dim = k8.shape[0], k8.shape[1], k8[0, 0].numel() // BLOCK
    k = k8.view(n, heads, dim // 16, BLOCK, 16).float().permute(0, 1, 3, 2, 4).reshape(n, heads, BLOCK, dim)
    v = v8.view(n, heads, 2, BLOCK // 4, 16, dim // 32, 4).float().permute(0, 1, 3, 6, 5, 2, 4).reshape(n, heads, BLOCK, dim)
    return k, v


def _bytes(k, v):
    n, heads, _, dim = k.shape
    k8 = k.to(torch.float8_e4m3fn).view(n, heads, BLOCK, dim // 16, 16).permute(0, 1, 3, 2, 4).reshape(n, heads, BLOCK * dim)
    v8 = v.to(torch.float8_e4m3fn).view(n, heads, BLOCK // 4, 4, dim // 32, 2, 16).permute(0, 1, 5, 2, 6, 4, 3).reshape(n, heads, BLOCK * dim)
    return k8, v8


def _append(state):
    low, high = EXPONENTS[state["case"]["dtype"]]
    written, segment, slot, older = state["written"], state["segment"], state["slot"], state["older"]
    new = torch.stack([state["k_new"], state["v_new"]], -2).float()  # [tokens][kv heads][2][d]
    shape = (len(written), new.shape[1], 2)
    amax = torch.zeros(shape, device=GPU).scatter_reduce(0, segment[:, None, None].expand(-1, shape[1], 2), new.abs().amax(-1), "amax")
    # the smallest e with amax <= 448 * 2^e: amax / 448 = m * 2^e with m in (1/2, 1]
    m, e = torch.frexp(amax.double() / E4M3_MAX)
    e = torch.where(amax > 0, e - (m == 0.5).int(), torch.full_like(e, low)).clamp(low, high)
    has_older = (older > 0)[:, None, None]
    before = state["scales"][written].int() - 127
    e = torch.where(has_older, torch.maximum(e, before), e)
    top = torch.where(e == high, 240.0, E4M3_MAX)  # 256 * 2^high is no finite number of the type of q
    old = torch.stack(_values(_blocks(state["k"], written), _blocks(state["v"], written)), 2)  # [written][kv heads][2][token][d]
    shrink = torch.ldexp(torch.ones_like(top), torch.where(has_older, before - e, torch.zeros_like(e)))[..., None, None]
    is_older = torch.arange(BLOCK, device=GPU)[None, :] < older[:, None]
    rows = torch.where(is_older[:, None, None, :, None], old * shrink, old)
    fresh = torch.ldexp(new, -e[segment][..., None]).clamp(-top[segment][..., None], top[segment][..., None])
    rows[segment, :, :, slot] = fresh
    k8, v8 = _bytes(rows[:, :, 0], rows[:, :, 1])
    state["k"].view(torch.uint8)[written] = k8.view(torch.uint8)
    state["v"].view(torch.uint8)[written] = v8.view(torch.uint8)
    state["scales"][written] = (e + 127).to(torch.uint8)


def _cached(state, first, last):
    """K and V of the sequences [first, last), float32 [n][kv heads][token][d], each padded to the longest."""
    longest = int(-(-(state["q_len"] + state["ctx"])[first:last].max() // BLOCK))
    ids = state["table_gpu"][first:last, :longest].reshape(-1)
    scale = torch.ldexp(torch.ones((), device=GPU), state["scales"][ids].int() - 127)
    k, v = _values(_blocks(state["k"], ids), _blocks(state["v"], ids))
    k, v = k * scale[:, :, 0, None, None], v * scale[:, :, 1, None, None]
    k, v = (x.view(last - first, longest, -1, BLOCK, x.shape[-1]).transpose(1, 2).flatten(2, 3) for x in (k, v))
    return k, v


def _attend(state, first, last):
    """Rows of the sequences [first, last), all of them with as many new tokens as the first has."""
    case, rows = state["case"], int(state["q_len"][first])
    heads, kv_heads, dim, n = case["heads"], case["kv_heads"], case["head_dim"], last - first
    a = int(state["q_start"][first])
    q = state["q"][a:a + n * rows].float().view(n, rows, kv_heads, heads // kv_heads, dim).permute(0, 2, 3, 1, 4).reshape(n, kv_heads, -1, dim)
    k, v = _cached(state, first, last)
    sees = state["kv_len_gpu"][first:last, None] - rows + 1 + torch.arange(rows, device=GPU)  # keys of every row
    hidden = torch.arange(k.shape[2], device=GPU) >= sees[..., None]  # [n][rows][key]
    x = torch.matmul(q * state["scale"], k.transpose(2, 3)).view(n, heads, rows, -1)
    x = x.masked_fill_(hidden[:, None], -math.inf)
    x = x.sub_(x.amax(-1, keepdim=True)).exp_().view(n, kv_heads, -1, k.shape[2])
    v = v * (~hidden[:, -1, None, :, None])  # what lies behind the last token may be anything
    o = torch.matmul(x, v) / x.sum(-1, keepdim=True)
    o = o.view(n, kv_heads, heads // kv_heads, rows, dim).permute(0, 3, 1, 2, 4).reshape(n * rows, heads, dim)
    state["out"][a:a + n * rows] = o.to(state["out"].dtype)


def _plain(state):
    kind, chunks = state["case"]["kind"], int(state["q_len"][0] > 1)
    if kind in ("append", "step"):
        _append(state)
    if kind == "read":
        k, v = _cached(state, 0, len(state["q_len"]))
        real = torch.arange(k.shape[2], device=GPU) < state["kv_len_gpu"][:, None]
        state["k_out"].copy_(k.transpose(1, 2)[real])
        state["v_out"].copy_(v.transpose(1, 2)[real])
    if kind in ("attention", "step"):
        if chunks:
            _attend(state, 0, 1)
        if len(state["q_len"]) > chunks:
            _attend(state, chunks, len(state["q_len"]))


def run(state):
    kind = state["case"]["kind"]
    if own:
        import paper_2508_01989_amd as tc
        plan, pool = state["plan"], state["pool"]
        if kind == "append":
            tc.tc_kvq_append(plan, pool, state["k_new"], state["v_new"])
        elif kind == "read":
            tc.tc_kvq_read(plan, pool, -1, state["k_out"], state["v_out"])
        elif kind == "attention":
            tc.tc_kvq_mixed_attention(plan, pool, state["q"], state["out"], state["scale"], state["workspace"])
        else:
            tc.tc_kvq_mixed_attention_append(plan, pool, state["q"], state["k_new"], state["v_new"], state["out"], state["scale"], state["workspace"])
    else:
        _plain(state)
    if kind == "read":
        return state["k_out"], state["v_out"]
    if kind == "attention":
        return state["out"]
    # the cache is E4M3 numbers beside their exponents, which are whole numbers
    cache = (state["k"], state["v"], state["scales"])
    return cache if kind == "append" else (state["out"], *cache)


def work(case):
    q, c = _lengths(case)
    heads, kv_heads, dim = case["heads"], case["kv_heads"], case["head_dim"]
    kv = q + c
    cached_token, row = 2 * kv_heads * dim, 4 * kv_heads * dim  # bytes of K and V of a token, in the cache and as new rows
    pages = -(-kv // BLOCK)
    scales = 2 * kv_heads
    append = int(q.sum()) * (row + cached_token) + int((pages - c // BLOCK).sum()) * scales
    if case["kind"] == "append":
        return {"bytes": append, "flops": 0}
    if case["kind"] == "read":
        return {"bytes": int(kv.sum()) * (cached_token + row) + int(pages.sum()) * scales, "flops": 0}
    pairs = int((q * c + q * (q + 1) // 2).sum())
    n_bytes = int(kv.sum()) * cached_token + int(pages.sum()) * scales + 2 * int(q.sum()) * heads * dim * 2
    if case["kind"] == "step":  # the new rows are quantised on the way: read as they come, stored, not read again
        n_bytes += append - int(q.sum()) * cached_token
    return {"bytes": n_bytes, "flops": 4 * dim * heads * pairs}


# ---- from the definition, in 64 bits

def _nearest_e4m3(x):
    """The E4M3 number next to x (at most 448), ties to the even one: steps of 2^-3 of the power of two below, of 2^-9 at least."""
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp_min(2.0 ** -6))) - 3)
    return torch.round(x / step) * step


def _places(dim):
    """Where the byte of (token, d) lies inside a block of one KV head, K and V, in the order [token][d]."""
    t, d = torch.arange(BLOCK, device=GPU)[:, None], torch.arange(dim, device=GPU)[None, :]
    k_at = (d // 16 * BLOCK + t) * 16 + d % 16
    v_at = (((d // 16 % 2 * 4 + t // 4) * 16 + d % 16) * (dim // 32) + d // 32) * 4 + t % 4
    return k_at.reshape(-1), v_at.reshape(-1)


def exact(case, seed):
    state = prepare(case, seed)
    heads, kv_heads, dim = case["heads"], case["kv_heads"], case["head_dim"]
    k_at, v_at = _places(dim)
    group = heads // kv_heads
    low, high = EXPONENTS[case["dtype"]]
    k_cache, v_cache = (state[x] for x in "kv")
    if case["kind"] in ("append", "step"):
        k_cache, v_cache = k_cache.double(), v_cache.double()
    outs = {"k": [], "v": []}
    out = torch.zeros(state["out"].shape, dtype=torch.float64, device=GPU) if "out" in state else None
    exponents = state["scales"].double() - 127
    for s, (n, c) in enumerate(zip(state["q_len"].tolist(), state["ctx"].tolist())):
        ids = torch.from_numpy(state["table"][s, :-(-(c + n) // BLOCK)].astype(np.int64)).to(GPU)
        a = int(state["q_start"][s])
        kv = {}
        for x, (name, at, cache) in enumerate((("k", k_at, k_cache), ("v", v_at, v_cache))):
            e = exponents[ids][:, :, x]  # [page][kv head]
            mine = (cache if cache.dtype == torch.float64 else cache.view(torch.uint8))[ids][:, :, at]
            mine = (mine if cache.dtype == torch.float64 else mine.view(torch.float8_e4m3fn).double()).view(-1, kv_heads, BLOCK, dim)
            if case["kind"] in ("append", "step"):
                p0, rows = c // BLOCK, torch.full((len(ids) * BLOCK, kv_heads, dim), math.nan, dtype=torch.float64, device=GPU)
                rows[c:c + n] = state[name + "_new"][a:a + n].double()
                rows = rows.view(-1, BLOCK, kv_heads, dim).permute(0, 2, 1, 3)[p0:]  # NaN: no new row in this slot
                fresh = ~rows.isnan()
                need = torch.ceil(torch.log2(rows.nan_to_num(0.0).abs().amax((2, 3)) / E4M3_MAX)).clamp(low, high)
                e = e.clone()
                before = e[p0:].clone()
                e[p0:] = need
                if c % BLOCK:
                    e[p0] = torch.maximum(need[0], before[0])
                limit = torch.where(e[p0:] == high, 240.0, E4M3_MAX)[:, :, None, None]
                scaled = torch.maximum(torch.minimum(rows * torch.exp2(-e[p0:])[:, :, None, None], limit), -limit)
                tail = torch.where(fresh, _nearest_e4m3(scaled.nan_to_num(0.0)), mine[p0:])
                if c % BLOCK:  # the rows that were there, at the block's exponent of now
                    tail[0, :, :c % BLOCK] = _nearest_e4m3(mine[p0, :, :c % BLOCK] * torch.exp2(before[0] - e[p0])[:, None, None])
                mine[p0:] = tail
                block = torch.empty_like(cache[ids[p0:]])
                block[:, :, at] = tail.reshape(len(ids) - p0, kv_heads, -1)
                cache[ids[p0:]] = block
            kv[name] = (mine * torch.exp2(e)[:, :, None, None]).permute(0, 2, 1, 3).reshape(-1, kv_heads, dim)[:c + n]
            if case["kind"] == "read":
                outs[name].append(kv[name])
        if out is None:
            continue
        k, v = kv["k"].permute(1, 2, 0).contiguous(), kv["v"].permute(1, 0, 2).contiguous()
        rows = max(1, (1 << 27) // (heads * (c + n)))  # query rows at a time: a gibibyte of scores
        for r in range(0, n, rows):
            m = min(rows, n - r)
            q = state["q"][a + r:a + r + m].double().view(m, kv_heads, group, dim).permute(1, 2, 0, 3).reshape(kv_heads, group * m, dim)
            x = torch.bmm(q, k).mul_(state["scale"]).view(kv_heads, group, m, c + n)
            later = torch.arange(c + n, device=GPU)[None, :] > c + r + torch.arange(m, device=GPU)[:, None]
            x = torch.softmax(x.masked_fill_(later, -math.inf), -1).view(kv_heads, group * m, c + n)
            out[a + r:a + r + m] = torch.bmm(x, v).view(kv_heads, group, m, dim).permute(2, 0, 1, 3).reshape(m, heads, dim)
    if case["kind"] == "read":
        return torch.cat(outs["k"]), torch.cat(outs["v"])
    if case["kind"] == "attention":
        return out
    return (k_cache, v_cache, None) if case["kind"] == "append" else (out, k_cache, v_cache, None)
