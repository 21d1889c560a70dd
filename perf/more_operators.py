"""Timed cases of operators around the key-value cache that a serving iteration uses beside perf/operators.py's: norms of queries and keys on their way into
the cache, a cache held in 8 bits, requests that share a long prefix.

  norm       a batch's new keys and values into the pages; queries and keys are normed head by head and turned by their positions in the same pass
  store      the same without norms into pages of e4m3 values, and all that the requests have cached read back out of them
  attend     causal attention of a batch over pages of e4m3 values
  prefix     causal attention of requests that begin with the same tokens, held once
  iteration  requests behind a shared prefix, pages of e4m3 values: they get their pages, every layer norms, turns, appends and attends, and what the last
             one has stored of the new tokens is read back

A case is a dict of plain values.  Its fields:
  op, heads, kv_heads, dim, page, layers, dtype   as named; query heads, key-value heads, values of a head, tokens of a page, layers of a pass, type of queries and outputs
  e4m3      pages of 8-bit values
  shared    tokens of the prefix that all requests share
  tokens, ctx, spread   requests of one new token; tokens of their own cached before it: the median, and the deviation of its logarithm
  prompts, before       prompt lengths ("77,300", or "8x": eight drawn lognormally); tokens cached before each prompt
  pairs     which values of a head turn together: "halves" or "neighbours"
  per_head  each head has norm weights of its own
  batch     seed of the batch's structure (the values come from prepare()'s seed)

Pages of bf16 and fp32 values are one tensor [pages][layers][2][kv_heads][page * dim], in chunks of u values (16 bytes): the keys of a page lie
[dim / u][token][u values of dim], its values [page / u][dim][u tokens].  Pages of e4m3 values are bytes [pages][layers][2 * kv_heads * page * (dim + 1)]:
the same with u = 16, and behind the two halves of a layer an exponent for each half, head and token: the token's values times 2^(exponent - 127) are meant.
A token's exponent is the smallest, from 10 to 247, for which no finite value of its head is over 448.
"""
import math

import numpy as np
import torch

own = False

EPS = 1e-6


def _case(name, op, heads, kv_heads, dim, **kw):
    c = dict(name=name, op=op, heads=heads, kv_heads=kv_heads, dim=dim, page=64, layers=1, dtype="bf16", e4m3=op in ("store", "attend", "iteration"), shared=0,
             tokens=0, ctx=0, spread=0.0, prompts="", before=0, pairs="halves", per_head=False, batch=1)
    c.update(kw)
    return c


def listed():
    return [
        # one user's next token, a 13B model's heads: launches and latency only
        _case("norm_one_13b", "norm", 40, 40, 128, tokens=1, ctx=333),
        # eight packed prompts of 32 to 2048 tokens, grouped heads
        _case("norm_prompts_grouped", "norm", 32, 8, 128, prompts="8x"),
        # the decode batch of a 7B model: 64 new tokens stored, the requests' caches read back (they move to another place)
        _case("store_64_7b", "store", 32, 32, 128, tokens=64, ctx=60, spread=0.8),
        # 496 tokens beside four prompts of 512, grouped heads
        _case("store_stress_grouped", "store", 64, 8, 128, tokens=496, ctx=40, spread=0.8, prompts="512,512,512,512"),
        # one user, one token of a 13B model, an odd cache length: latency
        _case("token8_one_13b", "attend", 40, 40, 128, tokens=1, ctx=333),
        # a loaded server with grouped heads: 512 requests
        _case("token8_512_grouped", "attend", 32, 8, 128, tokens=512, ctx=1000, spread=0.8),
        # one request far into a long document: the cache's length is all there is to share out
        _case("token8_long_grouped", "attend", 64, 8, 128, tokens=1, ctx=131071),
        # one long prompt with grouped heads: the matrix units' rate
        _case("prompt8_long_grouped", "attend", 32, 8, 128, prompts="8192", page=128),
        # eight continuations of one prompt of a 13B model, each a few tokens on
        _case("prefix_8_13b", "prefix", 40, 40, 128, shared=1500, tokens=8, ctx=20, spread=0.4),
        # a loaded server: 256 requests behind the same instructions
        _case("prefix_256_grouped", "prefix", 32, 8, 128, shared=2000, tokens=256, ctx=300, spread=0.8),
        # 32 questions about one long document
        _case("prefix_32_long", "prefix", 64, 8, 128, shared=100000, tokens=32, ctx=50, spread=0.8),
        # an iteration of all of it: 100 requests and three new prompts behind the same instructions
        _case("iteration_grouped", "iteration", 32, 8, 128, layers=2, shared=1000, tokens=100, ctx=200, spread=0.8, prompts="40,7,150", per_head=True, batch=3),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    heads, kv = rng.choice([(32, 32), (40, 40), (32, 8), (64, 8), (40, 8), (8, 1), (12, 4), (4, 4), (6, 2), (28, 4)])
    dim = rng.choice([128, 128, 128, 64, 64, 256])
    kw = dict(page=rng.choice([32, 64, 64, 128, 256]), batch=rng.randrange(1, 1 << 20), pairs=rng.choice(["halves", "neighbours"]))
    op = rng.choice(["norm"] * 2 + ["store"] * 2 + ["tokens"] * 3 + ["prompts"] * 2 + ["prefix"] * 4 + ["iteration"] * 2)
    if op in ("norm", "store"):
        kw.update(tokens=_log(rng, 1, 512), ctx=_log(rng, 1, 200), spread=0.8, before=rng.choice([0, 5, 64]))
        kw.update(prompts=",".join(str(_log(rng, 1, 600)) for _ in range(rng.randrange(0, 5))))
        if op == "norm":
            kw.update(dtype=rng.choice(["bf16", "bf16", "f32"]), per_head=rng.random() < 0.3)
        return _case("", op, heads, kv, dim, **kw)
    if op == "tokens":
        n = _log(rng, 1, 512)
        kw.update(tokens=n, ctx=_log(rng, 1, min(100000, 4000000 // (n * kv))), spread=rng.choice([0.0, 0.4, 0.8]))
        return _case("", "attend", heads, kv, dim, **kw)
    if op == "prompts":
        most = rng.choice([1, 2, 4, 8])
        kw.update(prompts=",".join(str(_log(rng, 1, 6000 // most)) for _ in range(most)), before=rng.choice([0, 0, _log(rng, 1, 2000)]))
        return _case("", "attend", heads, kv, dim, **kw)
    n = _log(rng, 2, 256)
    kw.update(tokens=n, shared=_log(rng, 30, min(60000, 8000000 // (n * heads))), ctx=_log(rng, 1, min(2000, 1000000 // (n * kv))), spread=rng.choice([0.0, 0.4, 0.8]))
    if rng.random() < 0.4:
        kw.update(prompts=",".join(str(_log(rng, 1, 200)) for _ in range(rng.randrange(1, 4))), before=rng.choice([0, 9]))
    if op == "iteration":
        return _case("", op, heads, kv, dim, layers=2, per_head=rng.random() < 0.3, **kw)
    return _case("", op, heads, kv, dim, dtype=rng.choice(["bf16", "bf16", "bf16", "f32"]), **kw)


def _batch(case):
    """The structure of a batch: cached tokens and new tokens of each request (those with one new token first), the pages of each, copies (from, to) of the
    page in which the shared tokens end, how many pages there are."""
    rng = np.random.default_rng(case["batch"])
    page, shared = case["page"], case["shared"]
    ctx = np.maximum(1, np.rint(case["ctx"] * np.exp(np.clip(case["spread"] * rng.normal(size=case["tokens"]), -1.6, 1.6)))).astype(np.int64)
    if case["prompts"].endswith("x"):  # a count
        lens = np.clip(np.rint(np.exp(rng.normal(6.0, 0.8, int(case["prompts"][:-1])))), 32, 2048).astype(np.int64)
    else:
        lens = np.asarray([int(v) for v in case["prompts"].split(",") if v], np.int64)
    ctx = np.concatenate([ctx, np.full(len(lens), case["before"])]).astype(np.int64) + shared
    new = np.concatenate([np.ones(case["tokens"], np.int64), lens])
    # the shared tokens' pages come first; then what is cached comes page by page, a page for every request that needs one more: the pages of a request
    # lie apart.  A request that is the first time about to write into the shared page has a copy of it
    at = -(-shared // page)
    pages, copies = [list(range(at)) for _ in new], []
    for had, upto in [(had, np.minimum(ctx, had + page)) for had in range(shared, int(ctx.max()), page)] + [(None, ctx + new)]:
        for i in range(len(new)):
            begin = int(ctx[i]) if had is None else had
            if upto[i] <= begin:
                continue
            if begin % page and begin // page < shared // page + 1 and pages[i][-1] == shared // page and shared % page:
                copies.append((pages[i][-1], at))
                pages[i][-1] = at
                at += 1
            while len(pages[i]) * page < upto[i]:
                pages[i].append(at)
                at += 1
    table = np.zeros((len(new), max(len(p) for p in pages)), np.int64)
    for i, p in enumerate(pages):
        table[i, : len(p)] = p
    return ctx, new, -(-(ctx + new) // page), table, copies, at


def _layer_bytes(case):
    return 2 * case["kv_heads"] * case["page"] * (case["dim"] + 1)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    ctx, new, need, table, copies, n_pages = _batch(case)
    heads, kv, dim, page, layers = case["heads"], case["kv_heads"], case["dim"], case["page"], case["layers"]
    dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    T = int(new.sum())
    cuda = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    state = {"case": case}
    # a layer's keys, values and queries have the spread that projections of normed activations give them
    if case["e4m3"]:
        pages = torch.empty(n_pages, layers, _layer_bytes(case), dtype=torch.uint8, device="cuda")
        split = 2 * kv * page * dim
        for at in range(0, n_pages, 64):
            part = pages[at : at + 64]
            x = torch.randn(*part.shape[:2], split, generator=gen, device="cuda", dtype=torch.bfloat16)
            part[..., :split] = (x * 100).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
            part[..., split:] = torch.randint(119, 122, part[..., split:].shape, generator=gen, device="cuda", dtype=torch.uint8)
    else:
        pages = torch.empty(n_pages, layers, 2, kv, page * dim, dtype=dt, device="cuda")
        for at in range(0, n_pages, 64):
            pages[at : at + 64].normal_(generator=gen)
    if copies:
        src, dst = (cuda(v) for v in np.asarray(copies).T)
        pages[dst] = pages[src]
    state["pages"] = pages
    seg = np.repeat(np.arange(len(new)), new)
    pos = np.arange(T) - np.repeat(np.cumsum(new) - new, new) + ctx[seg]
    # the queries, keys and values of a token lie together, as one projection writes them
    state["qkv"] = torch.randn(layers, T, heads + 2 * kv, dim, generator=gen, device="cuda", dtype=dt)
    if case["op"] in ("norm", "iteration"):
        weights = lambda n: 1 + 0.2 * torch.randn(n, dim, generator=gen, device="cuda")  # noqa: E731
        state["norm"] = (weights(heads), weights(kv)) if case["per_head"] else (weights(1)[0], weights(1)[0])
    else:
        state["norm"] = (None, None)
    state["q"] = torch.empty(layers, T, heads, dim, device="cuda", dtype=dt)
    state["out"] = torch.empty(layers, T, heads, dim, device="cuda", dtype=dt)
    angle = torch.arange(int(pos.max()) + 1, device="cuda", dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(0, dim, 2, device="cuda", dtype=torch.float64) / dim)
    state["rope"] = torch.cat([angle.cos(), angle.sin()], 1).float()
    state["pos"], state["page"] = cuda(pos), cuda(table[seg, pos // page])
    # what is read back: everything that the requests have cached, or the new tokens
    if case["op"] == "store":
        n = ctx + new
        who = np.repeat(np.arange(len(n)), n)
        back = np.arange(int(n.sum())) - np.repeat(np.cumsum(n) - n, n)
    else:
        who, back = seg, pos
    state["back"] = cuda(table[who, back // page]), cuda(back % page)
    if case["op"] in ("store", "iteration"):
        state["read"] = torch.empty(2, len(back), kv, dim, device="cuda", dtype=dt)
    # for the plain form: the pages that all requests share, and requests with one new token, and prompts, each kind padded to its longest
    state["common"], state["groups"] = cuda(table[0, : case["shared"] // page]), []
    for part in (slice(0, case["tokens"]), slice(case["tokens"], None)):
        if len(new[part]):
            width, first = int(new[part].max()), np.cumsum(new)[part] - new[part]
            at = first[:, None] + np.minimum(np.arange(width), new[part][:, None] - 1)
            end = ctx[part][:, None] + np.minimum(np.arange(width), new[part][:, None] - 1)
            rows = seg[int(first[0]) : int(first[0] + new[part].sum())] - part.start, np.concatenate([np.arange(n) for n in new[part]])
            state["groups"].append((cuda(at), cuda(end), cuda(table[part, case["shared"] // page : need[part].max()]), cuda(rows[0]), cuda(rows[1])))
    if own:
        from paper_2411_17741_amd import binding as B
        from paper_2411_17741_amd.kv import KvCache

        cache = KvCache(layers, heads, kv, dim, n_pages, page_tokens=page, max_seqs=len(new) + 1, max_batch_tokens=T, max_batch_seqs=len(new),
                        dtype=B.LORA_BF16 if case["dtype"] == "bf16" else B.LORA_F32, pages=pages, e4m3=case["e4m3"])
        ids = np.arange(len(new), dtype=np.int64)
        if case["shared"]:
            cache.add(-1)
            cache.extend(-1, case["shared"])
            cache.fork(-1, ids)
        else:
            cache.add(ids)
        for had in range(case["shared"], int(ctx.max()), page):
            who = np.flatnonzero(ctx > had)
            cache.extend(who, np.minimum(page, ctx[who] - had))
        state["cache"], state["ids"], state["ctx"], state["new"] = cache, ids, ctx.astype(np.int32), new.astype(np.int32)
        state["offsets"] = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        plan = cache.batch(ids, state["offsets"], shared=case["op"] == "prefix")
        assert all(np.array_equal(cache.pages_of(i), table[i, : need[i]]) for i in range(len(new)))
        if case["op"] == "iteration":  # a batch of its own in every pass
            cache.batch_destroy(plan)
            cache.truncate(ids, state["ctx"])
        else:
            state["plan"] = plan
    return state


def _turn(x, rope, pos, pairs):
    c, s = rope[pos].unsqueeze(1).chunk(2, -1)
    if pairs == "halves":
        a, b = x.chunk(2, -1)
        return torch.cat([a * c - b * s, b * c + a * s], -1)
    a, b = x[..., 0::2], x[..., 1::2]
    return torch.stack([a * c - b * s, b * c + a * s], -1).flatten(-2)


def _to_e4m3(x):
    """x [T][heads][dim] -> bytes of the values, exponents"""
    fraction, power = torch.frexp(x.abs().amax(-1))
    power = torch.where(fraction == 0, -117, power - 9 + (fraction > 0.875)).clamp(-117, 120)
    return torch.ldexp(x, -power.unsqueeze(-1)).to(torch.float8_e4m3fn).view(torch.uint8), (power + 127).to(torch.uint8)


def _halves(state, layer):
    """Views of a layer's keys [pages][kv][dim / u][page][u] and values [pages][kv][page / u][dim][u], and of their exponents [pages][kv][page]"""
    case, pages = state["case"], state["pages"]
    kv, dim, page = case["kv_heads"], case["dim"], case["page"]
    u, n = 16 // pages.element_size(), kv * page * dim
    flat = pages[:, layer].view(len(pages), -1)
    k, v = flat[:, :n].unflatten(1, (kv, dim // u, page, u)), flat[:, n : 2 * n].unflatten(1, (kv, page // u, dim, u))
    if not case["e4m3"]:
        return k, v, None, None
    return k, v, flat[:, 2 * n : 2 * n + kv * page].unflatten(1, (kv, page)), flat[:, 2 * n + kv * page :].unflatten(1, (kv, page))


def _append(state, layer):
    case = state["case"]
    kv, dim, page, u = case["kv_heads"], case["dim"], case["page"], 16 // state["pages"].element_size()
    q, k, v = state["qkv"][layer].split([case["heads"], kv, kv], 1)
    # values beside a border between two 8-bit ones are told apart in 64 bits
    q, k, rope = (t.double() if case["e4m3"] else t.float() for t in (q, k, state["rope"]))
    if state["norm"][0] is not None:
        q = q * torch.rsqrt(q.square().mean(-1, keepdim=True) + EPS) * state["norm"][0]
        k = k * torch.rsqrt(k.square().mean(-1, keepdim=True) + EPS) * state["norm"][1]
    state["q"][layer] = _turn(q, rope, state["pos"], case["pairs"]).to(state["q"].dtype)
    k = _turn(k, rope, state["pos"], case["pairs"])
    at, keys, vals, key_exps, val_exps = state["pos"] % page, *_halves(state, layer)
    if case["e4m3"]:
        k, key_exps[state["page"], :, at] = _to_e4m3(k)
        v, val_exps[state["page"], :, at] = _to_e4m3(v.float())
    keys[state["page"], :, :, at] = k.to(keys.dtype).view(-1, kv, dim // u, u)
    vals[state["page"], :, at // u, :, at % u] = v


def _values(state, layer, table):
    """The keys [..., kv, dim, tokens] and values [..., kv, tokens, dim] of lists of pages [..., n] in fp32"""
    keys, vals, key_exps, val_exps = _halves(state, layer)
    k, v = keys[table], vals[table]
    if key_exps is not None:
        k, v = k.view(torch.float8_e4m3fn).float(), v.view(torch.float8_e4m3fn).float()
        k *= torch.exp2(key_exps[table].float() - 127)[..., None, :, None]
        v *= torch.exp2(val_exps[table].float() - 127).unflatten(-1, (-1, 16))[..., None, :]
    # [..., n, kv, ...] -> the list's pages one after the other
    return k.float().movedim(-5, -3).transpose(-1, -2).transpose(-3, -2).flatten(-4, -3).flatten(-2), v.float().movedim(-5, -4).transpose(-1, -2).flatten(-4, -2)


def _attend(state, layer, q, group):
    """The group's rows of the output: softmax(q . K / sqrt(dim)) . V over the tokens up to each row's own.  Shared pages are taken once for all requests."""
    case = state["case"]
    kv, dim, page, common = case["kv_heads"], case["dim"], case["page"], state["common"]
    at, end, table, rows, cols = group
    n, width = at.shape
    q = q[at].view(n, width, kv, -1, dim).float() * (1.0 / math.sqrt(dim))
    group = q.shape[3]
    k, v = _values(state, layer, table)
    own_q = q.permute(0, 2, 1, 3, 4).reshape(n * kv, -1, dim)
    s = torch.bmm(own_q, k.flatten(0, 1).contiguous()).view(n, kv, width, group, -1)
    s.masked_fill_((len(common) * page + torch.arange(s.shape[-1], device="cuda") > end[:, :, None])[:, None, :, None], float("-inf"))
    top = s.amax(-1, keepdim=True)
    if len(common):
        ck, cv = _values(state, layer, common)
        all_q = q.permute(2, 0, 1, 3, 4).reshape(kv, -1, dim)
        cs = torch.bmm(all_q, ck.contiguous()).view(kv, n, width, group, -1)
        top = torch.maximum(top, cs.amax(-1, keepdim=True).transpose(0, 1))
        cs.sub_(top.transpose(0, 1)).exp_()
    s.sub_(top).exp_()
    o = torch.bmm(s.view(n * kv, -1, s.shape[-1]), v.flatten(0, 1).contiguous()).view(n, kv, width, group, dim)
    weight = s.sum(-1, keepdim=True)
    if len(common):
        o += torch.bmm(cs.view(kv, -1, cs.shape[-1]), cv.contiguous()).view(kv, n, width, group, dim).transpose(0, 1)
        weight += cs.sum(-1, keepdim=True).transpose(0, 1)
    return (o / weight).permute(0, 2, 1, 3, 4).reshape(n, width, -1, dim)[rows, cols].to(state["out"].dtype)


def _attend_all(state, layer, q):
    state["out"][layer] = torch.cat([_attend(state, layer, q, g) for g in state["groups"]])


def _read(state, layer):
    keys, vals, key_exps, val_exps = _halves(state, layer)
    page, off = state["back"]
    k = keys[page, :, :, off].view(torch.float8_e4m3fn).float().flatten(2) * torch.exp2(key_exps[page, :, off].float() - 127)[..., None]
    v = vals[page, :, off // 16, :, off % 16].view(torch.float8_e4m3fn).float() * torch.exp2(val_exps[page, :, off].float() - 127)[..., None]
    state["read"][0], state["read"][1] = k.to(state["read"].dtype), v.to(state["read"].dtype)
    return state["read"]


def _run_plain(state):
    case = state["case"]
    if case["op"] == "norm":
        _append(state, 0)
        return state["q"], state["pages"]
    if case["op"] == "store":
        _append(state, 0)
        return state["q"], _read(state, 0)
    if case["op"] in ("attend", "prefix"):
        _attend_all(state, 0, state["qkv"][0, :, : case["heads"]])
        return state["out"]
    for layer in range(case["layers"]):
        _append(state, layer)
        _attend_all(state, layer, state["q"][layer])
    return state["out"], state["q"], _read(state, case["layers"] - 1)


def run(state):
    if not own:
        return _run_plain(state)
    case, cache, qkv = state["case"], state["cache"], state["qkv"]
    heads, kv, scale, neighbours = case["heads"], case["kv_heads"], 1.0 / math.sqrt(case["dim"]), case["pairs"] == "neighbours"
    q_norm, k_norm = state["norm"]
    if case["op"] in ("attend", "prefix"):
        cache.attend(state["plan"], 0, qkv[0, :, :heads], state["out"][0], scale)
        return state["out"]
    if case["op"] in ("norm", "store"):
        cache.append(state["plan"], 0, qkv[0, :, heads : heads + kv], qkv[0, :, heads + kv :], q=qkv[0, :, :heads], q_out=state["q"][0], rope=state["rope"],
                     neighbours=neighbours, q_norm=q_norm, k_norm=k_norm, eps=EPS)
        if case["op"] == "norm":
            return state["q"], state["pages"]
        cache.read(state["ids"], 0, state["read"][0], state["read"][1])
        return state["q"], state["read"]
    plan = cache.batch(state["ids"], state["offsets"], shared=True)
    for layer in range(case["layers"]):
        cache.append(plan, layer, qkv[layer, :, heads : heads + kv], qkv[layer, :, heads + kv :], q=qkv[layer, :, :heads], q_out=state["q"][layer],
                     rope=state["rope"], neighbours=neighbours, q_norm=q_norm, k_norm=k_norm, eps=EPS)
        cache.attend(plan, layer, state["q"][layer], state["out"][layer], scale)
    cache.batch_destroy(plan)
    cache.read(state["ids"], case["layers"] - 1, state["read"][0], state["read"][1], first=state["ctx"], n_tokens=state["new"])
    cache.truncate(state["ids"], state["ctx"])  # the same iteration comes again
    return state["out"], state["q"], state["read"]


def work(case):
    ctx, new, _need, _table, _copies, _n = _batch(case)
    e = 2 if case["dtype"] == "bf16" else 4
    heads, kv, dim, layers, shared = case["heads"], case["kv_heads"], case["dim"], case["layers"], case["shared"]
    row = 2 * kv * ((dim + 1) if case["e4m3"] else dim * e)  # a token's keys and values in the pages
    T, pairs = int(new.sum()), int((new * ctx + new * (new + 1) // 2).sum())
    append = T * ((2 * heads + 2 * kv) * dim * e + row + 4 * dim)  # rows read and written, the turns of each position
    back = lambda tokens: tokens * (row + 2 * kv * dim * e)  # noqa: E731
    attend = 2 * T * heads * dim * e + (shared + int((ctx + new - shared).sum())) * row
    flops = 4 * pairs * heads * dim
    if case["op"] == "norm":
        return {"bytes": append, "flops": 0}
    if case["op"] == "store":
        return {"bytes": append + back(int((ctx + new).sum())), "flops": 0}
    if case["op"] in ("attend", "prefix"):
        return {"bytes": attend, "flops": flops}
    return {"bytes": layers * (append + attend) + back(T), "flops": layers * flops}


def _nearest_e4m3(x):
    """x [..., dim] in 64 bits -> what its e4m3 values and their exponent stand for: 3 bits behind the leading one, from 2^-6 on; halves to even"""
    top = x.abs().amax(-1, keepdim=True)
    exponent = torch.ceil(torch.log2(top / 448).clamp(-200, 200)).clamp(-117, 120)
    exponent = torch.where(top > 448 * 2.0**exponent, exponent + 1, exponent)
    exponent = torch.where((exponent > -117) & (top <= 448 * 2.0 ** (exponent - 1)), exponent - 1, exponent)
    y = x / 2.0**exponent
    step = 2.0 ** (torch.floor(torch.log2(y.abs().clamp(min=2.0**-6))) - 3)
    return torch.round(y / step) * step * 2.0**exponent


def exact(case, seed):
    """From the definitions, request by request in 64 bits, on the values as they were drawn."""
    state = prepare(case, seed)
    pages, op = state["pages"], case["op"]
    ctx, new, need, table, _copies, _n = _batch(case)
    heads, kv, dim, page, layers = case["heads"], case["kv_heads"], case["dim"], case["page"], case["layers"]
    u, group, split = 16 // pages.element_size(), heads // kv, 2 * kv * page * dim
    qkv, rope = state["qkv"].double(), state["rope"].double()
    first = np.cumsum(new) - new
    want_q, want_out = state["q"].double().zero_(), state["out"].double().zero_()
    want_pages, read_k, read_v = pages.double() if op == "norm" else None, [], []
    half, d, head = torch.arange(dim // 2, device="cuda"), torch.arange(dim, device="cuda"), torch.arange(kv, device="cuda")[:, None]
    lo, hi = (half, half + dim // 2) if case["pairs"] == "halves" else (2 * half, 2 * half + 1)
    code = torch.arange(256, device="cuda")
    power, fraction = (code >> 3) & 15, (code & 7).double()
    meant = torch.where(power == 0, fraction * 2.0**-9, (1 + fraction / 8) * 2.0 ** (power.double() - 7)) * torch.where(code > 127, -1.0, 1.0)

    def cached(layer, part, where, off):
        """[tokens][kv][dim] of keys (part 0) or values out of the pages"""
        inner = ((d // u) * page + off[:, None]) * u + d % u if part == 0 else ((off // u)[:, None] * dim + d) * u + (off % u)[:, None]
        at = (part * kv + head) * page * dim + inner[:, None]
        x = pages[:, layer].reshape(len(pages), -1)
        if not case["e4m3"]:
            return x[where[:, None, None], at].double()
        exponent = x[where[:, None], split + (part * kv + head.T) * page + off[:, None]].double() - 127
        return meant[x[where[:, None, None], at].long()] * 2.0 ** exponent[..., None]

    for layer in range(layers):
        for i in range(len(new)):
            n, c = int(ctx[i] + new[i]), int(ctx[i])
            t = torch.arange(n, device="cuda")
            where, off = torch.from_numpy(table[i]).cuda()[t // page], t % page
            rows = slice(int(first[i]), int(first[i] + new[i]))
            q, k, v = qkv[layer, rows, :heads], qkv[layer, rows, heads : heads + kv], qkv[layer, rows, heads + kv :]
            if op not in ("attend", "prefix"):
                if state["norm"][0] is not None:
                    q = q / torch.sqrt((q * q).sum(-1, keepdim=True) / dim + EPS) * state["norm"][0].double()
                    k = k / torch.sqrt((k * k).sum(-1, keepdim=True) / dim + EPS) * state["norm"][1].double()
                cs, sn = rope[c:n, None, : dim // 2], rope[c:n, None, dim // 2 :]
                turned = [torch.empty_like(x) for x in (q, k)]
                for x, y in zip((q, k), turned):
                    y[..., lo], y[..., hi] = x[..., lo] * cs - x[..., hi] * sn, x[..., lo] * sn + x[..., hi] * cs
                q, k = turned
                want_q[layer, rows] = q
                if op == "norm":
                    for h in range(kv):
                        want_pages[:, 0, 0, h][where[c:, None], ((d // u) * page + off[c:, None]) * u + d % u] = k[:, h]
                        want_pages[:, 0, 1, h][where[c:, None], ((off[c:] // u)[:, None] * dim + d) * u + (off[c:] % u)[:, None]] = v[:, h]
                    continue
                k, v = _nearest_e4m3(k), _nearest_e4m3(v)
            keys, vals = cached(layer, 0, where, off), cached(layer, 1, where, off)
            if op in ("store", "iteration"):
                keys[c:], vals[c:] = k, v
                if layer == layers - 1:
                    read_k.append(keys if op == "store" else k)
                    read_v.append(vals if op == "store" else v)
                if op == "store":
                    continue
                q = q.to(state["q"].dtype).double()  # what is attended with was rounded once when it was stored
            seen = t <= (c + torch.arange(int(new[i]), device="cuda"))[:, None]
            for h in range(heads):
                s = (q[:, h] @ keys[:, h // group].T.contiguous() / math.sqrt(dim)).masked_fill(~seen, float("-inf"))
                want_out[layer, rows, h] = torch.softmax(s, -1) @ vals[:, h // group].contiguous()
    if op in ("attend", "prefix"):
        return want_out
    if op == "norm":
        return want_q, want_pages
    read = torch.stack([torch.cat(read_k), torch.cat(read_v)])
    return (want_q, read) if op == "store" else (want_out, want_q, read)
