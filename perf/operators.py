"""Timed cases of the key-value cache's operators: what the attention of one serving iteration asks of the library beside the adapters.

  attend   causal attention of a batch of requests over the paged cache: whole prompts ("prompt" cases: packed, of different lengths, with grouped heads)
           and one new token each ("token" cases: the cache read once, split over its length)
  append   a batch's new keys and values into the pages, keys and queries turned by their positions
  pages    requests forked (pages shared, copied when written), freed, the pages in use moved together
  mixed    an iteration: the requests get their pages, then every layer appends and attends

A case is a dict of plain values.  Its fields:
  op        "attend", "append", "pages" or "mixed"
  heads, kv_heads, dim, page, layers, dtype   query heads, key-value heads, values of a head, tokens of a page, layers of a pass
  tokens, ctx, spread   requests of one new token; cached tokens before it: the median, and the deviation of its logarithm
  prompts, before       prompt lengths ("77,300", or "8x": eight drawn lognormally); tokens cached before each prompt
  children, compact     (pages) forks of one request; whether half of them end and the pages in use are moved together
  pairs                 (append) which values of a head turn together: "halves" or "neighbours"
  batch     seed of the batch's structure (the values come from prepare()'s seed)

The cache is one tensor [pages][layers][2][kv_heads][page * dim].  In chunks of u values (16 bytes), the keys of a page lie
[dim / u][token][u values of dim] and its values [page / u][dim][u tokens].
"""
import math

import numpy as np
import torch

own = False


def _case(name, op, heads, kv_heads, dim, **kw):
    c = dict(name=name, op=op, heads=heads, kv_heads=kv_heads, dim=dim, page=64, layers=1, dtype="bf16", tokens=0, ctx=0, spread=0.0,
             prompts="", before=0, children=0, compact=False, pairs="halves", batch=1)
    c.update(kw)
    return c


def listed():
    return [
        # the full-precision configuration's batch, 16 tokens in prompts of 1, 3, 5 and 7, 256 wide: launches and latency only
        _case("prompt_tiny_f32", "attend", 4, 4, 64, dtype="f32", prompts="1,3,5,7", page=32),
        # the prefill batch of a 7B model: eight packed prompts of 32 to 2048 tokens
        _case("prompt_packed_7b", "attend", 32, 32, 128, prompts="8x"),
        # one long prompt with grouped heads: the matrix units' rate
        _case("prompt_long_grouped", "attend", 32, 8, 128, prompts="8192", page=128),
        # one user, one token of a 13B model, an odd cache length: latency
        _case("token_one_13b", "attend", 40, 40, 128, tokens=1, ctx=333),
        # the decode batch of a 7B model: 64 requests of different lengths
        _case("token_64_7b", "attend", 32, 32, 128, tokens=64, ctx=600, spread=0.8),
        # a loaded server with grouped heads: 512 requests
        _case("token_512_grouped", "attend", 32, 8, 128, tokens=512, ctx=1000, spread=0.8),
        # one request far into a long document: the cache's length is all there is to share out
        _case("token_long_grouped", "attend", 64, 8, 128, tokens=1, ctx=131071),
        # the decode batch's keys and values
        _case("append_64_7b", "append", 32, 32, 128, tokens=64, ctx=60, spread=0.8),
        # the stress batch of a 13B model: 496 tokens beside four prompts of 512
        _case("append_stress_13b", "append", 40, 40, 128, tokens=496, ctx=40, spread=0.8, prompts="512,512,512,512"),
        # four continuations of one 7B request: the page they share is copied for each as its next token comes
        _case("pages_fork_7b", "pages", 32, 32, 128, layers=32, ctx=300, children=4),
        # 64 continuations with grouped heads; half of them end, the pages of the others are moved together
        _case("pages_churn_grouped", "pages", 32, 8, 128, layers=32, ctx=1000, children=64, compact=True),
        # an iteration of the mixed configuration: 224 tokens and 32 prompts, some of them cached in part
        _case("mixed_7b", "mixed", 32, 32, 128, layers=2, tokens=224, ctx=400, spread=0.8, prompts="32x", before=96, batch=3),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    heads, kv = rng.choice([(32, 32), (40, 40), (32, 8), (64, 8), (40, 8), (8, 1), (12, 4), (4, 4), (6, 2), (28, 4)])
    dim = rng.choice([128, 128, 128, 64, 64, 256])
    kw = dict(page=rng.choice([32, 64, 64, 128]), batch=rng.randrange(1, 1 << 20))
    kind = rng.choice(["prompt"] * 4 + ["token"] * 4 + ["append"] * 2 + ["pages"] * 2 + ["mixed"] * 2 + ["f32"] * 2)
    if kind == "prompt":
        most = rng.choice([1, 2, 4, 8])
        kw.update(prompts=",".join(str(_log(rng, 1, 6000 // most)) for _ in range(most)), before=rng.choice([0, 0, _log(rng, 1, 2000)]))
        return _case("", "attend", heads, kv, dim, **kw)
    if kind == "token":
        n = _log(rng, 1, 512)
        kw.update(tokens=n, ctx=_log(rng, 1, min(100000, 4000000 // (n * kv))), spread=rng.choice([0.0, 0.4, 0.8]))
        return _case("", "attend", heads, kv, dim, **kw)
    if kind == "append":
        kw.update(tokens=_log(rng, 1, 512), ctx=_log(rng, 1, 200), spread=0.8, pairs=rng.choice(["halves", "neighbours"]))
        kw.update(prompts=",".join(str(_log(rng, 1, 600)) for _ in range(rng.randrange(0, 5))), before=rng.choice([0, 5, 64]))
        return _case("", "append", heads, kv, dim, **kw)
    if kind == "pages":
        layers = _log(rng, 2, max(2, 1024 * 128 // (kv * dim * 4)))
        kw.update(layers=min(32, layers), ctx=_log(rng, 40, 2000), children=_log(rng, 1, 64), compact=rng.random() < 0.5)
        return _case("", "pages", heads, kv, dim, **kw)
    if kind == "mixed":
        kw.update(tokens=_log(rng, 1, 200), ctx=_log(rng, 8, 600), spread=rng.choice([0.0, 0.8]), before=rng.choice([0, 0, 7, 300]))
        kw.update(prompts=",".join(str(_log(rng, 1, 1200)) for _ in range(rng.randrange(1, 9))), pairs=rng.choice(["halves", "neighbours"]))
        return _case("", "mixed", heads, kv, dim, layers=2, **kw)
    kw.update(dtype="f32", tokens=rng.choice([0, 1, 9]), ctx=_log(rng, 1, 3000), prompts=rng.choice(["5", "33,64", "300,1,77"]), before=rng.choice([0, 31]))
    return _case("", "mixed", heads, kv, rng.choice([64, 128]), **kw)


def _batch(case):
    """The structure of a batch: cached tokens and new tokens of each request (those with one new token first), and the pages of each."""
    rng = np.random.default_rng(case["batch"])
    if case["op"] == "pages":
        ctx, new = np.asarray([case["ctx"]]), np.asarray([0])
    else:
        ctx = np.maximum(1, np.rint(case["ctx"] * np.exp(np.clip(case["spread"] * rng.normal(size=case["tokens"]), -1.6, 1.6)))).astype(np.int64)
        if case["prompts"].endswith("x"):  # a count
            lens = np.clip(np.rint(np.exp(rng.normal(6.0, 0.8, int(case["prompts"][:-1])))), 32, 2048).astype(np.int64)
        else:
            lens = np.asarray([int(v) for v in case["prompts"].split(",") if v], np.int64)
        before = rng.choice([0, case["before"]], len(lens)) if case["op"] == "mixed" else np.full(len(lens), case["before"])
        ctx, new = np.concatenate([ctx, before]).astype(np.int64), np.concatenate([np.ones(case["tokens"], np.int64), lens])
    # what is cached came page by page, a page for every request that needed one more: the pages of a request lie apart.  The new
    # tokens' pages are taken as the batch is made, request by request
    had, need = -(-ctx // case["page"]), -(-(ctx + new) // case["page"])
    table, at = np.zeros((len(need), int(need.max())), np.int64), 0
    for k in range(int(had.max())):
        who = np.flatnonzero(had > k)
        table[who, k] = at + np.arange(len(who))
        at += len(who)
    for i in np.flatnonzero(need > had):
        table[i, had[i] : need[i]] = at + np.arange(need[i] - had[i])
        at += int(need[i] - had[i])
    return ctx, new, need, table, at


def _pages_moves(case, used):
    """(from, to) of the copies when every child gets its next token, and of those that move the pages in use together; the pages there have to be."""
    n, last = case["children"], (case["ctx"] // case["page"] if case["ctx"] % case["page"] else None)
    to = used + np.arange(n)
    first = (np.full(n if last is not None else 0, used - 1), to[: n if last is not None else 0])
    if not case["compact"]:
        return first, (to[:0], to[:0]), used + n
    kept = to[1::2]  # the others end
    held = used + len(kept)
    holes = to[0::2]
    return first, (kept[kept >= held], holes[holes < held]), used + n


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    ctx, new, need, table, n_pages = _batch(case)
    heads, kv, dim, page, layers = case["heads"], case["kv_heads"], case["dim"], case["page"], case["layers"]
    dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    T = int(new.sum())
    cuda = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    state = {"case": case}
    if case["op"] == "pages":
        first, second, n_pages = _pages_moves(case, n_pages)
        state["moves"] = [cuda(v) for v in first + second]
    # a layer's keys, values and queries have the spread that projections of normed activations give them
    pages = torch.empty(n_pages, layers, 2, kv, page * dim, dtype=dt, device="cuda")
    for at in range(0, n_pages, 64):
        pages[at : at + 64].normal_(generator=gen)
    state["pages"] = pages
    if case["op"] != "pages":
        seg = np.repeat(np.arange(len(new)), new)
        pos = np.arange(T) - np.repeat(np.cumsum(new) - new, new) + ctx[seg]
        # the queries, keys and values of a token lie together, as one projection writes them
        state["qkv"] = torch.randn(layers, T, heads + 2 * kv, dim, generator=gen, device="cuda", dtype=dt)
        state["q"] = torch.empty(layers, T, heads, dim, device="cuda", dtype=dt)
        state["out"] = torch.empty(layers, T, heads, dim, device="cuda", dtype=dt)
        angle = torch.arange(int(pos.max()) + 1, device="cuda", dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(0, dim, 2, device="cuda", dtype=torch.float64) / dim)
        state["rope"] = torch.cat([angle.cos(), angle.sin()], 1).float()
        state["pos"], state["page"] = cuda(pos), cuda(table[seg, pos // page])
        # for the plain form: requests with one new token, and prompts, each kind padded to its longest
        state["groups"] = []
        for part in (slice(0, case["tokens"]), slice(case["tokens"], None)):
            if len(new[part]):
                width, first = int(new[part].max()), np.cumsum(new)[part] - new[part]
                at = first[:, None] + np.minimum(np.arange(width), new[part][:, None] - 1)
                end = ctx[part][:, None] + np.minimum(np.arange(width), new[part][:, None] - 1)
                rows = seg[int(first[0]) : int(first[0] + new[part].sum())] - part.start, np.concatenate([np.arange(n) for n in new[part]])
                state["groups"].append((cuda(at), cuda(end), cuda(table[part, : need[part].max()]), cuda(rows[0]), cuda(rows[1])))
    if own:
        from paper_2411_17741_amd import binding as B
        from paper_2411_17741_amd.kv import KvCache

        more = case["children"]
        cache = KvCache(layers, heads, kv, dim, n_pages, page_tokens=page, max_seqs=len(new) + more, max_batch_tokens=max(1, T, more),
                        max_batch_seqs=len(new) + more, dtype=B.LORA_BF16 if case["dtype"] == "bf16" else B.LORA_F32, pages=pages)
        cache.add(np.arange(len(new)))
        for at in range(0, int(ctx.max()), page):
            who = np.flatnonzero(ctx > at)
            cache.extend(who, np.minimum(page, ctx[who] - at))
        state["cache"], state["ids"] = cache, np.arange(len(new), dtype=np.int64)
        state["offsets"] = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        state["ctx"] = ctx
        plan = cache.batch(state["ids"], state["offsets"])
        assert all(np.array_equal(cache.pages_of(i), table[i, : need[i]]) for i in range(len(new)))
        if case["op"] in ("attend", "append"):
            state["plan"] = plan
        else:  # a batch of its own in every pass
            cache.batch_destroy(plan)
            cache.truncate(state["ids"], ctx)
    return state


def _turn(x, rope, pos, pairs):
    c, s = rope[pos].unsqueeze(1).chunk(2, -1)
    x = x.float()
    if pairs == "halves":
        a, b = x.chunk(2, -1)
        return torch.cat([a * c - b * s, b * c + a * s], -1)
    a, b = x[..., 0::2], x[..., 1::2]
    return torch.stack([a * c - b * s, b * c + a * s], -1).flatten(-2)


def _append(state, layer):
    case, pages = state["case"], state["pages"]
    kv, dim, page, u = case["kv_heads"], case["dim"], case["page"], 16 // pages.element_size()
    q, k, v = state["qkv"][layer].split([case["heads"], kv, kv], 1)
    state["q"][layer] = _turn(q, state["rope"], state["pos"], case["pairs"]).to(pages.dtype)
    k = _turn(k, state["rope"], state["pos"], case["pairs"]).to(pages.dtype)
    at = state["pos"] % page
    pages[:, layer, 0].view(-1, kv, dim // u, page, u)[state["page"], :, :, at] = k.view(-1, kv, dim // u, u)
    pages[:, layer, 1].view(-1, kv, page // u, dim, u)[state["page"], :, at // u, :, at % u] = v


def _attend(state, layer, q, group):
    """The group's rows of the output: softmax(q . K / sqrt(dim)) . V over the tokens up to each row's own."""
    case, pages = state["case"], state["pages"]
    kv, dim, page, u = case["kv_heads"], case["dim"], case["page"], 16 // pages.element_size()
    at, end, table, rows, cols = group
    n, width = at.shape
    x = pages[table, layer]
    k = x[:, :, 0].view(n, -1, kv, dim // u, page, u).permute(0, 2, 3, 5, 1, 4).reshape(n * kv, dim, -1).float()
    v = x[:, :, 1].view(n, -1, kv, page // u, dim, u).permute(0, 2, 1, 3, 5, 4).reshape(n * kv, -1, dim).float()
    q = q[at].view(n, width, kv, -1, dim).permute(0, 2, 1, 3, 4).reshape(n * kv, -1, dim).float()
    s = torch.bmm(q, k).mul_(1.0 / math.sqrt(dim)).view(n, kv, width, -1, k.shape[-1])
    s.masked_fill_((torch.arange(k.shape[-1], device="cuda") > end[:, :, None])[:, None, :, None], float("-inf"))
    s.sub_(s.amax(-1, keepdim=True)).exp_()
    o = torch.bmm(s.view(n * kv, -1, k.shape[-1]), v).view(n, kv, width, -1, dim) / s.sum(-1, keepdim=True)
    return o.permute(0, 2, 1, 3, 4).reshape(n, width, -1, dim)[rows, cols].to(pages.dtype)


def _attend_all(state, layer, q):
    state["out"][layer] = torch.cat([_attend(state, layer, q, g) for g in state["groups"]])


def _run_plain(state):
    case = state["case"]
    if case["op"] == "pages":
        a, b, c, d = state["moves"]
        state["pages"][b] = state["pages"][a]
        state["pages"][d] = state["pages"][c]
        return state["pages"]
    if case["op"] == "append":
        _append(state, 0)
        return state["q"], state["pages"]
    if case["op"] == "attend":
        _attend_all(state, 0, state["qkv"][0, :, : case["heads"]])
        return state["out"]
    for layer in range(case["layers"]):
        _append(state, layer)
        _attend_all(state, layer, state["q"][layer])
    return state["out"], state["q"], state["pages"]


def run(state):
    if not own:
        return _run_plain(state)
    case, cache = state["case"], state["cache"]
    heads, kv, scale = case["heads"], case["kv_heads"], 1.0 / math.sqrt(case["dim"])
    if case["op"] == "pages":
        children = np.arange(1, case["children"] + 1, dtype=np.int64)
        cache.fork(0, children)
        cache.batch_destroy(cache.batch(children, np.arange(case["children"] + 1, dtype=np.int32)))
        if case["compact"]:
            cache.free(children[0::2])
            cache.compact()
            children = children[1::2]
        cache.free(children)
        return state["pages"]
    qkv, pairs = state["qkv"], case["pairs"] == "neighbours"
    if case["op"] == "append":
        cache.append(state["plan"], 0, qkv[0, :, heads : heads + kv], qkv[0, :, heads + kv :], q=qkv[0, :, :heads], q_out=state["q"][0], rope=state["rope"], neighbours=pairs)
        return state["q"], state["pages"]
    if case["op"] == "attend":
        cache.attend(state["plan"], 0, qkv[0, :, :heads], state["out"][0], scale)
        return state["out"]
    plan = cache.batch(state["ids"], state["offsets"])
    for layer in range(case["layers"]):
        cache.append(plan, layer, qkv[layer, :, heads : heads + kv], qkv[layer, :, heads + kv :], q=qkv[layer, :, :heads], q_out=state["q"][layer],
                     rope=state["rope"], neighbours=pairs)
        cache.attend(plan, layer, state["q"][layer], state["out"][layer], scale)
    cache.batch_destroy(plan)
    cache.truncate(state["ids"], state["ctx"])  # the same iteration comes again
    return state["out"], state["q"], state["pages"]


def work(case):
    ctx, new, _need, _table, used = _batch(case)
    e = 2 if case["dtype"] == "bf16" else 4
    heads, kv, dim, layers = case["heads"], case["kv_heads"], case["dim"], case["layers"]
    if case["op"] == "pages":  # every page that is copied, read and written
        first, second, _n = _pages_moves(case, used)
        return {"bytes": max(1, 2 * (len(first[0]) + len(second[0])) * layers * 2 * kv * case["page"] * dim * e), "flops": 0}
    T, seen, pairs = int(new.sum()), int((ctx + new).sum()), int((new * ctx + new * (new + 1) // 2).sum())
    append = 2 * T * (heads + 2 * kv) * dim * e + 4 * dim * T  # rows read and written, the turns of each position
    attend = 2 * T * heads * dim * e + 2 * seen * kv * dim * e
    n_bytes = {"append": append, "attend": attend, "mixed": append + attend}[case["op"]]
    return {"bytes": layers * n_bytes, "flops": 0 if case["op"] == "append" else layers * 4 * pairs * heads * dim}


def exact(case, seed):
    """From the definitions, request by request and head by head in 64 bits, on the values as they were drawn."""
    state = prepare(case, seed)
    pages = state["pages"]
    ctx, new, need, table, _n = _batch(case)
    if case["op"] == "pages":
        want, lists = pages.double(), [m.tolist() for m in state["moves"]]
        for a, b in list(zip(*lists[:2])) + list(zip(*lists[2:])):
            want[b] = want[a]
        return want
    heads, kv, dim, page, layers = case["heads"], case["kv_heads"], case["dim"], case["page"], case["layers"]
    u, group = 16 // pages.element_size(), heads // kv
    qkv, rope = state["qkv"].double(), state["rope"].double()
    first = np.cumsum(new) - new
    want_q, want_out, want_pages = state["q"].double().zero_(), state["out"].double().zero_(), pages.double() if case["op"] != "attend" else None
    half = torch.arange(dim // 2, device="cuda")
    lo, hi = (half, half + dim // 2) if case["pairs"] == "halves" else (2 * half, 2 * half + 1)
    for layer in range(layers):
        for i in range(len(new)):
            n = int(ctx[i] + new[i])
            t = torch.arange(n, device="cuda")
            where, off = torch.from_numpy(table[i]).cuda()[t // page], t % page
            # [token][kv head][dim] out of the pages
            d = torch.arange(dim, device="cuda")
            keys = pages[:, layer, 0][where[:, None, None], torch.arange(kv, device="cuda")[:, None], ((d // u) * page + off[:, None])[:, None] * u + d % u].double()
            vals = pages[:, layer, 1][where[:, None, None], torch.arange(kv, device="cuda")[:, None], ((off // u)[:, None] * dim + d)[:, None] * u + (off % u)[:, None, None]].double()
            rows = slice(int(first[i]), int(first[i] + new[i]))
            q, k, v = qkv[layer, rows, :heads], qkv[layer, rows, heads : heads + kv], qkv[layer, rows, heads + kv :]
            if case["op"] != "attend":
                c, s = rope[int(ctx[i]) : n, None, : dim // 2], rope[int(ctx[i]) : n, None, dim // 2 :]
                q, k = q.clone(), k.clone()
                for x in (q, k):
                    a, b = x[..., lo], x[..., hi]
                    x[..., lo], x[..., hi] = a * c - b * s, a * s + b * c
                want_q[layer, rows] = q
                new_t = t[int(ctx[i]) :]
                for h in range(kv):
                    want_pages[:, layer, 0, h][where[new_t][:, None], ((d // u) * page + off[new_t][:, None]) * u + d % u] = k[:, h]
                    want_pages[:, layer, 1, h][where[new_t][:, None], ((off[new_t] // u)[:, None] * dim + d) * u + (off[new_t] % u)[:, None]] = v[:, h]
                # what is read back was rounded once when it was stored
                q, k = q.to(pages.dtype).double(), k.to(pages.dtype).double()
                keys[int(ctx[i]) :], vals[int(ctx[i]) :] = k, v
            if case["op"] == "append":
                continue
            seen = t <= (int(ctx[i]) + torch.arange(int(new[i]), device="cuda"))[:, None]
            for h in range(heads):
                s = (q[:, h] @ keys[:, h // group].T.contiguous() / math.sqrt(dim)).masked_fill(~seen, float("-inf"))
                want_out[layer, rows, h] = torch.softmax(s, -1) @ vals[:, h // group].contiguous()
    return want_out if case["op"] == "attend" else (want_q, want_pages) if case["op"] == "append" else (want_out, want_q, want_pages)
