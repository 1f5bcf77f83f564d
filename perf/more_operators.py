"""What the operators around the 4-bit cache are measured on: the plan (pages and slots of a batch's new tokens), the write
(keys and values rounded to 4 bits into their pages) and the attention that reads the pages.

Every case is a batch of B requests whose rows lie [B][R][...], a request using the first of its R rows; a request runs one of T
paths, path t uses the leading heads.  A cached token has, for every head, groups of 64 elements with a scale and a middle:
value = middle + scale * (code - 8).
"""
import math

import torch

own = False
_contexts = {}
DEV = "cuda"
G64 = 64          # elements that share a scale
BLOCK = 16        # tokens that lie together in a page


# ------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # plan: one step of a serving batch, a new token for every request; latency of one call
        dict(name="plan 64 tokens", op="plan", B=64, R=1, page=16, top=4096, full=True, ends=False),
        # plan: prompts of different lengths arrive, some requests end
        dict(name="plan 128 prompts", op="plan", B=128, R=2048, page=16, top=8192, full=False, ends=True),
        # write: one new token of a ViT-B-wide stream; latency of one call
        dict(name="write 1 token", op="write", B=1, R=1, H=12, D=64, group=1, T=1, page=16, full=True),
        # write: the tokens of a batch of images of slimmable ViT-B, some cropped, gathered by path
        dict(name="write 128 x 197, paths", op="write", B=128, R=197, H=12, D=64, group=1, T=4, page=64, full=False),
        # write: long prompts, shared heads
        dict(name="write 4 x 4096", op="write", B=4, R=4096, H=8, D=128, group=4, T=1, page=16, full=True),
        # attention: one new token of one request behind an image's tokens; latency of one call
        dict(name="attend 1 token", op="attend", B=1, R=1, H=12, D=64, group=1, T=1, page=16, top=197, full=True, prompt=False, window=0),
        # attention: one step of a serving batch, ragged lengths, shared heads
        dict(name="attend 64 tokens", op="attend", B=64, R=1, H=8, D=128, group=4, T=1, page=16, top=8192, full=True, prompt=False, window=0),
        # attention: one step of many short requests on mixed paths, every head its own
        dict(name="attend 256 tokens, paths", op="attend", B=256, R=1, H=12, D=64, group=1, T=4, page=64, top=1999, full=True, prompt=False,
             window=0),
        # attention: one token behind a very long text
        dict(name="attend 131071 back", op="attend", B=1, R=1, H=8, D=128, group=8, T=1, page=256, top=131071, full=True, prompt=False,
             window=0),
        # attention: a few tokens checked at once for every request, only the last 1000 seen
        dict(name="attend 24 x 5, window", op="attend", B=24, R=5, H=16, D=64, group=2, T=2, page=32, top=6001, full=False, prompt=False,
             window=1000),
        # attention: a piece of a prompt behind what is cached already
        dict(name="attend 2 x 512 more", op="attend", B=2, R=512, H=8, D=128, group=4, T=1, page=64, top=9999, full=False, prompt=False,
             window=0),
        # attention: whole prompts
        dict(name="attend 2 x 4096", op="attend", B=2, R=4096, H=8, D=128, group=4, T=1, page=16, top=4096, full=True, prompt=True, window=0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["plan", "write", "attend", "attend"])
    page = rng.choice([16, 16, 32, 48, 64, 128, 256])
    if op == "plan":
        R = rng.choice([1, 1, 4, _log(rng, 1, 4096)])
        B = max(1, min(_log(rng, 1, 2048), 262144 // R))
        return dict(op=op, B=B, R=R, page=page, top=R + _log(rng, 16, 32768), full=rng.random() < 0.5, ends=rng.random() < 0.5)
    D = rng.choice([64, 64, 128, 128])
    group = rng.choice([1, 1, 2, 3, 4, 5, 8, 16])
    H = max(1, min(_log(rng, 1, 32), 64 // group))
    T = rng.choice([1, 1, 2, 3, 4, 8])
    if op == "write":
        R = rng.choice([1, 1, 7, 49, 196, 197, _log(rng, 1, 4096)])
        B = max(1, min(512, _log(rng, 1, 16384) // R, 4 * 4096 * 8 * 128 * 6 // (R * H * D * (group + 2))))
        return dict(op=op, B=B, R=R, H=H, D=D, group=group, T=T, page=page, full=rng.random() < 0.5)
    prompt = rng.random() < 0.25
    most = 4096 * 4096 * 32 * 128                            # pairs * heads * width of the largest listed case
    R = rng.choice([1, 1, 1, 2, 5, 8, _log(rng, 1, 2048)])
    top = max(R, 64, _log(rng, 64, 131072) if rng.random() < 0.5 else _log(rng, 64, 4096))
    top = min(top, 48 * 8192 * 8 * 128 // (H * D))
    R = max(1, min(R, top, most // (top * H * group * D)))
    if prompt:
        R = top = min(_log(rng, 16, 4096), math.isqrt(2 * most // (H * group * D)))
    pairs = most // (R * (top // 2 if prompt else top) * H * group * D)
    B = max(1, min(256, _log(rng, 1, 256), pairs, 48 * 8192 * 8 * 128 // (top * H * D)))
    return dict(op=op, B=B, R=R, H=H, D=D, group=group, T=T, page=page, top=top, full=rng.random() < 0.5, prompt=prompt,
                window=rng.choice([0, 0, 0, _log(rng, 1, top)]))


def _heads(H, T):
    """Path t of T uses the leading half .. whole of the heads."""
    return [max(1, H * (T + t + 1) // (2 * T)) if t + 1 < T else H for t in range(T)]


def _spread(i, lo, hi):
    """Length of request i, ragged over lo .. hi; fixed, so that the work of a case does not depend on the seed."""
    return lo + (hi - lo) * ((i * 7919 + 1234) % 1000) // 999 if hi > lo else hi


def _lengths(case):
    """(tokens held before the call, new tokens) of every request."""
    B, R = case["B"], case["R"]
    new = [R if case["full"] else _spread(i, 1, R) for i in range(B)]
    if case["op"] == "write" or case.get("prompt"):
        return [0] * B, new
    if B == 1:
        return [case["top"] - new[0]], new
    return [_spread(i + 17, (case["top"] - R) // 2, case["top"] - R) for i in range(B)], new


def _ends(case):
    """Requests of a plan that end instead of growing: every ninth."""
    return [case["ends"] and i % 9 == 4 for i in range(case["B"])]


def _visible(case, held, n):
    """(keys that some query of a request sees, pairs of query and key)."""
    w = case["window"] or held + n
    per = [min(held + r + 1, w) for r in range(n)] if n <= 4096 else None
    first = max(0, held + 1 - w)
    return held + n - first, sum(per)


def work(case):
    B, R = case["B"], case["R"]
    held, new = _lengths(case)
    if case["op"] == "plan":
        page, ends = case["page"], _ends(case)
        pages = sum(-(-(h + n) // page) - -(-h // page) for h, n, e in zip(held, new, ends) if not e)
        back = sum(-(-h // page) for h, e in zip(held, ends) if e)
        return {"bytes": 16 * B + 4 * B * R + 8 * pages + 8 * back, "flops": B * R}
    D, g = case["D"], case["group"]
    heads = _heads(case["H"], case["T"])
    token = 72 * D // G64                                    # bytes of a cached token in one head
    total = {"bytes": 0, "flops": 0}
    for i in range(B):
        h = heads[i % case["T"]]
        if case["op"] == "write":
            total["bytes"] += new[i] * h * (4 * D + token + 4 * D) + 4 * new[i]
            total["flops"] += new[i] * h * 2 * D * 8
        else:
            keys, pairs = _visible(case, held[i], new[i])
            total["bytes"] += h * (keys * token + new[i] * g * 4 * D) + 4 * (keys // case["page"])
            total["flops"] += h * g * pairs * 4 * D
    return total


# ------------------------------------------------------------------------------------------ inputs
def _page_bytes(case):
    """A page of one head: blocks of 16 tokens, each [k codes][k scales][v codes][v scales]."""
    n = case["D"] // G64
    return case["page"] // BLOCK, 2 * n * BLOCK * (G64 // 2 + 4)


def _round_groups(x):
    """x [..., D] fp32 -> codes, scale, middle; codes [..., D / 64, 64], the others [..., D / 64]."""
    v = x.unflatten(-1, (-1, G64))
    lo, hi = v.amin(-1), v.amax(-1)
    fifteenth = torch.full((), 1.0 / 15, device=x.device)
    s = (hi * fifteenth - lo * fifteenth).to(torch.bfloat16).float()
    s = torch.where(s < 2.0 ** -126, 0.0, s)
    z = (2 * (0.5 * lo + 4 * s)).to(torch.bfloat16).float()
    inv = torch.where(s > 0, torch.ones_like(s) / torch.where(s > 0, s, 1.0), 0.0)
    code = (torch.round((v - z.unsqueeze(-1)) * inv.unsqueeze(-1)) + 8).clamp(0, 15)
    return code.to(torch.uint8), s, z


def _pack(k, v):
    """Rounded keys and values [P, H, page, D] -> bytes [P, H, page / 16, block]."""
    parts = []
    for x in (k, v):
        code, s, z = _round_groups(x)
        code = code[..., 0::2] | (code[..., 1::2] << 4)                                  # [P, H, page, n, 32]
        pair = torch.stack([s, z], -1).to(torch.bfloat16).contiguous().view(torch.uint8)   # [P, H, page, n, 4]
        for t in (code, pair):
            t = t.unflatten(2, (-1, BLOCK)).transpose(3, 4)                              # [P, H, blocks, n, 16, .]
            parts.append(t.flatten(3))
    return torch.cat(parts, -1)


def _unpack(pages, D):
    """The reverse of _pack, as values: bytes [..., blocks, block] -> k, v [..., tokens, D] fp32."""
    n, out, at = D // G64, [], 0
    for _ in range(2):
        code = pages[..., at:at + n * BLOCK * 32].unflatten(-1, (n, BLOCK, 32))
        at += n * BLOCK * 32
        pair = pages[..., at:at + n * BLOCK * 4].contiguous().view(torch.bfloat16).unflatten(-1, (n, BLOCK, 2)).float()
        at += n * BLOCK * 4
        c = torch.stack([code & 15, code >> 4], -1).flatten(-2).float() - 8
        v = c * pair[..., :1] + pair[..., 1:]                                            # [..., blocks, n, 16, 64]
        out.append(v.transpose(-3, -2).flatten(-2).flatten(-3, -2))
    return out


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    B, R, page = case["B"], case["R"], case["page"]
    held, new = _lengths(case)
    s = {"case": case}

    def ints(v):
        return torch.tensor(v, dtype=torch.int32, device=DEV)

    whole = [-(-(h + n) // page) for h, n in zip(held, new)]
    have = [-(-h // page) for h in held]
    if case["op"] == "plan":
        ends = _ends(case)
        want = [n if not e else -1 for n, e in zip(new, ends)]
        need = sum(w - h for w, h, e in zip(whole, have, ends) if not e)
        n_pages = sum(have) + need + 7
        s["max_pages"], s["n_pages"] = max(whole), n_pages
        s["held"], s["new"] = ints(held), ints(want)
        order = torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32)
        s["table"] = _table(order, have, s["max_pages"])
        free = n_pages - sum(have)
        first = int(torch.randint(0, n_pages, (1,), generator=g, device=DEV))
        s["pool"] = torch.full((n_pages,), -1, dtype=torch.int32, device=DEV)
        s["pool"][(torch.arange(free, device=DEV) + first) % n_pages] = order[sum(have):]
        s["state"] = ints([first, free])
        for k, shape in (("lengths", (B,)), ("placed", (B,)), ("slots", (B, R)), ("state_out", (2,))):
            s[k] = torch.zeros(shape, dtype=torch.int32, device=DEV)
        if own:
            _keep_descriptor(s)
        return s

    H, D, T = case["H"], case["D"], case["T"]
    s["idx"] = (torch.arange(B, device=DEV) % T)                                         # path of every request
    order = torch.sort(s["idx"], stable=True).indices
    counts = torch.bincount(s["idx"], minlength=T)
    s["perm"] = order.to(torch.int32)
    s["inv"] = torch.argsort(order).to(torch.int32)
    s["counts"] = counts.to(torch.int32)
    s["offsets"] = torch.cat([counts.new_zeros(1), counts.cumsum(0)]).to(torch.int32)
    s["heads"] = _heads(H, T)
    s["max_pages"], s["n_pages"] = max(whole), sum(whole) + 3
    s["table"] = _table(torch.randperm(s["n_pages"], generator=g, device=DEV).to(torch.int32), whole, s["max_pages"])
    s["lengths"], s["placed"] = ints([h + n for h, n in zip(held, new)]), ints(new)
    # slots of the new rows, -1 where a request has no such row
    at = ints(held).view(-1, 1) + torch.arange(R, device=DEV, dtype=torch.int32)
    page_of = torch.gather(s["table"].long(), 1, (at // page).clamp(max=s["max_pages"] - 1).long())
    live = torch.arange(R, device=DEV) < s["placed"].view(-1, 1)
    s["slots"] = torch.where(live, page_of * page + at % page, -1).to(torch.int32)
    s["live"] = live
    # rows as the QKV layer leaves them: queries and values around zero, keys with channels that have an offset
    vectors = case["group"] + 2
    shift = torch.zeros(H, vectors, D, device=DEV)
    shift[:, -2] = 2 * torch.randn(H, D, generator=g, device=DEV) * (torch.rand(H, D, generator=g, device=DEV) < 0.1)
    x = torch.randn(B, R, H, vectors, D, generator=g, device=DEV)
    s["qkv"] = (x + shift).to(torch.bfloat16).view(B, R, H * vectors * D)
    del x
    blocks, block = _page_bytes(case)
    if case["op"] == "write":
        s["pages"] = torch.zeros(s["n_pages"], H, blocks, block, dtype=torch.uint8, device=DEV)
        s["values"] = torch.zeros(B, R, H * 2 * D, dtype=torch.bfloat16, device=DEV)
    else:
        s["pages"] = torch.empty(s["n_pages"], H, blocks, block, dtype=torch.uint8, device=DEV)
        step = max(1, (1 << 25) // (H * page * D))
        for p in range(0, s["n_pages"], step):
            m = min(step, s["n_pages"] - p)
            k = torch.randn(m, H, page, D, generator=g, device=DEV) + shift[:, -2].unsqueeze(1)
            v = torch.randn(m, H, page, D, generator=g, device=DEV)
            s["pages"][p:p + m] = _pack(k, v)
        s["out"] = torch.zeros(B, R, H * case["group"] * D, dtype=torch.bfloat16, device=DEV)
    if own:
        _keep_descriptor(s)
    return s


def _table(order, count, width):
    """Pages dealt out in the given order: request i has the next count[i]; -1 behind them."""
    n = torch.tensor(count, device=DEV)
    cols = torch.arange(width, device=DEV)
    at = (n.cumsum(0) - n).view(-1, 1) + cols
    return torch.where(cols < n.view(-1, 1), order[at.clamp(max=len(order) - 1)], -1).to(torch.int32)


def _keep_descriptor(s):
    """What a user's program keeps beside its cache: the context, the routing, the descriptor, the workspace."""
    import paper_2109_10060_b200 as dsn
    dev = torch.cuda.current_device()
    if dev not in _contexts:
        _contexts[dev] = dsn.Context(dev)
    s["ctx"] = _contexts[dev]
    case = s["case"]
    if case["op"] == "plan":
        s["d"] = dsn.make_cache_desc(case["R"], 1, 64, [1], page=case["page"], n_pages=s["n_pages"], max_pages=s["max_pages"])
        s["c"] = dsn.make_cache(table=s["table"], lengths=s["held"], placed=s["placed"], slots=s["slots"], pool=s["pool"],
                                pool_state=s["state"])
        return
    s["r"] = dsn.make_routing(case["B"], case["T"], s["counts"], s["offsets"], s["perm"], s["inv"])
    s["d"] = dsn.make_cache_desc(case["R"], case["H"], case["D"], s["heads"], group=case["group"], page=case["page"], n_pages=s["n_pages"],
                                 max_pages=s["max_pages"], order=dsn.GROUPED, window=case.get("window", 0))
    s["c"] = dsn.make_cache(pages=s["pages"], table=s["table"], lengths=s["lengths"], placed=s["placed"], slots=s["slots"])
    if case["op"] == "attend":
        n = dsn.dsn_cache_attention_q4_workspace_bytes(s["d"], case["B"])
        s["ws"] = torch.empty(n, dtype=torch.uint8, device=DEV) if n else None


# ------------------------------------------------------------------------------------------ one pass
def run(s):
    op = s["case"]["op"]
    if own:
        import paper_2109_10060_b200 as dsn
        if op == "plan":
            dsn.dsn_cache_plan(s["ctx"], s["d"], s["c"], s["case"]["B"], s["new"], lengths_out=s["lengths"], pool_state_out=s["state_out"])
            return {k: s[k] for k in ("placed", "lengths", "table", "slots", "pool", "state_out")}
        if op == "write":
            dsn.dsn_cache_write_q4(s["ctx"], s["d"], s["c"], s["r"], s["qkv"], values=s["values"])
            return {"values": s["values"], "pages": s["pages"]}
        dsn.dsn_cache_attention_q4(s["ctx"], s["d"], s["c"], s["r"], s["qkv"], s["out"], s["ws"])
        return {"out": s["out"]}
    return {"plan": _plan, "write": _write, "attend": _attend}[op](s)


def _plan(s):
    case, page, N = s["case"], s["case"]["page"], s["n_pages"]
    held, new = s["held"].long(), s["new"].long()
    end = new < 0
    have = (held + page - 1) // page
    need = torch.where(end, 0, (held + new + page - 1) // page - have)
    up_to = need.cumsum(0)
    first, free = s["state"].long()
    ok = ~end & ((need == 0) | (up_to <= free)) & (have + need <= s["max_pages"])
    take = torch.where(ok, need, 0)
    placed = torch.where(ok, new, 0)
    lengths = torch.where(end, 0, held + placed)
    cols = torch.arange(s["max_pages"], device=DEV)
    j = cols - have.view(-1, 1)                                           # which of a request's new pages a column is
    fresh = (j >= 0) & (j < take.view(-1, 1))
    at = (first + (up_to - need).view(-1, 1) + j) % N
    table = torch.where(fresh, s["pool"][at].long(), s["table"].long())
    back = end.view(-1, 1) & (cols < have.view(-1, 1))                    # pages that return, request by request
    returned = s["table"][back]
    pool = s["pool"].clone()
    pool[(first + free + torch.arange(len(returned), device=DEV)) % N] = returned
    pos = held.view(-1, 1) + torch.arange(case["R"], device=DEV)
    page_of = torch.gather(table, 1, (pos // page).clamp(max=s["max_pages"] - 1))
    slots = torch.where(pos < lengths.view(-1, 1), page_of * page + pos % page, -1)
    used = take.sum()
    state = torch.stack([(first + used) % N, free - used + len(returned)])
    out = dict(placed=placed, lengths=lengths, table=table, slots=slots, pool=pool, state_out=state)
    return {k: v.to(torch.int32) for k, v in out.items()}


def _rows_by_request(s, x):
    """Rows lie by grouped position; returns them by request."""
    return x[s["inv"].long()]


def _write(s):
    case = s["case"]
    B, R, H, D = case["B"], case["R"], case["H"], case["D"]
    kv = s["qkv"].view(B, R, H, case["group"] + 2, D)[..., -2:, :].float()
    path = s["idx"][s["perm"].long()]                                     # as the rows lie
    live = s["live"][s["perm"].long()].view(B, R, 1) & (torch.arange(H, device=DEV) < torch.tensor(s["heads"], device=DEV)[path].view(B, 1, 1))
    code, sc, z = _round_groups(kv)
    val = ((code.float() - 8) * sc.unsqueeze(-1) + z.unsqueeze(-1)).flatten(-2)
    values = torch.where(live.view(B, R, H, 1, 1), val, 0.0).to(torch.bfloat16).view(B, R, H * 2 * D)
    # bytes of a token in its block: [k codes][k scales][v codes][v scales], each by group, then by token
    n = D // G64
    blocks, block = _page_bytes(case)
    pages = torch.zeros(s["n_pages"], H, blocks, block, dtype=torch.uint8, device=DEV)
    b, r, h = live.nonzero(as_tuple=True)
    slot = s["slots"][s["perm"].long()][b, r].long()
    page, tok = slot // case["page"], slot % case["page"]
    code = code[..., 0::2] | (code[..., 1::2] << 4)
    pair = torch.stack([sc, z], -1).to(torch.bfloat16).view(torch.uint8)
    half = block // 2
    for which in range(2):
        for j in range(n):
            c0 = which * half + (j * BLOCK + tok % BLOCK) * 32
            pages[page.unsqueeze(1), h.unsqueeze(1), (tok // BLOCK).unsqueeze(1), c0.unsqueeze(1) + torch.arange(32, device=DEV)] = \
                code[b, r, h, which, j]
            p0 = which * half + n * BLOCK * 32 + (j * BLOCK + tok % BLOCK) * 4
            pages[page.unsqueeze(1), h.unsqueeze(1), (tok // BLOCK).unsqueeze(1), p0.unsqueeze(1) + torch.arange(4, device=DEV)] = \
                pair[b, r, h, which, j]
    return {"values": values, "pages": pages}


def _attend(s):
    case = s["case"]
    B, R, H, D, g, page = (case[k] for k in ("B", "R", "H", "D", "group", "page"))
    held, new = _lengths(case)
    w = case["window"]
    out = torch.zeros_like(s["out"]).view(B, R, H, g, D)
    inv = torch.argsort(torch.tensor([i % case["T"] for i in range(B)]), stable=True).tolist()
    at = {sample: p for p, sample in enumerate(inv)}                      # where a request's rows lie
    q = s["qkv"].view(B, R, H, g + 2, D)
    for i in range(B):
        n, L, h = new[i], held[i] + new[i], s["heads"][i % case["T"]]
        lo = max(0, held[i] + 1 - w) // page if w else 0
        hi = -(-L // page)
        pages = s["pages"][s["table"][i, lo:hi].long(), :h].transpose(0, 1)     # [h, pages, blocks, block]
        k, v = _unpack(pages, D)
        k, v = (x.flatten(1, -2)[:, : L - lo * page] for x in (k, v))
        pos = held[i] + torch.arange(n, device=DEV)
        key = lo * page + torch.arange(k.shape[1], device=DEV)
        seen = key <= pos.view(-1, 1)
        if w:
            seen &= key > pos.view(-1, 1) - w
        step = max(1, (1 << 28) // (n * g * k.shape[1]))
        for a in range(0, h, step):
            b = min(h, a + step)
            qa = q[at[i], :n, a:b, :g].float().permute(1, 2, 0, 3)        # [heads, g, n, D]
            t = (qa.reshape(b - a, g * n, D) @ k[a:b].transpose(1, 2)).view(b - a, g, n, -1) / math.sqrt(D)
            t = torch.where(seen, t, -math.inf)
            t = torch.exp(t - t.amax(-1, keepdim=True))
            o = (t.view(b - a, g * n, -1) @ v[a:b]).view(b - a, g, n, D) / t.sum(-1, keepdim=True)
            out[at[i], :n, a:b] = o.permute(2, 0, 1, 3).to(torch.bfloat16)
    return {"out": out.view(B, R, H * g * D)}


# ------------------------------------------------------------------------------------------ the definitions in 64 bits
def exact(case, seed):
    if case["op"] == "plan":
        return None                                                       # whole numbers only
    s = prepare(case, seed)
    B, R, H, D, g = (case[k] for k in ("B", "R", "H", "D", "group"))
    vec = s["qkv"].view(B, R, H, g + 2, D).double()
    held, new = _lengths(case)
    perm = s["perm"].tolist()
    if case["op"] == "write":
        # the two numbers of a group are stored in 16 bits, and a code is a product in 32: those roundings are part of the definition
        out = torch.zeros(B, R, H, 2, D, dtype=torch.float64, device=DEV)
        for p, i in enumerate(perm):
            n, h = new[i], s["heads"][i % case["T"]]
            for j in range(0, D, G64):
                x = vec[p, :n, :h, g:, j:j + G64]
                lo, hi = x.min(-1, keepdim=True).values, x.max(-1, keepdim=True).values
                f = torch.tensor(1 / 15, dtype=torch.float32, device=DEV).double()
                step = ((hi * f).float().double() - (lo * f).float().double()).float().bfloat16().double()
                mid = (lo / 2 + step * 4).float().double().mul(2).bfloat16().double()
                code = torch.round(((x - mid).float().double() * (1 / step).float().double()).float().double()).clamp(-8, 7)
                out[p, :n, :h, :, j:j + G64] = torch.where(step > 0, mid + step * torch.nan_to_num(code), mid)
        return {"values": out.view(B, R, H * 2 * D), "pages": None}
    if work(case)["flops"] > 3e12:
        return None
    out = torch.zeros(B, R, H, g, D, dtype=torch.float64, device=DEV)
    n64 = D // G64
    for p, i in enumerate(perm):
        n, L = new[i], held[i] + new[i]
        tokens = torch.arange(L, device=DEV)
        page = s["table"][i][tokens // case["page"]].long()
        blk, row = tokens % case["page"] // BLOCK, tokens % BLOCK
        for h in range(s["heads"][i % case["T"]]):
            raw = s["pages"][page, h, blk]                                # [L, block]
            kv = []
            for which in range(2):
                part = raw[:, which * raw.shape[1] // 2:][:, : raw.shape[1] // 2]
                codes = part[:, : n64 * BLOCK * 32].view(L, n64, BLOCK, 32)[tokens, :, row].long()
                pair = part[:, n64 * BLOCK * 32:].contiguous().view(L, n64, BLOCK, 4)[tokens, :, row].contiguous().view(torch.bfloat16).double()
                c = torch.empty(L, n64, 64, dtype=torch.float64, device=DEV)
                c[..., 0::2], c[..., 1::2] = (codes % 16).double(), torch.div(codes, 16, rounding_mode="floor").double()
                kv.append((pair[..., 1:] + pair[..., :1] * (c - 8)).reshape(L, D))
            for a in range(0, n, 2048):
                m = min(n, a + 2048)
                pos = held[i] + torch.arange(a, m, device=DEV).view(-1, 1)
                hide = tokens > pos
                if case["window"]:
                    hide |= tokens <= pos - case["window"]
                for e in range(g):
                    t = vec[p, a:m, h, e] @ kv[0].t() * D ** -0.5
                    out[p, a:m, h, e] = torch.softmax(t.masked_fill(hide, -math.inf), -1) @ kv[1]
    return {"out": out.view(B, R, H * g * D)}
