"""Timed cases of many samples of one prompt on one GPU: attention that reads a shared prefix once,
page tables kept on the device, draws with settings of each row's own.

A batch draws several samples of each prompt.  Its rows hold their keys and values on pages of
64 positions, in 8 bits (e4m3 codes, one power-of-two scale per page, layer, K/V head and side); the
rows of one prompt stand next to each other and name the same pages for the prompt's whole pages.
Three operators:

attend  Finds which rows share their leading pages (once a pass) and attends, in every layer of the pass, over the
        shared pages, each row's other pages and its window of new tokens.
turn    Gives the rows' new tokens pages from a stack of free ones, all on the device, with the slot of
        every token, and takes the pages back (a draft that was rejected).
draw    One token of each row of logits from a uniform number of its own, with the row's own temperature, top-k,
        top-p and min-p, and its log-probability in what those leave.

Layout of the pages: codes uint8 [n_pages, n_layers, Hkv, 2, 64 * dh], side 0 the keys [64, dh],
side 1 the values transposed [dh, 64]; scales float32 [n_pages, n_layers, Hkv, 2].

A draw is defined on whole numbers, so that it is the same everywhere: with l' = l (1 / temperature) and m their
maximum, entry v weighs q_v = rint(exp32(l'_v - m) 2^40), exp32 being the float32 exponential below, whose operations
are rounded one by one.  Entries are ordered by l' descending, ties by the lowest index.  K: the first
top_k (all for 0); Q: their weight; P: the shortest prefix of K that weighs ceil(ceil(2^24 top_p) Q / 2^24) or more;
F: those of P with q_v >= ceil(2^40 min_p); T: their weight.  The token is the lowest index at which the running sum of F's
weights, in the order of the indices, exceeds floor(floor(2^24 u) T / 2^24).  Temperature 0 takes the first entry in order.  NaN and
-inf weigh nothing; a row of them alone gives -1 and -inf.

Plain form: `own` is False and the operators run as elementary torch operations.
"""
import math

import torch

own = False

PAGE = 64

# head layouts of the workload models: (query heads, K/V heads, head width, type)
HEADS = {
    "tiny": (4, 4, 16, "f32"),
    "small": (12, 12, 64, "bf16"),
    "block": (16, 4, 128, "bf16"),
    "1b": (16, 16, 128, "bf16"),
    "26b": (32, 16, 128, "bf16"),
}
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
VOCABS = (256, 32768, 50304, 128256, 262144)  # of the workload models


# ------------------------------------------------------------------- the cases
def _attend(heads, batch, groups, n, prefix, own_most, layers, **more):
    """batch rows of `groups` prompts of up to `prefix` positions, each row with up to own_most positions of its own behind
    them and a window of up to n tokens; one pass over `layers` layers."""
    H, Hkv, dh, dtype = HEADS[heads]
    c = dict(op="attend", heads=H, kv_heads=Hkv, head_dim=dh, dtype=dtype, batch=batch, groups=groups, n=n, prefix=prefix,
             own_most=own_most, layers=layers, ragged=False, empty=False, absent=False, window=True)
    c.update(more)
    return c


def _turn(batch, n, held, **more):
    """batch rows that hold up to `held` positions take up to n tokens each; free: pages of the stack for each 64 needed."""
    c = dict(op="turn", batch=batch, n=n, held=held, ragged=True, short=False)
    c.update(more)
    return c


def _draw(rows, vocab, kind, **more):
    """kind: which settings the rows have: "all" mixes them, "k", "p" and "min" one of them, "plain" none."""
    c = dict(op="draw", rows=rows, vocab=vocab, kind=kind, masked=False, stride=vocab)
    c.update(more)
    return c


def listed():
    return [
        # the float32 model: 5 samples of one prompt, a window of 24, lengths that end inside pages, a row without tokens
        dict(_attend("tiny", 5, 1, 24, 320, 40, 2, ragged=True, empty=True), name="attend float32"),
        # two prompts of 1 000 tokens, four samples of each, one token: a call's latency
        dict(_attend("small", 8, 2, 1, 1000, 100, 1, ragged=True), name="attend 8 x 1, 2 prompts"),
        # 64 samples of a prompt of 8 192 tokens, a token each, the 26B-class heads: what sharing is for
        dict(_attend("26b", 64, 1, 1, 8192, 512, 2, ragged=True), name="attend 64 x 1 over 8K"),
        # 16 samples of a prompt of 4 096 tokens, a canvas of 64 each: a step of the block workload
        dict(_attend("block", 16, 1, 64, 4096, 448, 2, ragged=True), name="attend 16 x 64 over 4K"),
        # four samples of a long document, a canvas of 256 each, the 26B-class heads
        dict(_attend("26b", 4, 1, 256, 16384, 256, 1), name="attend 4 x 256 over 16K"),
        # sixteen rows that share nothing, single tokens: what the search for shared pages costs where there are none
        dict(_attend("block", 16, 16, 1, 2048, 1024, 2, ragged=True), name="attend 16 x 1, none shared"),
        # one more token for each of 64 samples: most stay on the page they are on
        dict(_turn(64, 1, 8700), name="turn 64 x 1"),
        # a canvas of 256 for 16 rows, of which the stack has too few pages for the last
        dict(_turn(16, 256, 2000, short=True), name="turn 16 x 256, too few pages"),
        # prompts of up to 4 096 tokens for 64 rows
        dict(_turn(64, 4096, 64), name="turn 64 x 4096"),
        # one row of the 26B-class vocabulary with a nucleus: a call's latency
        dict(_draw(1, 262144, "p"), name="draw 1 x 262144"),
        # 64 samples of the block workload's vocabulary, every row with settings of its own, masked entries among them
        dict(_draw(64, 128256, "all", masked=True), name="draw 64 x 128256"),
        # the masked positions of the small workload's batch at once
        dict(_draw(1024, 32768, "all"), name="draw 1024 x 32768"),
    ]


def _spread(rng, low, high):
    """A whole number of [low, high], spread over its logarithm."""
    return min(high, max(low, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    op = rng.choice(["attend", "attend", "attend", "turn", "draw", "draw"])
    if op == "attend":
        heads = rng.choice(["tiny", "small", "small", "block", "block", "1b", "26b"])
        H, Hkv, dh, dtype = HEADS[heads]
        batch = _spread(rng, 1, 64)
        groups = _spread(rng, 1, batch)
        n = _spread(rng, 1, 256 if batch <= 16 else 16)
        layers = rng.choice([1, 1, 2])
        most = 4 * 256 * 16640 * 32 * 128 // (batch * n * H * dh * layers)  # no more products than the largest
        bytes_most = 64 * 8704 * 16 * 256 // (batch * Hkv * 2 * dh)         # nor more cache
        prefix = _spread(rng, 1, max(2, min(32768 if dtype == "bf16" else 1024, most - 768, bytes_most - 512)))
        return _attend(heads, batch, groups, n, prefix, _spread(rng, 1, max(2, min(512, prefix))), layers,
                       ragged=rng.random() < 0.7, empty=rng.random() < 0.3, absent=rng.random() < 0.2,
                       window=rng.random() < 0.8)
    if op == "turn":
        batch = _spread(rng, 1, 64)
        return _turn(batch, _spread(rng, 1, 4096), _spread(rng, 1, 8192), ragged=rng.random() < 0.7, short=rng.random() < 0.3)
    vocab = rng.choice(VOCABS) - rng.choice([0, 0, 1, 2, 3])
    return _draw(_spread(rng, 1, min(1024, 1024 * 32768 // vocab)), vocab, rng.choice(["all", "all", "k", "p", "min", "plain"]),
                 masked=rng.random() < 0.4, stride=vocab + rng.choice([0, 0, 1, 64]))


# ------------------------------------------------------- sizes that a case fixes
def _group_of(c, b):
    return b * c["groups"] // c["batch"]


def _prefixes(c):
    """Positions of each prompt."""
    p, g = c["prefix"], c["groups"]
    return [max(1, p - (p * i) // (2 * g)) if c["ragged"] else p for i in range(g)]


def _lens(c):
    """Committed positions of each row; none in the last row where `empty` says so."""
    if c["op"] == "turn":
        return [max(0, c["held"] - (c["held"] * b) // c["batch"]) if c["ragged"] else c["held"] for b in range(c["batch"])]
    pre, o, B = _prefixes(c), c["own_most"], c["batch"]
    lens = [pre[_group_of(c, b)] + (o - (o * ((b * 7) % B)) // B if c["ragged"] else o) for b in range(B)]
    if c["empty"]:
        lens[-1] = 0
    return lens


def _news(c):
    """Tokens of each row's window."""
    B, n = c["batch"], c["n"]
    if c["op"] == "turn":
        return [max(1, n - (n * b) // (2 * B)) if c["ragged"] else n for b in range(B)]
    news = [max(1, n - (n * b) // (3 * B)) if c["ragged"] else n for b in range(B)]
    if c["empty"] and B > 1:
        news[-1] = 0
    return news


def _up(x):
    return -(-x // PAGE)


def _max_pages(c):
    if c["op"] == "turn":
        return _up(c["held"] + c["n"])
    return _up(c["prefix"] + c["own_most"])


def _needs(c):
    """Pages that each row's new tokens need beyond those that it holds."""
    return [_up(a + n) - _up(a) for a, n in zip(_lens(c), _news(c))]


def work(case):
    c = case
    if c["op"] == "draw":
        return {"bytes": c["rows"] * (4 * c["vocab"] + 4 + 16 + 8), "flops": 0}
    lens, news, B = _lens(c), _news(c), c["batch"]
    if c["op"] == "turn":
        return {"bytes": B * 12 + sum(_needs(c)) * 16 + B * c["n"] * 8, "flops": 0}
    H, Hkv, dh = c["heads"], c["kv_heads"], c["head_dim"]
    e = 4 if c["dtype"] == "f32" else 2
    w = 1 if c["window"] else 0
    keys = 0  # positions that have to be read: those on shared pages once for their group
    for g, p in enumerate(_prefixes(c)):
        rows = [lens[b] for b in range(B) if _group_of(c, b) == g and lens[b] > 0]
        keys += sum(rows) - (len(rows) - 1) * (p // PAGE) * PAGE if rows else 0
    by = 2 * Hkv * dh * keys + sum(n * (2 * H * dh * e + 4 * H + 2 * w * Hkv * dh * e) for n in news)
    return {"bytes": c["layers"] * by, "flops": c["layers"] * sum(4 * H * dh * n * (ln + w * n) for ln, n in zip(lens, news))}


# ------------------------------------------------------------------- the inputs
def _codes(shape, gen, dev):
    """Random e4m3 codes without NaN, as a quantised cache has them: bell-shaped, few near the top."""
    x = torch.randn(math.prod(shape), device=dev, generator=gen).mul_(90.0).clamp_(-448.0, 448.0)
    return x.to(torch.float8_e4m3fn).view(torch.uint8).view(shape)


def _prepare_attend(c, gen, dev):
    H, Hkv, dh, B, n, layers = c["heads"], c["kv_heads"], c["head_dim"], c["batch"], c["n"], c["layers"]
    dt, P = TYPES[c["dtype"]], _max_pages(c)
    pre, lens = _prefixes(c), _lens(c)
    count = sum(p // PAGE for p in pre) + sum(_up(ln) for ln in lens) + 5
    ids = torch.randperm(count, device=dev, generator=gen).tolist()
    shared = [[ids.pop() for _ in range(p // PAGE)] for p in pre]  # a prompt's whole pages
    table = []
    for b in range(B):
        row = list(shared[_group_of(c, b)]) if lens[b] else []
        row += [ids.pop() for _ in range(_up(lens[b]) - len(row))]
        if c["absent"] and len(row) > 2:
            row[1] = -1
        table.append(row + [-1] * (P - len(row)))
    state = dict(data=_codes((count, layers, Hkv, 2, PAGE * dh), gen, dev),
                 scale=torch.exp2(torch.randint(-8, -5, (count, layers, Hkv, 2), device=dev, generator=gen).float()),
                 table=torch.tensor(table, dtype=torch.int32, device=dev),
                 len=torch.tensor(lens, dtype=torch.int32, device=dev),
                 new=torch.tensor(_news(c), dtype=torch.int32, device=dev))
    cap = _up(n) * PAGE
    loud = 1.0 + 3.0 * (torch.rand(dh, device=dev, generator=gen) < 0.06).float()  # a few wide key channels
    state["k"] = (torch.randn(layers, B, Hkv, cap, dh, device=dev, generator=gen) * loud).to(dt)
    state["vt"] = torch.randn(layers, B, Hkv, dh, cap, device=dev, generator=gen).to(dt)
    state["q"] = torch.randn(layers, B, H, n, dh, device=dev, generator=gen).to(dt)
    state["o"] = torch.zeros(layers, B, n, H * dh, dtype=dt, device=dev)
    state["lse"] = torch.zeros(layers, B, H, n, device=dev)
    state["lead"] = torch.zeros(B, dtype=torch.int32, device=dev)
    state["shared"] = torch.zeros(B, dtype=torch.int32, device=dev)
    return state


def _prepare_turn(c, gen, dev):
    B, P = c["batch"], _max_pages(c)
    lens, needs = _lens(c), _needs(c)
    held = sum(_up(x) for x in lens)
    free = max(0, sum(needs) - 1) if c["short"] else sum(needs) + 7
    ids = torch.randperm(held + free, device=dev, generator=gen).to(torch.int32)
    table = torch.full((B, P), -1, dtype=torch.int32)
    at, host = 0, ids.cpu()
    for b, x in enumerate(lens):
        table[b, :_up(x)] = host[at:at + _up(x)]
        at += _up(x)
    stack = torch.full((held + free,), -1, dtype=torch.int32, device=dev)
    stack[:free] = ids[held:]
    return dict(table=table.to(dev), len=torch.tensor(lens, dtype=torch.int32, device=dev),
                new=torch.tensor(_news(c), dtype=torch.int32, device=dev), ids=stack,
                count=torch.tensor([free, 0, 0, 0], dtype=torch.int32, device=dev),
                granted=torch.zeros(B, dtype=torch.int32, device=dev),
                slots=torch.zeros(B, c["n"], dtype=torch.int64, device=dev))


def _prepare_draw(c, gen, dev):
    R, V = c["rows"], c["vocab"]

    def pick(values):
        return torch.tensor(values, device=dev)[torch.randint(0, len(values), (R,), device=dev, generator=gen)]

    full = torch.empty(R, c["stride"], device=dev)
    width = 1.0 + 3.0 * torch.rand(R, 1, device=dev, generator=gen)  # confident rows and flat ones
    full.copy_(torch.randn(full.shape, device=dev, generator=gen) * width)
    logits = full[:, :V]
    for _ in range(3):  # a few likely tokens
        logits[torch.arange(R, device=dev), torch.randint(0, V, (R,), device=dev, generator=gen)] += 4.0 * width[:, 0]
    if c["masked"]:  # tokens that a grammar forbids
        logits.masked_fill_(torch.rand(R, V, device=dev, generator=gen) < 0.3, -math.inf)
        logits[0, V // 2] = math.nan
    kind = c["kind"]
    temperature = pick([0.7, 1.0, 1.0, 1.3] + ([0.0] if kind == "all" else []))
    state = dict(logits=logits, u=torch.rand(R, device=dev, generator=gen), temperature=temperature)
    if kind in ("all", "k"):
        state["top_k"] = pick([1, 20, 50, 200] + ([0, 0] if kind == "all" else [1000])).to(torch.int32)
    if kind in ("all", "p"):
        state["top_p"] = pick([0.9, 0.95] + ([1.0, 0.3] if kind == "all" else [])).float()
    if kind in ("all", "min"):
        state["min_p"] = pick([0.02, 0.1] + ([0.0, 0.0] if kind == "all" else [])).float()
    state["token"] = torch.zeros(R, dtype=torch.int32, device=dev)
    state["logp"] = torch.zeros(R, device=dev)
    return state


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    state = {"attend": _prepare_attend, "turn": _prepare_turn, "draw": _prepare_draw}[case["op"]](case, gen, dev)
    state["case"] = case
    return state


# --------------------------------------------------------------- the plain forms
def _plain_groups(state):
    """First row of each row's group and the pages that the group shares (0 where a row is alone)."""
    table, ln = state["table"], state["len"]
    B, P = table.shape
    dev = table.device
    rows = torch.arange(B, device=dev)
    whole = torch.minimum(ln[1:], ln[:-1]) // PAGE  # whole pages that a row and the one before it both hold
    same = (table[1:] == table[:-1]) & (torch.arange(P, device=dev) < whole[:, None])
    common = torch.cat([torch.zeros(1, dtype=torch.long, device=dev), same.long().cumprod(1).sum(1)])
    lead = torch.cummax(torch.where(common >= 1, 0, rows), 0).values
    joined = lead != rows
    least = torch.full((B,), P + 1, dtype=torch.long, device=dev)
    least = least.scatter_reduce(0, lead, torch.where(joined, common, P + 1), "amin")[lead]
    return lead, torch.where(least > P, 0, least)


def _plain_attend(state):
    c, table = state["case"], state["table"].long()
    H, Hkv, dh, n, B = c["heads"], c["kv_heads"], c["head_dim"], c["n"], c["batch"]
    lead, shared = _plain_groups(state)
    state["lead"].copy_(lead)
    state["shared"].copy_(shared)
    P = table.shape[1]
    there = (table >= 0) & (table < state["data"].shape[0])
    at = torch.where(there, table, 0)
    pos = torch.arange(P * PAGE, device=table.device)
    committed = (pos < state["len"][:, None]) & there.repeat_interleave(PAGE, 1)
    step = torch.arange(n, device=table.device) < state["new"][:, None]  # [B, n]
    seen = torch.cat([committed, step], 1) if c["window"] else committed
    for layer in range(c["layers"]):
        codes = state["data"][at, layer].view(torch.float8_e4m3fn).float()
        values = codes * state["scale"][at, layer].unsqueeze(-1)  # [B, P, Hkv, 2, 64 dh]
        k = values[:, :, :, 0].reshape(B, P, Hkv, PAGE, dh).permute(0, 2, 1, 3, 4).reshape(B, Hkv, P * PAGE, dh)
        v = values[:, :, :, 1].reshape(B, P, Hkv, dh, PAGE).permute(0, 2, 1, 4, 3).reshape(B, Hkv, P * PAGE, dh)
        if c["window"]:
            k = torch.cat([k, state["k"][layer, :, :, :n].float()], 2)
            v = torch.cat([v, state["vt"][layer, :, :, :, :n].float().transpose(2, 3)], 2)
        v = torch.where(seen[:, None, :, None], v, 0.0)
        q = state["q"][layer].float().reshape(B, Hkv, -1, dh)  # the query heads that share a K/V head, one after the other
        s = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(1.0 / math.sqrt(dh))
        s.masked_fill_(~seen[:, None, None, :], -math.inf)
        top = s.amax(-1, keepdim=True)
        top = torch.where(torch.isfinite(top), top, 0.0)
        s.sub_(top).exp_()
        total = s.sum(-1, keepdim=True)
        o = torch.matmul(s, v) / torch.where(total > 0, total, 1.0)
        lse = (top + total.log()).view(B, H, n)
        o = o.view(B, H, n, dh).permute(0, 2, 1, 3).reshape(B, n, H * dh).to(state["o"].dtype)
        state["o"][layer].copy_(torch.where(step[:, :, None], o, state["o"][layer]))
        state["lse"][layer].copy_(torch.where(step[:, None, :], lse, state["lse"][layer]))
    return state["o"], state["lse"], state["lead"], state["shared"]


def _plain_turn(state):
    table, ln, new, ids, count = (state[k] for k in ("table", "len", "new", "ids", "count"))
    B, P = table.shape
    n = state["case"]["n"]
    dev = table.device
    ln, new = ln.long(), new.long()
    first, last = (ln + PAGE - 1) // PAGE, (ln + new + PAGE - 1) // PAGE
    need = last - first
    upto = need.cumsum(0)
    granted = torch.where((need == 0) | (upto <= count[0]), new, 0)
    place = torch.arange(P, device=dev)
    k = (upto - need)[:, None] + place - first[:, None]  # which of the pages needed each entry takes
    fresh = (place >= first[:, None]) & (place < last[:, None]) & (granted > 0)[:, None]
    taken = torch.where(granted > 0, need, 0).sum()
    table.copy_(torch.where(fresh, ids[(count[0] - 1 - k).clamp(0, ids.shape[0] - 1)], table))
    state["granted"].copy_(granted)
    j = torch.arange(n, device=dev)
    pos = ln[:, None] + j
    page = torch.gather(table, 1, (pos // PAGE).clamp(max=P - 1)).long()
    there = (j < granted[:, None]) & (page >= 0) & (page < ids.shape[0])
    state["slots"].copy_(torch.where(there, page * PAGE + pos % PAGE, -1))
    count[0] -= taken
    # and back: the entries in their order, rows one after the other
    back = fresh & (table >= 0) & (table < ids.shape[0])
    order = back.reshape(-1).long().cumsum(0).view(B, P) - 1
    scratch = torch.cat([ids, ids.new_zeros(1)])
    scratch[torch.where(back, count[0] + order, ids.shape[0])] = table
    ids.copy_(scratch[:-1])
    count[0] += back.sum()
    table.masked_fill_(fresh, -1)
    return state["granted"], state["slots"], table, ids, count


def _exp32(y):
    """The float32 exponential of the draws, y <= 0, every operation rounded by itself; 0 below -30."""
    low = y < -30.0
    y = torch.where(low, -30.0, y)
    k = (y * _bits(0x3FB8AA3B) + 12582912.0) - 12582912.0
    kl = k * _bits(0x35BFBE8E)
    rh = y - k * _bits(0x3F317200)
    r = rh - kl
    p = torch.full_like(r, _bits(0x39500D01))
    for b in (0x3AB60B61, 0x3C088889, 0x3D2AAAAB, 0x3E2AAAAB, 0x3F000000):
        p = p * r
        p = p + _bits(b)
    q = (r * r) * p
    p = (rh + (q - kl)) + 1.0
    return torch.where(low, 0.0, p * torch.exp2(k))


def _bits(b):
    """The float32 with these bits."""
    return torch.tensor(b, dtype=torch.int32).view(torch.float32).item()


def _share(a, total, up):
    """a total / 2^24, a at most 2^24, rounded up or down, without passing 64 bits."""
    high, low = total >> 24, total & 0xFFFFFF
    return a * high + ((a * low + (0xFFFFFF if up else 0)) >> 24)


def _plain_draw(state):
    l, u = state["logits"], state["u"]
    R, V = l.shape
    t = state["temperature"]
    l = torch.where(torch.isnan(l), -math.inf, l)
    x = l * torch.where(t > 0, 1.0 / t, 1.0)[:, None]
    top_k = state["top_k"].long() if "top_k" in state else torch.zeros(R, dtype=torch.long, device=l.device)
    top_k = torch.where(t > 0, torch.where((top_k > 0) & (top_k < V), top_k, V), 1)
    x, ids = torch.sort(x, dim=1, descending=True, stable=True)
    m = x[:, :1]
    q = torch.round(_exp32(torch.where(x == m, 0.0, x - m)) * 2.0 ** 40).long()
    q = torch.where(torch.isneginf(x), 0, q)
    q = torch.where(torch.arange(V, device=l.device) < top_k[:, None], q, 0)
    run_ = q.cumsum(1)
    if "top_p" in state:
        p = torch.ceil(state["top_p"].double() * 2.0 ** 24).clamp(1, 2 ** 24).long()
        target = _share(p, run_[:, -1], True)
        q = torch.where(run_ - q < target[:, None], q, 0)
    if "min_p" in state:
        q = torch.where(q >= torch.ceil(state["min_p"].double() * 2.0 ** 40).clamp(0, 2 ** 40)[:, None].long(), q, 0)
    weight = torch.zeros_like(q).scatter_(1, ids, q)  # in the order of the indices again
    run_ = weight.cumsum(1)
    total = run_[:, -1]
    target = _share(torch.floor(u.double() * 2.0 ** 24).clamp(0, 2 ** 24 - 1).long(), total, False)
    token = (run_ <= target[:, None]).sum(1)
    some = total > 0
    token = torch.where(some, token, 0)
    chosen = torch.gather(weight, 1, token[:, None])[:, 0]
    state["logp"].copy_(torch.where(some, torch.log(chosen.double() / total.clamp(min=1).double()), -math.inf))
    state["token"].copy_(torch.where(some, token, -1))
    return state["token"], state["logp"]


# ------------------------------------------------------------ the framework's calls
_models = {}   # one model handle per head layout and vocabulary, as a serving program has
_streams = {}  # and the stream that each works on


def _handle(heads, kv_heads, head_dim, dtype, vocab, dev):
    import paper_2609_37924_amd as tadm
    key = (heads, kv_heads, head_dim, dtype, vocab)
    if key not in _models:
        cfg = dict(dtype=dtype, vocab=vocab, d_model=64, n_heads=heads, n_kv_heads=kv_heads, head_dim=head_dim, d_ffn=64,
                   ffn_kind="gelu", n_shared=0, n_anchor=1, n_denoise=1, fusion_kind="gated_mlp", rms_eps=1e-6, ln_eps=1e-5,
                   rope_theta=10000.0)
        _models[key] = tadm.tadm_model_create(tadm.make_config(cfg, max_batch=64, max_seq=1024))
    stream = torch._C._cuda_getCurrentRawStream(dev.index or 0)  # the caller's, without a Stream object
    if _streams.get(key) != stream:
        tadm.tadm_set_stream(_models[key], stream)
        _streams[key] = stream
    return tadm, _models[key]


def _own_attend(state):
    c, dev = state["case"], state["data"].device
    tadm, m = _handle(c["heads"], c["kv_heads"], c["head_dim"], c["dtype"], 64, dev)
    n = c["n"]
    if "pages" not in state:  # descriptors and scratch that a program keeps beside its pages
        state["pages"] = tadm.page_set(state["data"], state["scale"])
        state["rows"] = tadm.page_rows(state["table"], _max_pages(c) * PAGE, state["len"], state["new"])
        state["plan"] = tadm.page_plan(torch.empty(tadm.tadm_pages_plan_bytes(m, state["rows"], n), dtype=torch.uint8, device=dev))
        size = tadm.tadm_pages_attend_shared_work(m, state["rows"], n)
        state["work"] = torch.empty(size, dtype=torch.uint8, device=dev)
        state["views"] = [[state[t][i] for t in ("q", "k", "vt", "o", "lse")] for i in range(c["layers"])]
    pages, rows, plan = state["pages"], state["rows"], state["plan"]
    tadm.tadm_pages_share(m, rows, n, 1, plan, state["lead"], state["shared"])
    cap = state["k"].shape[3]
    for layer, (q, k, vt, o, lse) in enumerate(state["views"]):
        if not c["window"]:
            k = vt = None
        tadm.tadm_pages_attend_shared(m, pages, layer, rows, plan, q, n, k, vt, cap, o, lse, state["work"])
    return state["o"], state["lse"], state["lead"], state["shared"]


def _own_turn(state):
    c, dev = state["case"], state["table"].device
    tadm, m = _handle(*HEADS["tiny"], 64, dev)
    if "stack" not in state:
        state["stack"] = tadm.page_stack(state["ids"], state["count"])
        state["take"] = tadm.page_rows(state["table"], c["held"], state["len"], state["new"])
        state["give"] = tadm.page_rows(state["table"], c["held"], state["len"], state["granted"])
    tadm.tadm_pages_assign(m, state["stack"], state["take"], c["n"], state["granted"], state["slots"])
    tadm.tadm_pages_release(m, state["stack"], state["give"], c["n"])
    return state["granted"], state["slots"], state["table"], state["ids"], state["count"]


def _own_draw(state):
    dev = state["logits"].device
    tadm, m = _handle(*HEADS["tiny"], state["case"]["vocab"], dev)
    if "settings" not in state:
        state["settings"] = tadm.row_settings(*(state.get(k) for k in ("temperature", "top_k", "top_p", "min_p")))
        size = tadm.tadm_sample_rows_work(m, state["case"]["rows"])
        state["work"] = torch.empty(max(size, 1), dtype=torch.uint8, device=dev)
    tadm.tadm_sample_rows(m, state["logits"], state["settings"], state["u"], state["token"], state["logp"], state["work"])
    return state["token"], state["logp"]


PLAIN = {"attend": _plain_attend, "turn": _plain_turn, "draw": _plain_draw}
OWN = {"attend": _own_attend, "turn": _own_turn, "draw": _own_draw}


def run(state):
    return (OWN if own else PLAIN)[state["case"]["op"]](state)


# ----------------------------------------------------------------------- 64 bits
def _value(codes):
    """What e4m3 codes stand for, in 64 bits."""
    x = codes.to(torch.int64)
    exp, mant = (x >> 3) & 15, (x & 7).double()
    mag = torch.where(exp == 0, mant * 2.0 ** -9, (8.0 + mant) * torch.exp2(exp.double() - 10.0))
    return torch.where(x >= 128, -mag, mag)


def _exact_attend(c, s):
    H, Hkv, dh, B = c["heads"], c["kv_heads"], c["head_dim"], c["batch"]
    G = H // Hkv
    lens, news, table = _lens(c), _news(c), s["table"].tolist()
    lead, shared = list(range(B)), [0] * B
    for b in range(1, B):
        common = 0
        while common < min(lens[b], lens[b - 1]) // PAGE and table[b][common] == table[b - 1][common]:
            common += 1
        if common:
            lead[b] = lead[b - 1]
            shared[lead[b]] = min(shared[lead[b]] or common, common)
    shared = [shared[a] for a in lead]
    o, lse = s["o"].double(), s["lse"].double()
    for layer in range(c["layers"]):
        for b in range(B):
            if news[b] == 0:
                continue
            ids = torch.tensor(table[b][:_up(lens[b])], dtype=torch.int64, device=s["data"].device)
            keep = (ids >= 0).repeat_interleave(PAGE)[:lens[b]]
            ids = ids.clamp(min=0)
            sides = _value(s["data"][ids, layer]) * s["scale"][ids, layer].double().unsqueeze(-1)  # [P, Hkv, 2, 64 dh]
            K = sides[:, :, 0].reshape(-1, Hkv, PAGE, dh).permute(1, 0, 2, 3).reshape(Hkv, -1, dh)[:, :lens[b]][:, keep]
            V = sides[:, :, 1].reshape(-1, Hkv, dh, PAGE).permute(1, 0, 3, 2).reshape(Hkv, -1, dh)[:, :lens[b]][:, keep]
            if c["window"]:
                K = torch.cat([K, s["k"][layer, b, :, :news[b]].double()], 1)
                V = torch.cat([V, s["vt"][layer, b, :, :, :news[b]].double().transpose(1, 2)], 1)
            for h in range(H):
                at = slice(h * dh, (h + 1) * dh)
                if K.shape[1] == 0:
                    o[layer, b, :news[b], at] = 0.0
                    lse[layer, b, h, :news[b]] = -math.inf
                    continue
                score = s["q"][layer, b, h, :news[b]].double() @ K[h // G].T / math.sqrt(dh)
                lse[layer, b, h, :news[b]] = torch.logsumexp(score, -1)
                o[layer, b, :news[b], at] = torch.softmax(score, -1) @ V[h // G]
    return o, lse, torch.tensor(lead, dtype=torch.int32), torch.tensor(shared, dtype=torch.int32)


def _exact_draw(c, s):
    import numpy as np
    f = np.float32
    ln2_hi, ln2_lo, log2e = (np.uint32(b).view(f) for b in (0x3F317200, 0x35BFBE8E, 0x3FB8AA3B))
    coefficients = [np.uint32(b).view(f) for b in (0x39500D01, 0x3AB60B61, 0x3C088889, 0x3D2AAAAB, 0x3E2AAAAB, 0x3F000000)]
    logits = s["logits"].cpu().numpy()
    R, V = logits.shape

    def setting(name, default):
        return s[name].cpu().numpy() if name in s else np.full(R, default, dtype=f)

    temperature, top_k, top_p, min_p = (setting(k, d) for k, d in (("temperature", 1), ("top_k", 0), ("top_p", 1), ("min_p", 0)))
    u = s["u"].cpu().numpy()
    token, logp = np.full(R, -1, dtype=np.int32), np.full(R, -np.inf)
    for r in range(R):
        x = logits[r]
        at = np.flatnonzero(x > -np.inf)  # neither NaN nor -inf
        if at.size == 0:
            continue
        x = x[at]
        if temperature[r] == 0:
            token[r], logp[r] = at[np.argmax(x)], 0.0
            continue
        x = x * (f(1) / temperature[r])
        y = np.where(x == x.max(), f(0), x - x.max())
        low = y < -30
        y = np.where(low, f(-30), y)
        k = (y * log2e + f(12582912)) - f(12582912)
        rh, kl = y - k * ln2_hi, k * ln2_lo
        d = rh - kl
        p = np.full_like(d, coefficients[0])
        for a in coefficients[1:]:
            p = p * d + a
        p = f(1) + (rh + ((d * d) * p - kl))
        q = np.where(low, 0, np.rint(np.ldexp(p.astype(np.float64), k.astype(np.int32) + 40))).astype(np.int64)
        order = np.argsort(-x, kind="stable")
        if 0 < top_k[r] < V:
            order = order[:top_k[r]]
        run_ = np.cumsum(q[order])
        share = min(max(math.ceil(float(top_p[r]) * 2 ** 24), 1), 2 ** 24)
        order = order[:int(np.searchsorted(run_, -(-share * int(run_[-1]) // 2 ** 24))) + 1]
        order = np.sort(order[q[order] >= min(math.ceil(float(min_p[r]) * 2 ** 40), 2 ** 40)])
        run_ = np.cumsum(q[order])
        i = int(np.searchsorted(run_, math.floor(float(u[r]) * 2 ** 24) * int(run_[-1]) // 2 ** 24, side="right"))
        token[r], logp[r] = at[order[i]], math.log(int(q[order[i]]) / int(run_[-1]))
    return torch.from_numpy(token), torch.from_numpy(logp)


def exact(case, seed):
    if case["op"] == "turn":
        return None  # nothing is computed
    return {"attend": _exact_attend, "draw": _exact_draw}[case["op"]](case, prepare(case, seed))
