"""Timed cases of the paged 8-bit K/V store on one GPU: attention over it, append, copy, read.

A context of the block-diffusion path can keep its keys and values in pages of 64 positions,
held in 8 bits (e4m3) with one power-of-two scale per page, layer, K/V head and side.  Four
operators work on the pages: new keys and values are appended (quantised), a window of
queries attends to them and to its own unquantised keys, pages are copied (a fork copies the
page that both sides would write, compaction moves pages together) and pages are read back.

Layout: codes uint8 [n_pages, n_layers, Hkv, 2, 64 * dh], side 0 the keys [64, dh], side 1
the values transposed [dh, 64]; scales float32 [n_pages, n_layers, Hkv, 2].  A row of the
batch lists its pages in an int32 table [B, max_pages]; an id outside [0, n_pages) is an
absent page, whose positions take no part.

Plain form: `own` is False and the operators run as elementary torch operations in float32.
"""
import math

import torch

own = False

PAGE = 64
TOP = 448.0              # the largest e4m3 value
E_LOW, E_HIGH = -110, 120  # exponents that a scale may have

# head layouts of the workload models: (query heads, K/V heads, head width, type, layers)
HEADS = {
    "tiny": (4, 4, 16, "f32", 3),
    "small": (12, 12, 64, "bf16", 14),
    "block": (16, 4, 128, "bf16", 24),
    "1b": (16, 16, 128, "bf16", 24),
    "26b": (32, 16, 128, "bf16", 46),
}
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


# ------------------------------------------------------------------- the cases
def _case(op, heads, batch, n, ctx, **more):
    """n: tokens of the window (queries and own keys of a call); ctx: committed positions of the longest row."""
    H, Hkv, dh, dtype, _ = HEADS[heads]
    c = dict(op=op, heads=H, kv_heads=Hkv, head_dim=dh, dtype=dtype, layers=1, layer=0, batch=batch, n=n, ctx=ctx,
             ragged=False, empty=False, absent=False, window=True, copies=0)
    c.update(more)
    return c


def listed():
    return [
        # one sequence, one token, a short context: a call's latency
        dict(_case("attend", "block", 1, 1, 200), name="attend one token"),
        # single tokens of 16 sequences of different lengths, the 26B-class head layout
        dict(_case("attend", "26b", 16, 1, 8192, ragged=True), name="attend 16 x 1 over 8K"),
        # one token at the end of a very long context: the key axis alone has the work
        dict(_case("attend", "block", 1, 1, 131071), name="attend 1 over 128K"),
        # a block of 64 tokens per row behind prompts of different lengths: a step of the block workload
        dict(_case("attend", "block", 16, 64, 1024, ragged=True), name="attend 16 x 64 over 1K"),
        # a block of 256 tokens behind a long document, the 26B-class head layout
        dict(_case("attend", "26b", 4, 256, 16384), name="attend 4 x 256 over 16K"),
        # the float32 model's window, with lengths that end inside pages and a row without tokens
        dict(_case("attend", "tiny", 5, 24, 333, ragged=True, empty=True), name="attend float32"),
        # one more token for each of 16 rows, inside a page that holds others
        dict(_case("append", "block", 16, 1, 999, ragged=True), name="append 16 x 1"),
        # a prompt of 1 024 tokens per row, starting inside a page
        dict(_case("append", "26b", 4, 1024, 37), name="append 4 x 1024"),
        # a fork of 4 rows: the page that each row ends in, over all layers
        dict(_case("copy", "block", 4, 1, 512, layers=24, copies=4), name="copy for a fork"),
        # compaction of a pool: 96 pages of the 26B-class model move to the front
        dict(_case("copy", "26b", 1, 1, 6144, layers=46, copies=96), name="copy for a compaction"),
        # contexts of odd lengths read back, one layer of the small model
        dict(_case("read", "small", 8, 1, 777, ragged=True), name="read 8 x 777"),
        # a long context read back, one of several layers
        dict(_case("read", "26b", 4, 1, 16384, layers=3, layer=1), name="read 4 x 16K"),
    ]


def _spread(rng, low, high):
    """A whole number of [low, high], spread over its logarithm."""
    return min(high, max(low, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    op = rng.choice(["attend", "attend", "attend", "append", "append", "copy", "read"])
    heads = rng.choice(["tiny", "small", "small", "block", "block", "1b", "26b"])
    H, Hkv, dh, dtype, layers = HEADS[heads]
    batch = _spread(rng, 1, 16)
    flags = dict(ragged=rng.random() < 0.6, empty=rng.random() < 0.3, absent=rng.random() < 0.2)
    if op == "attend":
        n = _spread(rng, 1, 256)
        most = 4 * 4 * 256 * 16384 * 32 * 128 // 4 // (batch * n * H * dh)  # no more products than the largest
        bytes_most = 4 * 16384 * 16 * 256 // (batch * Hkv * 2 * dh)         # nor more cache
        ctx = _spread(rng, 1, max(2, min(131072 if dtype == "bf16" else 2048, most, bytes_most)))
        n_layers = rng.choice([1, 1, 2])
        return _case("attend", heads, batch, n, ctx, layers=n_layers, layer=n_layers - 1,
                     window=rng.random() < 0.8, **flags)
    if op == "append":
        return _case("append", heads, batch, _spread(rng, 1, 1024 if batch <= 4 else 256), _spread(rng, 1, 4096), **flags)
    if op == "copy":
        page = layers * Hkv * 2 * PAGE * dh
        return _case("copy", heads, 1, 1, 64, layers=layers, copies=_spread(rng, 1, min(512, 96 * 46 * 16 * 16384 // page)))
    n_layers = rng.choice([1, 3])
    return _case("read", heads, batch, 1, _spread(rng, 1, 16384 if batch <= 4 else 4096), layers=n_layers,
                 layer=n_layers - 1, **flags)


# ------------------------------------------------------- sizes that a case fixes
def _lens(c):
    """Committed positions of each row before the call: the longest first, a last row without any where `empty` says so."""
    B, ctx = c["batch"], c["ctx"]
    lens = [ctx - (ctx * b) // (2 * B) if c["ragged"] else ctx for b in range(B)]
    if c["empty"]:
        lens[-1] = 0
    return lens


def _news(c):
    """Tokens of each row's window."""
    B, n = c["batch"], c["n"]
    news = [max(1, n - (n * b) // (3 * B)) if c["ragged"] else n for b in range(B)]
    if c["empty"] and B > 1:
        news[-1] = 0
    return news


def _cap(n):
    return -(-n // PAGE) * PAGE


def _max_pages(c):
    return -(-(c["ctx"] + (c["n"] if c["op"] == "append" else 0)) // PAGE)


def work(case):
    c = case
    H, Hkv, dh = c["heads"], c["kv_heads"], c["head_dim"]
    e = 4 if c["dtype"] == "f32" else 2
    if c["op"] == "copy":
        return {"bytes": 2 * c["copies"] * c["layers"] * Hkv * (2 * PAGE * dh + 8), "flops": 0}
    lens, news = _lens(c), _news(c)
    if c["op"] == "attend":
        own_keys = 1 if c["window"] else 0
        by = sum(2 * Hkv * dh * ln + n * (2 * H * dh * e + 4 * H + 2 * own_keys * Hkv * dh * e) for ln, n in zip(lens, news))
        return {"bytes": by, "flops": sum(4 * H * dh * n * (ln + own_keys * n) for ln, n in zip(lens, news))}
    if c["op"] == "append":
        return {"bytes": sum(news) * 2 * Hkv * dh * (e + 1), "flops": 0}
    return {"bytes": sum(lens) * 2 * Hkv * dh * (1 + e), "flops": 0}


# ------------------------------------------------------------------- the inputs
def _codes(shape, gen, dev):
    """Random e4m3 codes without NaN, as a quantised cache has them: bell-shaped, few near the top."""
    n = math.prod(shape)
    if n > 1 << 29:  # for pages that are only moved: any finite code
        x = torch.randint(0, 256, (n,), dtype=torch.uint8, device=dev, generator=gen)
        return torch.where((x & 127) == 127, x - 1, x).view(shape)
    x = torch.randn(n, device=dev, generator=gen).mul_(90.0).clamp_(-TOP, TOP)
    return x.to(torch.float8_e4m3fn).view(torch.uint8).view(shape)


def prepare(case, seed):
    c = case
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    H, Hkv, dh, B, n, layers = c["heads"], c["kv_heads"], c["head_dim"], c["batch"], c["n"], c["layers"]
    dt = TYPES[c["dtype"]]
    if c["op"] == "copy":
        n_pages = 2 * c["copies"] + 3
    else:
        n_pages = B * _max_pages(c) + 5
    state = dict(case=c)
    state["data"] = _codes((n_pages, layers, Hkv, 2, PAGE * dh), gen, dev)
    state["scale"] = torch.exp2(torch.randint(-8, -5, (n_pages, layers, Hkv, 2), device=dev, generator=gen).float())
    if c["op"] == "copy":  # pages of the back half to free pages of the front half, in no order
        cpu = torch.Generator()
        cpu.manual_seed(seed)
        half = n_pages // 2
        state["src"] = (half + torch.randperm(n_pages - half, generator=cpu)[:c["copies"]]).to(torch.int32).numpy()
        state["dst"] = torch.randperm(half, generator=cpu)[:c["copies"]].to(torch.int32).numpy()
        return state
    table = torch.randperm(n_pages, device=dev, generator=gen)[:B * _max_pages(c)].view(B, -1).to(torch.int32)
    if c["absent"] and c["op"] != "append" and table.shape[1] > 2:
        table[:, 1] = -1
    state["table"] = table.contiguous()
    state["len"] = torch.tensor(_lens(c), dtype=torch.int32, device=dev)
    state["new"] = torch.tensor(_news(c), dtype=torch.int32, device=dev)
    if c["op"] == "read":
        cap = _cap(c["ctx"])
        state["k"] = torch.zeros(B, Hkv, cap, dh, dtype=dt, device=dev)
        state["vt"] = torch.zeros(B, Hkv, dh, cap, dtype=dt, device=dev)
        return state
    cap = _cap(n)
    loud = 1.0 + 3.0 * (torch.rand(dh, device=dev, generator=gen) < 0.06).float()  # a few wide key channels
    k = torch.randn(B, Hkv, cap, dh, device=dev, generator=gen) * loud
    vt = torch.randn(B, Hkv, dh, cap, device=dev, generator=gen)
    state["k"], state["vt"] = k.to(dt), vt.to(dt)
    if c["op"] == "attend":
        state["q"] = torch.randn(B, H, n, dh, device=dev, generator=gen).to(dt)
        state["o"] = torch.zeros(B, n, H * dh, dtype=dt, device=dev)
        state["lse"] = torch.zeros(B, H, n, device=dev)
    return state


# --------------------------------------------------------------- the plain forms
def _sides(state, layer):
    """Keys [B, Hkv, P 64, dh] and values [B, Hkv, P 64, dh] of each row's pages in float32, and which positions are there."""
    c, table = state["case"], state["table"].long()
    Hkv, dh = c["kv_heads"], c["head_dim"]
    B, P = table.shape
    there = (table >= 0) & (table < state["data"].shape[0])
    at = torch.where(there, table, 0)
    codes = state["data"][at, layer].view(torch.float8_e4m3fn).float()
    values = codes * state["scale"][at, layer].unsqueeze(-1)  # [B, P, Hkv, 2, 64 dh]
    k = values[:, :, :, 0].reshape(B, P, Hkv, PAGE, dh).permute(0, 2, 1, 3, 4).reshape(B, Hkv, P * PAGE, dh)
    v = values[:, :, :, 1].reshape(B, P, Hkv, dh, PAGE).permute(0, 2, 1, 4, 3).reshape(B, Hkv, P * PAGE, dh)
    pos = torch.arange(P * PAGE, device=table.device)
    return k, v, (pos < state["len"][:, None]) & there.repeat_interleave(PAGE, 1), pos


def _plain_attend(state):
    c = state["case"]
    H, Hkv, dh, n = c["heads"], c["kv_heads"], c["head_dim"], c["n"]
    B = c["batch"]
    k, v, seen, _ = _sides(state, c["layer"])
    step = torch.arange(n, device=k.device) < state["new"][:, None]  # [B, n]
    if c["window"]:
        k = torch.cat([k, state["k"][:, :, :n].float()], 2)
        v = torch.cat([v, state["vt"][:, :, :, :n].float().transpose(2, 3)], 2)
        seen = torch.cat([seen, step], 1)
    v = torch.where(seen[:, None, :, None], v, 0.0)
    q = state["q"].float().reshape(B, Hkv, -1, dh)  # the query heads that share a K/V head, one after the other
    s = torch.matmul(q, k.transpose(2, 3)).mul_(1.0 / math.sqrt(dh))
    s.masked_fill_(~seen[:, None, None, :], -math.inf)
    top = s.amax(-1, keepdim=True)
    top = torch.where(torch.isfinite(top), top, 0.0)
    s.sub_(top).exp_()
    total = s.sum(-1, keepdim=True)
    o = torch.matmul(s, v) / torch.where(total > 0, total, 1.0)
    lse = (top + total.log()).view(B, H, n)
    o = o.view(B, H, n, dh).permute(0, 2, 1, 3).reshape(B, n, H * dh).to(state["o"].dtype)
    state["o"].copy_(torch.where(step[:, :, None], o, state["o"]))
    state["lse"].copy_(torch.where(step[:, None, :], lse, state["lse"]))
    return state["o"], state["lse"]


def _exponent(top):
    """The least e with top <= 448 2^e, within the range of a scale."""
    m, x = torch.frexp(top / TOP)
    e = torch.where(m == 0.5, x - 1, x)
    return torch.where(top > 0, e, E_LOW).clamp(E_LOW, E_HIGH).float()


def _plain_append(state):
    c = state["case"]
    Hkv, dh, layer = c["kv_heads"], c["head_dim"], c["layer"]
    table = state["table"].long()
    B, P = table.shape
    dev = table.device
    codes = state["data"][table, layer].view(torch.float8_e4m3fn).float()  # [B, P, Hkv, 2, 64 dh]
    old_scale = state["scale"][table, layer]
    old = torch.stack([codes[:, :, :, 0].view(B, P, Hkv, PAGE, dh), codes[:, :, :, 1].view(B, P, Hkv, dh, PAGE).transpose(3, 4)], 3)
    pos = torch.arange(P * PAGE, device=dev)
    first = state["len"][:, None].long()
    fresh = (pos >= first) & (pos < first + state["new"][:, None])
    at = (pos - first).clamp(0, c["n"] - 1)  # the window's token of each position
    kv = torch.stack([state["k"].float(), state["vt"].float().transpose(2, 3)], 3)  # [B, Hkv, cap, 2, dh]
    new = torch.gather(kv, 2, at[:, None, :, None, None].expand(B, Hkv, P * PAGE, 2, dh))
    new = new.view(B, Hkv, P, PAGE, 2, dh).permute(0, 2, 1, 4, 3, 5)  # [B, P, Hkv, 2, 64, dh]
    fresh = fresh.view(B, P, 1, 1, PAGE, 1)
    top = torch.where(fresh, new.abs(), 0.0).amax((4, 5))
    held = (pos.view(1, P, PAGE)[:, :, 0] < first)[:, :, None, None]  # the page has positions before the call
    touched = fresh.any(4).view(B, P, 1, 1)
    scale = torch.exp2(_exponent(top))
    scale = torch.where(held, torch.maximum(scale, old_scale), scale)
    scale = torch.where(touched, scale, old_scale)
    prior = (pos < first).view(B, P, 1, 1, PAGE, 1)
    old = torch.where(prior, old * (old_scale / scale)[..., None, None], old)  # what lies behind the row stays as it is
    new = new / scale[..., None, None]
    page = torch.where(fresh, new, old).to(torch.float8_e4m3fn)
    page = torch.stack([page[:, :, :, 0].reshape(B, P, Hkv, -1), page[:, :, :, 1].transpose(3, 4).reshape(B, P, Hkv, -1)], 3)
    state["data"][table, layer] = page.view(torch.uint8)
    state["scale"][table, layer] = scale
    return state["data"].view(torch.float8_e4m3fn), state["scale"]


def _plain_copy(state):
    dev = state["data"].device
    src, dst = torch.from_numpy(state["src"]).to(dev).long(), torch.from_numpy(state["dst"]).to(dev).long()
    state["data"][dst] = state["data"][src]
    state["scale"][dst] = state["scale"][src]
    return state["data"].view(torch.float8_e4m3fn), state["scale"]


def _plain_read(state):
    k, v, seen, pos = _sides(state, state["case"]["layer"])
    before = (pos < state["len"][:, None])[:, None, :, None]
    seen = seen[:, None, :, None]
    k, v = torch.where(seen, k, 0.0).to(state["k"].dtype), torch.where(seen, v, 0.0).to(state["k"].dtype)
    state["k"].copy_(torch.where(before, k, state["k"]))
    state["vt"].copy_(torch.where(before, v, state["vt"].transpose(2, 3)).transpose(2, 3))
    return state["k"], state["vt"]


# ------------------------------------------------------------ the framework's calls
_models = {}   # one model handle per head layout, as a serving program has
_streams = {}  # and the stream that each works on


def _handle(state):
    import paper_2609_37924_amd as tadm
    c = state["case"]
    key = (c["heads"], c["kv_heads"], c["head_dim"], c["dtype"])
    if key not in _models:
        cfg = dict(dtype=c["dtype"], vocab=64, d_model=64, n_heads=c["heads"], n_kv_heads=c["kv_heads"],
                   head_dim=c["head_dim"], d_ffn=64, ffn_kind="gelu", n_shared=0, n_anchor=1, n_denoise=1,
                   fusion_kind="gated_mlp", rms_eps=1e-6, ln_eps=1e-5, rope_theta=10000.0)
        _models[key] = tadm.tadm_model_create(tadm.make_config(cfg, max_batch=16, max_seq=1024))
    stream = torch._C._cuda_getCurrentRawStream(state["data"].get_device())  # the caller's, without a Stream object
    if _streams.get(key) != stream:
        tadm.tadm_set_stream(_models[key], stream)
        _streams[key] = stream
    return tadm, _models[key]


def _own(state):
    tadm, m = _handle(state)
    c = state["case"]
    if "pages" not in state:  # descriptors and workspace that a program keeps beside its pages
        state["pages"] = tadm.page_set(state["data"], state["scale"])
        if c["op"] != "copy":
            state["rows"] = tadm.page_rows(state["table"], _max_pages(c) * PAGE, state["len"], state["new"])
        if c["op"] == "attend":
            size = tadm.tadm_pages_attend_work(m, state["rows"], c["n"])
            state["work"] = torch.empty(max(size, 1), dtype=torch.uint8, device=state["data"].device)
    if c["op"] == "copy":
        tadm.tadm_pages_copy(m, state["pages"], state["src"], state["dst"])
        return state["data"].view(torch.float8_e4m3fn), state["scale"]
    if c["op"] == "read":
        tadm.tadm_pages_read(m, state["pages"], c["layer"], state["rows"], state["k"], state["vt"], state["k"].shape[2])
        return state["k"], state["vt"]
    cap = state["k"].shape[2]
    if c["op"] == "append":
        tadm.tadm_pages_append(m, state["pages"], c["layer"], state["rows"], state["k"], state["vt"], c["n"], cap)
        return state["data"].view(torch.float8_e4m3fn), state["scale"]
    k, vt = (state["k"], state["vt"]) if c["window"] else (None, None)
    tadm.tadm_pages_attend(m, state["pages"], c["layer"], state["rows"], state["q"], c["n"], k, vt, cap, state["o"],
                           state["lse"], state["work"])
    return state["o"], state["lse"]


PLAIN = {"attend": _plain_attend, "append": _plain_append, "copy": _plain_copy, "read": _plain_read}


def run(state):
    if own:
        return _own(state)
    return PLAIN[state["case"]["op"]](state)


# ----------------------------------------------------------------------- 64 bits
def _value(codes):
    """What e4m3 codes stand for, in 64 bits."""
    x = codes.to(torch.int64)
    exp, mant = (x >> 3) & 15, (x & 7).double()
    mag = torch.where(exp == 0, mant * 2.0 ** -9, (8.0 + mant) * torch.exp2(exp.double() - 10.0))
    return torch.where(x >= 128, -mag, mag)


def exact(case, seed):
    c = case
    if c["op"] == "copy":
        return None  # nothing is computed
    s = prepare(c, seed)
    H, Hkv, dh, n, layer = c["heads"], c["kv_heads"], c["head_dim"], c["n"], c["layer"]
    G = H // Hkv
    lens, news, table = _lens(c), _news(c), s["table"].tolist()
    if c["op"] == "append":
        data, scale = _value(s["data"]), s["scale"].double()
        for b in range(c["batch"]):
            for p in range(lens[b] // PAGE, -(-(lens[b] + news[b]) // PAGE)):
                page, start = table[b][p], p * PAGE
                lo, hi = max(lens[b], start), min(lens[b] + news[b], start + PAGE)
                if hi <= lo:
                    continue
                for side, new in ((0, s["k"][b, :, lo - lens[b]:hi - lens[b]].double()),
                                  (1, s["vt"][b, :, :, lo - lens[b]:hi - lens[b]].double())):
                    top = new.abs().amax((1, 2))
                    e = torch.floor(torch.log2(torch.clamp(top, min=1e-300) / TOP)) - 1.0
                    for _ in range(3):  # up to the least e with top <= 448 2^e
                        e = e + (top > TOP * torch.exp2(e)).double()
                    step = torch.exp2(e.clamp(E_LOW, E_HIGH))
                    if start < lens[b]:
                        step = torch.maximum(step, scale[page, layer, :, side])
                    grown = (scale[page, layer, :, side] / step)[:, None, None]
                    was = data[page, layer, :, side].clone()
                    part = was.view(Hkv, PAGE, dh) if side == 0 else was.view(Hkv, dh, PAGE).transpose(1, 2)
                    part[:, :lo - start] *= grown
                    part[:, lo - start:hi - start] = (new if side == 0 else new.transpose(1, 2)) / step[:, None, None]
                    data[page, layer, :, side] = was
                    scale[page, layer, :, side] = step
        return data, scale
    if c["op"] == "read":
        k, vt = s["k"].double(), s["vt"].double()
    else:
        o, lse = s["o"].double(), s["lse"].double()
    for b in range(c["batch"]):
        ids = torch.tensor(table[b][:-(-lens[b] // PAGE)], dtype=torch.int64, device=s["data"].device)
        keep = (ids >= 0).repeat_interleave(PAGE)[:lens[b]]
        ids = ids.clamp(min=0)
        for h in range(Hkv):
            sides = _value(s["data"][ids, layer, h]) * s["scale"][ids, layer, h].double()[:, :, None]
            K = sides[:, 0].reshape(-1, dh)[:lens[b]]
            V = sides[:, 1].reshape(-1, dh, PAGE).transpose(1, 2).reshape(-1, dh)[:lens[b]]
            if c["op"] == "read":
                k[b, h, :lens[b]] = torch.where(keep[:, None], K, 0.0)
                vt[b, h, :, :lens[b]] = torch.where(keep[:, None], V, 0.0).T
                continue
            K, V = K[keep], V[keep]
            if c["window"]:
                K = torch.cat([K, s["k"][b, h, :news[b]].double()])
                V = torch.cat([V, s["vt"][b, h, :, :news[b]].double().T])
            for g in range(h * G, h * G + G):
                score = s["q"][b, g, :news[b]].double() @ K.T / math.sqrt(dh)
                if news[b] == 0:
                    continue
                if K.shape[0] == 0:
                    o[b, :news[b], g * dh:(g + 1) * dh] = 0.0
                    lse[b, g, :news[b]] = -math.inf
                    continue
                lse[b, g, :news[b]] = torch.logsumexp(score, -1)
                o[b, :news[b], g * dh:(g + 1) * dh] = torch.softmax(score, -1) @ V
    return (k, vt) if c["op"] == "read" else (o, lse)
