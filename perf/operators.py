"""The paged-cache operators as measured work: cases, inputs, plain forms and 64-bit values.

Four operators, the path of a layer that keeps its whole history in pages instead of in a bounded cache:

  rope    per-head RMS norm of queries and keys and the rotation by position, in one pass
  cache   new keys and values written to the pages (8-bit forms with a scale per row) and read back
  attend  attention of one new token per sequence over its pages
  sparse  the pages chosen per sequence and KV head by a bound on their logits, and the attention over those

`run` computes them from elementary torch operations, or, where `own` is set, through the package.
A pool is [1 layer][pages][kv heads][page tokens][head dim]; a sequence's pages are listed in its row
of `table`. Lengths follow from a case alone, everything else from the seed.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn, "i8": torch.int8}
SIZE = {"f32": 4, "bf16": 2, "e4m3": 1, "i8": 1}
TOP = {"e4m3": 448.0, "i8": 127.0}
TINY = 2.0 ** -100
EPS = 1e-6
THETA = 500000.0


# ---- cases ---------------------------------------------------------------------------------------

def listed():
    return [
        # one decode step of a 16-sequence grouped-query batch
        rope("rope step", 16, 32, 8, 128, "bf16", 128, False, 1, 40000),
        # a test-sized prompt of the fp32 path, a quarter of each head rotated in neighbouring pairs
        rope("rope odd f32", 1537, 7, 7, 64, "f32", 16, True, 1537, 1 << 20),
        # one long summarisation prompt, grouped-query heads
        rope("rope prompt", 32768, 32, 8, 128, "bf16", 128, False, 32768, 32768),
        # one decode step of 32 ragged question-answering sequences into an 8-bit cache
        cache("cache step e4m3", 32, 1, 1, 8192, 8, 128, "bf16", "e4m3", 16),
        # odd prompts continued in the middle of a page, fp32 rows kept in 8 bits
        cache("cache odd i8", 5, 3, 700, 333, 5, 64, "f32", "i8", 32),
        # the prompts of the 16-sequence batch
        cache("cache prompts i8", 16, 4096, 8192, 0, 8, 128, "bf16", "i8", 64),
        # a single short conversation: latency
        attend("attend one", 1, 517, 517, 32, 8, 128, "bf16", "bf16", 16),
        # the 16-sequence grouped-query batch at its full ragged length
        attend("attend batch", 16, 4001, 8192, 32, 8, 128, "bf16", "bf16", 16),
        # 32 ragged document sets in an 8-bit cache: the largest
        attend("attend documents i8", 32, 8192, 16384, 32, 8, 128, "bf16", "i8", 64),
        # a few sequences of test size, fp32, one head per KV head
        sparse("sparse odd f32", 3, 77, 1999, 6, 6, 64, "f32", "f32", 16, 1, 2, 13),
        # one very long sequence: choosing costs more than attending
        sparse("sparse long", 1, 131072, 131072, 32, 8, 128, "bf16", "bf16", 16, 1, 8, 119),
        # a batch of long summaries in an 8-bit cache, all heads their own
        sparse("sparse batch e4m3", 8, 16384, 32768, 32, 32, 128, "bf16", "e4m3", 32, 1, 15, 112),
    ]


def rope(name, tokens, q_heads, kv_heads, dim, dtype, rotary, interleaved, run_length, far):
    return dict(name=name, op="rope", tokens=tokens, q_heads=q_heads, kv_heads=kv_heads, dim=dim, dtype=dtype, rotary=rotary,
                interleaved=interleaved, run_length=run_length, far=far)


def cache(name, batch, least, most, before, kv_heads, dim, dtype, kept, page):
    return dict(name=name, op="cache", batch=batch, least=least, most=most, before=before, kv_heads=kv_heads, dim=dim, dtype=dtype,
                kept=kept, page=page)


def attend(name, batch, least, most, q_heads, kv_heads, dim, dtype, kept, page):
    return dict(name=name, op="attend", batch=batch, least=least, most=most, q_heads=q_heads, kv_heads=kv_heads, dim=dim, dtype=dtype,
                kept=kept, page=page)


def sparse(name, batch, least, most, q_heads, kv_heads, dim, dtype, kept, page, sink, recent, top):
    return dict(attend(name, batch, least, most, q_heads, kv_heads, dim, dtype, kept, page), op="sparse", sink=sink, recent=recent, top=top)


def draw(rng):
    def log(a, b):
        return min(b, max(a, int(round(math.exp(rng.uniform(math.log(a), math.log(b)))))))

    op = rng.choice(["rope", "cache", "attend", "sparse"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    kept = rng.choice([dtype, "e4m3", "i8"])
    kv_heads = rng.choice([1, 2, 3, 4, 5, 7, 8, 16, 32])
    q_heads = kv_heads * rng.choice([g for g in (1, 2, 4, 8) if g * kv_heads <= 64])
    dim, page = rng.choice([64, 128]), rng.choice([16, 32, 64, 128])
    if op == "rope":
        tokens = log(1, max(1, min(32768, (1 << 28) // ((q_heads + kv_heads) * dim * SIZE[dtype]))))
        case = rope("", tokens, q_heads, kv_heads, dim, dtype, rng.choice([r for r in (16, 32, 48, 64, 96, 128) if r <= dim]), rng.random() < 0.5,
                    rng.choice([1, tokens]), log(tokens, 1 << 20))
    elif op == "cache":
        batch = log(1, 32)
        most = log(1, max(1, min(8192, (1 << 27) // (batch * kv_heads * dim * 4))))
        case = cache("", batch, rng.randint(1, most), most, rng.choice([0, log(1, 8192)]), kv_heads, dim, dtype, kept, page)
    else:
        batch = log(1, 32)
        row = kv_heads * dim * (8 if op == "attend" else 16)      # fp32 K and V rows of the plain form
        most = log(1, max(1, min(16384 if op == "attend" else 65536, (1 << 31) // (batch * row))))
        case = attend("", batch, rng.randint(1, most), most, q_heads, kv_heads, dim, dtype, kept, page)
        if op == "sparse":
            case = dict(case, op=op, sink=rng.randint(0, 4), recent=rng.randint(1, 8), top=log(1, 96))
    del case["name"]
    return case


# ---- inputs --------------------------------------------------------------------------------------

def lengths(case):
    """Per sequence a length between the case's bounds, both of them among them."""
    b, lo, hi = case["batch"], case["least"], case["most"]
    return [hi if i == 0 else lo if i == b - 1 else lo + int((hi - lo) * ((0.6180339887 * i) % 1.0)) for i in range(b)]


def quantise(x, kind):
    """Rows of x (fp32, last dimension) as 8-bit codes and an fp32 scale per row; wider kinds pass through rounded, without a scale."""
    if kind not in TOP:
        return x.to(TYPES[kind]), None
    top = x.abs().amax(-1)
    scale = (top / torch.full_like(top, TOP[kind])).clamp_min(TINY)       # by a tensor: a quotient by a number is a product with its reciprocal
    y = (x / scale.unsqueeze(-1)).clamp(-TOP[kind], TOP[kind])
    return (y.round() if kind == "i8" else y).to(TYPES[kind]), scale


def make_pool(case, lens, gen, centred):
    """A pool that holds sequences of these lengths on shuffled pages: dict of k, v, scales, bounds, and their table."""
    P, H, D = case["page"], case["kv_heads"], case["dim"]
    counts = [-(-n // P) for n in lens]
    total, width = sum(counts) + 3, max(max(counts), 1)
    perm = torch.randperm(total, generator=gen, device=DEV).to(torch.int32)
    at = torch.arange(width, device=DEV).unsqueeze(0)
    np_ = torch.tensor(counts, device=DEV).unsqueeze(1)
    first = torch.tensor([sum(counts[:i]) for i in range(len(counts))], device=DEV).unsqueeze(1)
    table = torch.where(at < np_, perm[torch.where(at < np_, first + at, 0)], -1).to(torch.int32)
    pool = {"table": table, "lens": torch.tensor(lens, dtype=torch.int32, device=DEV)}
    for name in ("k", "v"):
        x = torch.randn(1, total, H, P, D, generator=gen, device=DEV)
        if name == "k":
            x *= torch.where(torch.rand(1, total, H, P, 1, generator=gen, device=DEV) < 0.03, 3.0, 1.0)   # a few heavy hitters
            if centred:                                                                                   # neighbours look alike
                x += torch.randn(1, total, H, 1, D, generator=gen, device=DEV)
                x = x.to(TYPES[case["dtype"]]).float()
                live = torch.zeros(total, dtype=torch.long, device=DEV)
                n = (pool["lens"].unsqueeze(1) - at * P).clamp(0, P)
                live[perm[: sum(counts)].long()] = n[at < np_].long()
                off = (torch.arange(P, device=DEV).unsqueeze(0) >= live.unsqueeze(1)).view(1, total, 1, P, 1)
                low, high = x.masked_fill(off, math.inf).amin(3), x.masked_fill(off, -math.inf).amax(3)
                pool["bounds"] = torch.stack([low, high], 3).nan_to_num(posinf=0.0, neginf=0.0).to(TYPES[case["dtype"]])
        x = x.to(TYPES[case["dtype"]]).float()
        pool[name], pool[name + "_scale"] = quantise(x, case["kept"])
        del x
    return pool


def handle(case, pool, bounds):
    """The cache object that a user's program keeps over these buffers."""
    from paper_2410_23079_b200 import BuzzPaged
    names = ["k", "v"] + (["k_scale", "v_scale"] if case["kept"] in TOP else []) + (["bounds"] if bounds else [])
    return BuzzPaged(layers=1, pages=pool["k"].shape[1], page_tokens=case["page"], q_heads=case.get("q_heads", case["kv_heads"]),
                     kv_heads=case["kv_heads"], head_dim=case["dim"], dtype=TYPES[case["dtype"]], cache_dtype=TYPES[case["kept"]],
                     bounds=bounds, buffers={n: pool[n] for n in names}, device=DEV)


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(int(seed))
    dt = TYPES[case["dtype"]]

    def randn(*shape):
        return torch.randn(*shape, generator=gen, device=DEV)

    s = {"case": case}
    if case["op"] == "rope":
        T, D = case["tokens"], case["dim"]
        wide = case["q_heads"] + 2 * case["kv_heads"]                     # q | k | v as one projection leaves them
        qkv = (randn(T, wide, D) * (0.5 + torch.rand(1, wide, 1, generator=gen, device=DEV))).to(dt)
        s["q"], s["k"] = qkv[:, :case["q_heads"]], qkv[:, case["q_heads"]:case["q_heads"] + case["kv_heads"]]
        start = torch.randint(0, case["far"] - min(case["far"], case["run_length"]) + 1, (-(-T // case["run_length"]), 1), generator=gen, device=DEV)
        s["positions"] = (start + torch.arange(case["run_length"], device=DEV)).reshape(-1)[:T].to(torch.int32)
        s["inv_freq"] = (THETA ** (-torch.arange(0, case["rotary"], 2, device=DEV, dtype=torch.float64) / case["rotary"])).float()
        s["q_weight"], s["k_weight"] = (1 + 0.1 * randn(D)).to(dt), (1 + 0.1 * randn(D)).to(dt)
        return s
    if case["op"] == "cache":
        new, H, D, P = lengths(case), case["kv_heads"], case["dim"], case["page"]
        lens = [n + case["before"] for n in new]
        width = -(-max(lens) // P)
        total = width * case["batch"]
        s["table"] = torch.randperm(total, generator=gen, device=DEV).to(torch.int32).view(case["batch"], width)
        s["lens"] = torch.tensor(lens, dtype=torch.int32, device=DEV)
        cu = [0]
        for n in new:
            cu.append(cu[-1] + n)
        s["cu"], s["max_new"] = torch.tensor(cu, dtype=torch.int32, device=DEV), max(new)
        s["k_new"], s["v_new"] = randn(cu[-1], H, D).to(dt), randn(cu[-1], H, D).to(dt)
        for n in ("k", "v"):
            s[n] = torch.zeros(1, total, H, P, D, dtype=torch.int8, device=DEV).view(TYPES[case["kept"]]) if case["kept"] in TOP else \
                torch.zeros(1, total, H, P, D, dtype=dt, device=DEV)
            s[n + "_scale"] = torch.zeros(1, total, H, P, device=DEV)
        s["k_back"], s["v_back"] = torch.empty_like(s["k_new"]), torch.empty_like(s["v_new"])
        if own:
            s["handle"] = handle(case, s, False)
        return s
    lens = lengths(case)
    s.update(make_pool(case, lens, gen, case["op"] == "sparse"))
    q = randn(case["batch"], case["q_heads"], case["dim"])
    if case["op"] == "sparse":                                            # a query that looks for one of its pages
        pick = (torch.rand(case["batch"], generator=gen, device=DEV) * ((s["lens"] + case["page"] - 1) // case["page"])).long()
        page = s["table"].gather(1, pick.unsqueeze(1)).squeeze(1).long()
        q += s["bounds"][0, page].float().mean(2).repeat_interleave(case["q_heads"] // case["kv_heads"], 1)
        s["selected"] = torch.empty(case["batch"], case["kv_heads"], case["sink"] + case["recent"] + case["top"], dtype=torch.int32, device=DEV)
    s["q"] = q.to(dt)
    s["out"], s["lse"] = torch.empty_like(s["q"]), torch.empty(case["batch"], case["q_heads"], device=DEV)
    if own:
        s["handle"] = handle(case, s, case["op"] == "sparse")
    return s


# ---- one pass ------------------------------------------------------------------------------------

def run(s):
    return (run_own if own else run_plain)(s)


def run_own(s):
    case = s["case"]
    if case["op"] == "rope":
        from paper_2410_23079_b200 import norm_rope
        return norm_rope(s["q"], s["k"], s["positions"], s["inv_freq"], s["q_weight"], s["k_weight"], eps=EPS, interleaved=case["interleaved"])
    h = s["handle"]
    if case["op"] == "cache":
        h.append(0, s["k_new"], s["v_new"], s["lens"], s["table"], s["cu"], s["max_new"])
        h.read(0, s["lens"], s["table"], s["k_back"], s["v_back"], s["cu"], s["max_new"])
        return s["k_back"], s["v_back"]
    if case["op"] == "attend":
        h.decode(0, s["q"], s["lens"], s["table"], case["most"], s["out"], lse=s["lse"])
        return s["out"], s["lse"]
    h.select(0, s["q"], s["lens"], s["table"], case["most"], case["sink"], case["recent"], case["top"], s["selected"])
    h.decode(0, s["q"], s["lens"], s["table"], case["most"], s["out"], lse=s["lse"], selected=s["selected"])
    return s["out"], s["lse"], s["selected"]


def run_plain(s):
    return {"rope": plain_rope, "cache": plain_cache, "attend": plain_attend, "sparse": plain_sparse}[s["case"]["op"]](s)


def plain_rope(s):
    case = s["case"]
    angle = s["positions"].double().unsqueeze(1) * s["inv_freq"].double()
    cos, sin = angle.cos().float().unsqueeze(1), angle.sin().float().unsqueeze(1)
    R = case["rotary"]

    def one(x, w):
        x = x.float()
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * w.float()
        if case["interleaved"]:
            a, b = x[..., 0:R:2], x[..., 1:R:2]
            turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
        else:
            a, b = x[..., :R // 2], x[..., R // 2:R]
            turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
        return torch.cat([turned, x[..., R:]], -1).to(TYPES[case["dtype"]])

    return one(s["q"], s["q_weight"]), one(s["k"], s["k_weight"])


def plain_cache(s):
    case = s["case"]
    n = s["cu"].diff().long()
    seq = torch.repeat_interleave(torch.arange(case["batch"], device=DEV), n, output_size=s["k_new"].shape[0])
    pos = torch.arange(s["k_new"].shape[0], device=DEV) - s["cu"][seq] + s["lens"][seq] - n[seq]
    page, slot = s["table"][seq, pos // case["page"]].long(), pos % case["page"]
    back = []
    for name in ("k", "v"):
        codes, scale = quantise(s[name + "_new"].float(), case["kept"])
        if scale is None:
            s[name][0, page, :, slot] = codes
            back.append(s[name][0, page, :, slot])
            continue
        bits = s[name].view(torch.int8)
        bits[0, page, :, slot] = codes.view(torch.int8)
        s[name + "_scale"][0, page, :, slot] = scale
        back.append((bits[0, page, :, slot].view(TYPES[case["kept"]]).float() * s[name + "_scale"][0, page, :, slot].unsqueeze(-1)).to(TYPES[case["dtype"]]))
    return tuple(back)


def gather(s, name, pages):
    """fp32 rows of pages [batch, heads or 1, n], laid out [batch, heads, n * page, dim]."""
    case, pool = s["case"], s[name]
    head = torch.arange(case["kv_heads"], device=DEV).view(1, -1, 1)
    pages = pages.clamp_min(0).long()
    if case["kept"] in TOP:
        x = pool.view(torch.int8)[0][pages, head].view(pool.dtype).float()
        x *= s[name + "_scale"][0][pages, head].unsqueeze(-1)
    else:
        x = pool[0][pages, head].float()
    return x.flatten(2, 3)


def weigh(s, pages, live):
    """Softmax attention of s's queries over the pages' live tokens [batch, heads or 1, n * page]: outputs and log-sum-exps."""
    case = s["case"]
    B, H, D = case["batch"], case["kv_heads"], case["dim"]
    q = s["q"].float().view(B, H, -1, D)
    logits = (q @ gather(s, "k", pages).transpose(2, 3)) / math.sqrt(D)
    logits = torch.where(live.unsqueeze(2), logits, -math.inf)
    top = logits.amax(-1, keepdim=True)
    p = (logits - top).exp()
    total = p.sum(-1, keepdim=True)
    out = (p @ gather(s, "v", pages)) / total
    return out.view(B, -1, D).to(TYPES[case["dtype"]]), (top + total.log()).view(B, -1)


def plain_attend(s):
    P, table = s["case"]["page"], s["table"]
    live = torch.arange(table.shape[1] * P, device=DEV).view(1, 1, -1) < s["lens"].view(-1, 1, 1)
    return weigh(s, table.unsqueeze(1), live)


def plain_sparse(s):
    case, table = s["case"], s["table"]
    B, H, D, P = case["batch"], case["kv_heads"], case["dim"], case["page"]
    q = s["q"].double().view(B, H, -1, D)
    up, down = q.clamp_min(0).sum(2), q.clamp_max(0).sum(2)               # a group's queries, by sign
    low, high = s["bounds"][0][table.clamp_min(0).long()].double().unbind(3)
    score = torch.einsum("bhd,bnhd->bhn", up, high) + torch.einsum("bhd,bnhd->bhn", down, low)
    at = torch.arange(table.shape[1], device=DEV)
    count = ((s["lens"] + P - 1) // P).view(-1, 1, 1)
    score = torch.where((at < case["sink"]) | (at >= count - case["recent"]), math.inf, score)
    score = torch.where(at < count, score, -math.inf)
    most = min(case["sink"] + case["recent"] + case["top"], table.shape[1])
    best = score.sort(stable=True, dim=-1, descending=True).indices[..., :most]
    best = torch.where(best < count, best, 1 << 30).sort(-1).values
    good = best < count
    selected = torch.full_like(s["selected"], -1)
    selected[..., :most] = torch.where(good, best, -1)
    pages = table.unsqueeze(1).expand(-1, H, -1).gather(2, torch.where(good, best, 0))
    token = (best.unsqueeze(-1) * P + torch.arange(P, device=DEV)).flatten(2)
    live = (token < s["lens"].view(-1, 1, 1)) & good.repeat_interleave(P, -1)
    return weigh(s, pages, live) + (selected,)


# ---- work ----------------------------------------------------------------------------------------

def work(case):
    e = SIZE[case["dtype"]]
    D, H = case["dim"], case["kv_heads"]
    if case["op"] == "rope":
        rows = case["tokens"] * (case["q_heads"] + H)
        return {"bytes": 2 * rows * D * e + 4 * case["tokens"] + 2 * case["rotary"] + 2 * D * e, "flops": rows * (4 * D + 3 * case["rotary"])}
    kept = D * SIZE[case["kept"]] + (4 if case["kept"] in TOP else 0)
    lens = lengths(case)
    if case["op"] == "cache":
        rows = 2 * sum(lens) * H
        return {"bytes": rows * (2 * D * e + 2 * kept), "flops": 3 * rows * D}
    P = case["page"]
    pages = [-(-n // P) for n in lens]
    tokens, extra, flops = lens, 4 * sum(pages), 0
    if case["op"] == "sparse":
        most = case["sink"] + case["recent"] + case["top"]
        tokens = [min(n, most * P) for n in lens]
        middle = sum(max(0, n - case["sink"] - case["recent"]) for n in pages if n > most)
        extra += middle * H * 2 * D * e + 4 * case["batch"] * H * most
        flops = 4 * D * middle * H
    return {"bytes": sum(tokens) * H * 2 * kept + extra + case["batch"] * case["q_heads"] * (2 * D * e + 4),
            "flops": flops + 4 * D * sum(tokens) * case["q_heads"]}


# ---- values in 64 bits ---------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return {"rope": exact_rope, "cache": exact_cache, "attend": exact_attention, "sparse": exact_attention}[case["op"]](case, s)


def exact_rope(case, s):
    R, out = case["rotary"], []
    turn = torch.polar(torch.ones((), dtype=torch.float64, device=DEV), s["positions"].double()[:, None] * s["inv_freq"].double()[None])
    for x, w in ((s["q"], s["q_weight"]), (s["k"], s["k_weight"])):
        y = x.double()
        y = y * w.double() / ((y * y).sum(-1, keepdim=True) / y.shape[-1] + EPS).sqrt()
        pairs = y[..., :R].unflatten(-1, (R // 2, 2)) if case["interleaved"] else y[..., :R].unflatten(-1, (2, R // 2)).transpose(-1, -2)
        z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn[:, None])
        y[..., :R] = (z if case["interleaved"] else z.transpose(-1, -2)).flatten(-2)
        out.append(y)
    return tuple(out)


def exact_cache(case, s):
    out = []
    for x in (s["k_new"].double(), s["v_new"].double()):
        if case["kept"] in TOP:
            top = TOP[case["kept"]]
            scale = torch.clamp(x.abs().max(-1, keepdim=True).values / top, min=TINY).float().double()    # kept in 32 bits
            y = torch.clamp((x / scale).float().double(), -top, top)                                     # the quotient as well
            if case["kept"] == "i8":
                x = torch.round(y) * scale
            else:                                                          # four significant bits, down to 2^-9
                unit = torch.exp2(torch.clamp(torch.frexp(y).exponent - 1, min=-6).double() - 3)
                x = torch.round(y / unit) * unit * scale
        out.append(x)
    return tuple(out)


def exact_attention(case, s):
    B, H, D, P = case["batch"], case["kv_heads"], case["dim"], case["page"]
    outs, sums, chosen = [], [], []
    for b, n in enumerate(lengths(case)):
        count = -(-n // P)
        pages = s["table"][b, :count].long()
        q = s["q"][b].double().view(H, -1, D)
        keep = torch.ones(H, count, dtype=torch.bool, device=DEV)
        if case["op"] == "sparse":
            most = case["sink"] + case["recent"] + case["top"]
            rows = []
            for h in range(H):
                ends = s["bounds"][0, pages, h].double()                   # [pages, 2, dim]
                score = sum(torch.maximum(qq * ends[:, 0], qq * ends[:, 1]).sum(-1) for qq in q[h]).cpu().numpy()
                score[:case["sink"]] = np.inf
                score[max(0, count - case["recent"]):] = np.inf
                rows.append(np.sort(np.lexsort((np.arange(count), -score))[:most]))
            pick = torch.from_numpy(np.stack(rows)).to(DEV)
            keep = torch.zeros_like(keep).scatter_(1, pick, True)
            chosen.append(torch.cat([pick, pick.new_full((H, most - pick.shape[1]), -1)], 1).int())
        def rows_of(name):
            x = s[name][0, pages].transpose(0, 1).double() if case["kept"] not in TOP else \
                s[name][0].view(torch.int8)[pages].view(s[name].dtype).transpose(0, 1).double() * s[name + "_scale"][0, pages].transpose(0, 1)[..., None].double()
            return x.flatten(1, 2)[:, :n]
        logits = torch.einsum("hgd,hnd->hgn", q, rows_of("k")) * D ** -0.5
        logits = logits.masked_fill(~keep.repeat_interleave(P, 1)[:, None, :n], -math.inf)
        outs.append(torch.einsum("hgn,hnd->hgd", torch.softmax(logits, -1), rows_of("v")).reshape(-1, D))
        sums.append(torch.logsumexp(logits, -1).reshape(-1))
    return (torch.stack(outs), torch.stack(sums)) + ((torch.stack(chosen),) if case["op"] == "sparse" else ())
