"""The cache operators as they are measured: their cases, inputs, plain forms and definitions in 64 bits.

The cache holds keys and values in 8 bits (int8 or e4m3), in pages of `block` tokens with one scale for each page and
key head.  Four operators work on it: append (quantise new tokens into it), attend (attention of the last tokens'
queries over it, with the attention weight that each kept token received), evict (keep the tokens that received most)
and read (the values back in 16 bits).  What is held in 8 bits is returned through read, so the passes of append and
evict end with one.
"""
import random

import torch

own = False

DTYPE = {"bf16": torch.bfloat16, "fp16": torch.float16}
LARGEST_CODE = {"int8": 127.0, "e4m3": 448.0}
LEAST_EXPONENT = -100


# ---- cases ---------------------------------------------------------------------------------
def _case(name, op, batch, kv_heads, dim, block, format, type, length, **more):
    return dict(name=name, op=op, batch=batch, kv_heads=kv_heads, dim=dim, block=block, format=format, type=type,
                length=length, **more)


def listed():
    return [
        # one step of an answer over one 28x28-patch image with its CLS token; 16 heads of 64 as in the encoder
        _case("attend one, one image", "attend", 1, 16, 64, 16, "int8", "bf16", 785, heads=16, tokens=1, causal=True,
              weights=True),
        # a serving step of two dozen conversations of all lengths, grouped heads
        _case("attend one, a batch", "attend", 24, 8, 128, 64, "int8", "bf16", 8191, heads=32, tokens=1, causal=True,
              weights=True),
        # one reader of a whole slide: 512x512 patches and a question, few key heads
        _case("attend one, one long", "attend", 1, 4, 128, 128, "e4m3", "fp16", 262147, heads=32, tokens=1,
              causal=True, weights=True),
        # a full server: many long sequences
        _case("attend one, many long", "attend", 32, 8, 128, 32, "e4m3", "bf16", 16385, heads=64, tokens=1,
              causal=True, weights=True),
        # a few draft tokens checked at once over a 146x146 grid; 24 heads of 64 as in the larger encoder
        _case("attend few", "attend", 6, 8, 64, 64, "e4m3", "fp16", 21317, heads=24, tokens=5, causal=True,
              weights=False),
        # a prompt that follows an image in the cache
        _case("attend prompt", "attend", 2, 8, 128, 64, "int8", "bf16", 6001, heads=32, tokens=1501, causal=True,
              weights=True),
        # the step's new token of every conversation
        _case("append one, a batch", "append", 48, 8, 128, 64, "int8", "bf16", 4096, tokens=1),
        # images and prompts of a ragged batch
        _case("append prompt", "append", 3, 8, 128, 64, "e4m3", "bf16", 130, tokens=4099),
        # one image's cache cut to what a small reader can hold
        _case("evict one image", "evict", 1, 16, 64, 16, "int8", "bf16", 786, budget=512, first=1, last=32),
        # a batch cut to a quarter
        _case("evict a batch", "evict", 16, 8, 128, 64, "int8", "bf16", 16385, budget=4096, first=4, last=256),
        # the newest tokens of one sequence
        _case("read one", "read", 1, 8, 128, 64, "e4m3", "fp16", 65),
        # a batch's caches, to be kept elsewhere in 16 bits
        _case("read a batch", "read", 8, 8, 128, 32, "int8", "bf16", 8190),
    ]


def _log_int(rng, low, high):
    return int(round(low * (high / low) ** rng.random()))


def draw(rng):
    op = rng.choice(["attend", "attend", "attend", "attend", "append", "append", "evict", "evict", "read"])
    kv_heads, dim = rng.choice([1, 2, 3, 4, 5, 8, 12, 16]), rng.choice([64, 128])
    base = dict(op=op, kv_heads=kv_heads, dim=dim, block=rng.choice([16, 32, 64, 128]),
                format=rng.choice(["int8", "e4m3"]), type=rng.choice(["bf16", "fp16"]))
    batch = _log_int(rng, 1, 48)
    if op == "attend":
        tokens = rng.choice([1, 1, 1, rng.randint(2, 16), _log_int(rng, 17, 1500)])
        group = rng.choice([1, 2, 3, 4, 6, 8, 16])
        case = dict(base, batch=batch, heads=kv_heads * group, tokens=tokens,
                    length=max(tokens, _log_int(rng, 60, 262144)), causal=rng.random() < 0.7,
                    weights=rng.random() < 0.6)
    elif op == "append":
        case = dict(base, batch=batch, tokens=rng.choice([1, rng.randint(2, 16), _log_int(rng, 17, 4100)]),
                    length=_log_int(rng, 1, 2000))
    else:
        case = dict(base, batch=batch, length=_log_int(rng, 40, 32768))
    most = [work(c) for c in listed() if c["op"] == op]
    share = rng.uniform(0.1, 0.9)
    while True:
        if op == "evict":
            case["budget"] = max(1, int(case["length"] * share))
            case["first"] = min(4, case["budget"] // 8)
            case["last"] = case["budget"] // 16
        # no more bytes than the operator's largest listed case, and no more products
        w = work(case)
        if all(w[m] <= max(x[m] for x in most) for m in w):
            return case
        if case["batch"] > 1:
            case["batch"] = (case["batch"] + 1) // 2
        elif case["length"] > 2 * case.get("tokens", 1):
            case["length"] //= 2
        else:
            case["tokens"] //= 2


def _lengths(case):
    """The sequences' lengths: the case's own for the first, a twentieth of it and more for the others."""
    r = random.Random("%d %d %d" % (case["batch"], case["length"], case["kv_heads"]))
    low = case.get("tokens", 1) if case["op"] == "attend" else 1
    return [case["length"]] + [max(low, int(case["length"] * r.uniform(0.05, 1.0))) for _ in range(case["batch"] - 1)]


def _counts(case):
    """New tokens of each sequence: a prompt batch is padded to its longest."""
    n = case.get("tokens", 1)
    r = random.Random("%d %d" % (case["batch"], n))
    return [n] + [n if n < 17 else max(1, int(n * r.uniform(0.3, 1.0))) for _ in range(case["batch"] - 1)]


def _blocks(n, block):
    return (n + block - 1) // block


# ---- inputs --------------------------------------------------------------------------------
def _power_of_two_scale(largest, format):
    """The smallest power of two s with largest <= (largest code) * s."""
    mantissa, exponent = torch.frexp(largest.float())
    edge, step = (127 / 128, 7) if format == "int8" else (0.875, 9)
    exponent = exponent - step + (mantissa > edge).to(exponent.dtype)
    exponent = torch.where(largest > 0, exponent, torch.full_like(exponent, LEAST_EXPONENT))
    return ((exponent.clamp(min=LEAST_EXPONENT).int() + 127) << 23).view(torch.float32)  # 2^exponent, exactly


def _to_codes(x, format):
    if format == "int8":
        return torch.round(x).clamp(-127, 127).to(torch.int8)
    return x.clamp(-448, 448).to(torch.float8_e4m3fn)


def _pool(case, pages, g, spread):
    """Codes and scales of a pool of pages: normal values, some channels larger than others as in trained keys."""
    h, blk, d = case["kv_heads"], case["block"], case["dim"]
    codes = torch.empty((pages, h, blk, d), device="cuda",
                        dtype=torch.int8 if case["format"] == "int8" else torch.float8_e4m3fn)
    scale = torch.empty((pages, h), device="cuda")
    channel = torch.exp(spread * torch.randn((1, h, 1, d), device="cuda", generator=g))
    part = max(1, (1 << 26) // (h * blk * d))
    for p in range(0, pages, part):
        n = min(part, pages - p)
        x = channel * torch.randn((n, h, blk, d), device="cuda", generator=g)
        s = _power_of_two_scale(x.abs().amax((2, 3)), case["format"])
        codes[p:p + n] = _to_codes(x / s[:, :, None, None], case["format"])
        scale[p:p + n] = s
    return codes, scale


def _table(lengths, block, columns, at, order):
    """[batch, columns] pages; the entries behind a sequence's last page are -1."""
    rows = []
    for n in lengths:
        used = _blocks(n, block)
        rows.append(order[at:at + used] + [-1] * (columns - used))
        at += used
    return torch.tensor(rows, dtype=torch.int32, device="cuda"), at


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    host = random.Random(seed)
    op, b, h, d, blk = case["op"], case["batch"], case["kv_heads"], case["dim"], case["block"]
    dtype = DTYPE[case["type"]]
    lengths, counts = _lengths(case), _counts(case)
    held = [n + c for n, c in zip(lengths, counts)] if op == "append" else lengths
    budget = case.get("budget", 0)
    survivors = [min(n, budget) for n in lengths] if op == "evict" else []
    used = sum(_blocks(n, blk) for n in held) + sum(_blocks(n, blk) for n in survivors)
    order = list(range(used + 3))  # a few pages of the pool belong to nobody
    host.shuffle(order)
    s = dict(case=case)
    s["k"], s["k_scale"] = _pool(case, len(order), g, 0.4)
    s["v"], s["v_scale"] = _pool(case, len(order), g, 0.1)
    columns = _blocks(max(held), blk)
    s["table"], at = _table(held, blk, columns, 0, order)
    s["lengths"] = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    ragged = any(c != counts[0] for c in counts)
    s["counts"] = torch.tensor(counts, dtype=torch.int32, device="cuda") if ragged else None
    if op == "attend":
        n, heads = case["tokens"], case["heads"]
        # the projection's output holds q, k and v of a token side by side; the operator is given the view of q
        fused = torch.randn((b, n, heads + 2 * h, d), device="cuda", generator=g) * 1.5
        s["q"] = fused.to(dtype)[:, :, :heads]
        s["out"] = torch.zeros((b, n, heads, d), dtype=dtype, device="cuda")
        if case["weights"]:
            s["weights_in"] = torch.rand((b, h, case["length"]), device="cuda", generator=g) ** 4
            s["weights_out"] = torch.zeros((b, h, case["length"]), device="cuda")
    elif op == "append":
        n = case["tokens"]
        fused = torch.randn((b, n, 4 * h, d), device="cuda", generator=g)
        fused *= torch.exp(0.3 * torch.randn((b, n, 1, 1), device="cuda", generator=g))
        fused = fused.to(dtype)
        s["new_k"], s["new_v"] = fused[:, :, 2 * h:3 * h], fused[:, :, 3 * h:]
        first = [n // blk * blk for n in lengths]
        rows = max(n - f for n, f in zip(held, first))
        s["read_first"] = torch.tensor(first, dtype=torch.int32, device="cuda")
        s["read_count"] = torch.tensor([n - f for n, f in zip(held, first)], dtype=torch.int32, device="cuda")
    elif op == "evict":
        w = torch.exp(2 * torch.randn((b, h, case["length"]), device="cuda", generator=g))
        w[torch.rand(w.shape, device="cuda", generator=g) < 0.2] = 0.0  # never attended in 32 bits: ties
        s["weights_in"] = w
        s["weights_out"] = torch.zeros((b, h, budget), device="cuda")
        s["kept"] = torch.zeros((b, h, budget), dtype=torch.int32, device="cuda")
        s["new_lengths"] = torch.zeros((b,), dtype=torch.int32, device="cuda")
        s["to"], at = _table(survivors, blk, _blocks(budget, blk), at, order)
        rows = min(budget, max(lengths))
    else:
        rows = max(lengths)
    if op != "attend":
        s["k_out"] = torch.zeros((b, rows, h, d), dtype=dtype, device="cuda")
        s["v_out"] = torch.zeros((b, rows, h, d), dtype=dtype, device="cuda")
    return s


# ---- the framework's calls -----------------------------------------------------------------
_contexts = {}


def _run_own(s):
    import paper_2601_12150_b200 as spv
    ctx = _contexts.get(0)
    if ctx is None:
        ctx = _contexts[0] = spv.Context(0)
    cache = s.get("cache")
    if cache is None:  # the handle that a program keeps beside its pool
        cache = s["cache"] = spv.KvCache(s["k"], s["v"], s["k_scale"], s["v_scale"])
    op = s["case"]["op"]
    if op == "attend":
        w_out = s.get("weights_out")
        ctx.kv_cache_attention(cache, s["q"], s["table"], s["lengths"], counts=s["counts"],
                               causal=s["case"]["causal"], out=s["out"], weights_in=s.get("weights_in"),
                               weights_out=w_out)
        return {"out": s["out"]} if w_out is None else {"out": s["out"], "weights": w_out}
    if op == "append":
        ctx.kv_cache_append(cache, s["new_k"], s["new_v"], s["table"], s["lengths"], counts=s["counts"])
        ctx.kv_cache_read(cache, s["table"], s["read_count"], first=s["read_first"], k_out=s["k_out"],
                          v_out=s["v_out"])
        return {"k": s["k_out"], "v": s["v_out"]}
    if op == "evict":
        ctx.kv_cache_evict(cache, s["weights_in"], s["table"], s["lengths"], s["case"]["budget"],
                           keep_first=s["case"]["first"], keep_last=s["case"]["last"], dst_table=s["to"],
                           kept=s["kept"], weights_out=s["weights_out"], new_lengths=s["new_lengths"])
        ctx.kv_cache_read(cache, s["to"], s["new_lengths"], k_out=s["k_out"], v_out=s["v_out"])
        return {"kept": s["kept"], "lengths": s["new_lengths"], "weights": s["weights_out"], "k": s["k_out"],
                "v": s["v_out"]}
    ctx.kv_cache_read(cache, s["table"], s["lengths"], k_out=s["k_out"], v_out=s["v_out"])
    return {"k": s["k_out"], "v": s["v_out"]}


# ---- the plain forms -----------------------------------------------------------------------
def _values(codes, scale, table):
    """[batch, heads, slots, dim] in 32 bits: what the pages of a table stand for."""
    page = table.clamp(min=0).long()
    x = codes[page].float() * scale[page][..., None, None]
    b, c, h, blk, d = x.shape
    return x.permute(0, 2, 1, 3, 4).reshape(b, h, c * blk, d)


def _per_sequence(s, name, otherwise):
    t = s[name]
    return torch.full_like(s["lengths"], otherwise) if t is None else t


def _plain_attend(s):
    case, q = s["case"], s["q"].float()
    b, n, heads, d = q.shape
    h = case["kv_heads"]
    group = heads // h
    k = _values(s["k"], s["k_scale"], s["table"])
    rows = q.reshape(b, n, h, group, d).permute(0, 2, 1, 3, 4).reshape(b, h, n * group, d) * d ** -0.5
    z = torch.matmul(rows, k.transpose(2, 3)).view(b, h, n, group, -1)
    del k
    slot = torch.arange(z.shape[-1], device=q.device)
    query = torch.arange(n, device=q.device)
    length, count = s["lengths"].long(), _per_sequence(s, "counts", n).long()
    end = length[:, None].expand(b, n)
    if case["causal"]:
        end = torch.minimum(end, (length - count)[:, None] + query + 1)
    given = query < count[:, None]
    seen = (slot < end[:, :, None]) & given[:, :, None]
    seen = seen[:, None, :, None]
    z = z.masked_fill_(~seen, float("-inf"))
    top = z.amax(-1, keepdim=True)
    top = torch.where(torch.isinf(top), torch.zeros_like(top), top)
    p = z.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    p = p.div_(torch.where(total > 0, total, torch.ones_like(total)))
    v = _values(s["v"], s["v_scale"], s["table"]).masked_fill_((slot >= length[:, None])[:, None, :, None], 0.0)
    out = torch.matmul(p.view(b, h, n * group, -1), v)
    out = out.view(b, h, n, group, d).permute(0, 2, 1, 3, 4).reshape(b, n, heads, d).to(s["q"].dtype)
    if not case["weights"]:
        return {"out": out}
    w = p.sum((2, 3))[:, :, :case["length"]] + s["weights_in"]
    w = torch.where((slot[:case["length"]] < length[:, None])[:, None], w, torch.zeros_like(w))
    return {"out": out, "weights": w}


def _quantised(x, valid, format):
    """Values of x [..., block, dim] after it went through 8 bits with one scale for the valid rows of a block."""
    x = torch.where(valid[..., None], x, torch.zeros_like(x))
    scale = _power_of_two_scale(x.abs().amax((-2, -1)), format)[..., None, None]
    return _to_codes(x / scale, format).float() * scale


def _plain_append(s):
    case = s["case"]
    b, n, h, d = s["new_k"].shape
    blk, format = case["block"], case["format"]
    length, count = s["lengths"].long(), _per_sequence(s, "counts", n).long()
    offset = length % blk
    rows = s["k_out"].shape[1]
    blocks = _blocks(rows, blk)
    at = torch.arange(blocks * blk, device=length.device) - offset[:, None]  # new token of each row
    new = (at >= 0) & (at < count[:, None])
    old = at < 0
    pick = at.clamp(0, n - 1)[:, :, None, None].expand(b, blocks * blk, h, d)
    page = s["table"].long().gather(1, (length // blk)[:, None].clamp(max=s["table"].shape[1] - 1))[:, 0].clamp(min=0)
    result = {}
    for name in ("k", "v"):
        x = s["new_" + name].float().gather(1, pick)
        x = torch.where(new[:, :, None, None], x, torch.zeros_like(x)).view(b, blocks, blk, h, d)
        scale = _power_of_two_scale(x.abs().amax((2, 4)), format)
        before = torch.where((offset > 0)[:, None], s[name + "_scale"][page], scale[:, 0])
        scale[:, 0] = torch.maximum(scale[:, 0], before)
        kept = s[name][page].float().permute(0, 2, 1, 3) * before[:, None, :, None]
        x[:, 0] = torch.where(old[:, :blk, None, None], kept, x[:, 0])
        scale = scale[:, :, None, :, None]
        x = (_to_codes(x / scale, format).float() * scale).view(b, blocks * blk, h, d)
        x = torch.where((new | old)[:, :, None, None], x, torch.zeros_like(x))
        result[name] = x[:, :rows].to(s["new_k"].dtype)
    return result


def _plain_evict(s):
    case = s["case"]
    blk, budget, format = case["block"], case["budget"], case["format"]
    w = s["weights_in"]
    b, h, most = w.shape
    length = s["lengths"].long()[:, None, None]
    slot = torch.arange(most, device=w.device)
    w = torch.where(torch.isnan(w), torch.full_like(w, -3e38), w)
    w = torch.where((slot < case["first"]) | (slot >= length - case["last"]), torch.full_like(w, float("inf")), w)
    w = torch.where(slot < length, w, torch.full_like(w, float("-inf")))
    best = torch.sort(w, dim=-1, descending=True, stable=True).indices[:, :, :budget]
    survivors = length.clamp(max=budget)
    rank = torch.arange(best.shape[-1], device=w.device)
    kept = torch.where(rank < survivors, best, torch.full_like(best, most)).sort(-1).values
    valid = rank < survivors
    pick = torch.where(valid, kept, torch.zeros_like(kept))
    result = {"lengths": survivors.view(b).int()}
    result["kept"] = torch.full_like(s["kept"], -1)
    result["kept"][:, :, :best.shape[-1]] = torch.where(valid, kept, torch.full_like(kept, -1)).int()
    result["weights"] = torch.zeros_like(s["weights_out"])
    result["weights"][:, :, :best.shape[-1]] = torch.where(valid, s["weights_in"].gather(2, pick),
                                                           torch.zeros_like(s["weights_out"][:, :, :best.shape[-1]]))
    page = s["table"].long().clamp(min=0)[:, None].expand(b, h, -1).gather(2, pick // blk)
    head = torch.arange(h, device=w.device)[:, None]
    rows = s["k_out"].shape[1]
    room = _blocks(rows, blk) * blk
    inside = torch.zeros((b, h, room), dtype=torch.bool, device=w.device)
    inside[:, :, :rows] = valid[:, :, :rows]
    for name in ("k", "v"):
        x = torch.zeros((b, h, room, case["dim"]), device=w.device)
        x[:, :, :rows] = (s[name][page, head, pick % blk].float() * s[name + "_scale"][page, head][..., None])[:, :, :rows]
        x = _quantised(x.view(b, h, -1, blk, case["dim"]), inside.view(b, h, -1, blk), format)
        result[name] = x.view(b, h, room, -1)[:, :, :rows].transpose(1, 2).contiguous().to(s["k_out"].dtype)
    return result


def _plain_read(s):
    rows = s["k_out"].shape[1]
    inside = (torch.arange(rows, device="cuda") < s["lengths"][:, None])[:, :, None, None]
    result = {}
    for name in ("k", "v"):
        x = _values(s[name], s[name + "_scale"], s["table"])[:, :, :rows].transpose(1, 2)
        result[name] = torch.where(inside, x, torch.zeros_like(x)).to(s["k_out"].dtype)
    return result


def run(state):
    if own:
        return _run_own(state)
    return {"attend": _plain_attend, "append": _plain_append, "evict": _plain_evict,
            "read": _plain_read}[state["case"]["op"]](state)


# ---- what a pass cannot do without ---------------------------------------------------------
def work(case):
    h, d = case["kv_heads"], case["dim"]
    lengths, counts = _lengths(case), _counts(case)
    tokens = sum(lengths)
    if case["op"] == "attend":
        pairs = 0
        for length, n in zip(lengths, counts):
            pairs += n * length - (n * (n - 1) // 2 if case["causal"] else 0)
        rows = sum(counts) * case["heads"] * d
        moved = 2 * tokens * h * d + 8 * h * sum(_blocks(n, case["block"]) for n in lengths) + 4 * rows
        return {"bytes": moved + (8 * tokens * h if case["weights"] else 0), "flops": 4 * d * case["heads"] * pairs}
    if case["op"] == "append":  # 16 bits in, 8 bits into the cache, 16 bits read back
        return {"bytes": sum(counts) * h * d * 2 * (2 + 1 + 2), "flops": 4 * sum(counts) * h * d}
    if case["op"] == "evict":
        left = sum(min(n, case["budget"]) for n in lengths)
        return {"bytes": 4 * tokens * h + left * h * (8 + 2 * d * (1 + 1 + 2)), "flops": 4 * left * h * d}
    return {"bytes": tokens * h * d * 2 * (1 + 2), "flops": 2 * tokens * h * d}


# ---- the definitions in 64 bits ------------------------------------------------------------
def _slots64(codes, scale, pages, slots, block, head):
    """[len(slots), dim]: the values of some slots of one sequence and head."""
    page = pages[slots // block]
    return codes.view(torch.uint8)[page, head, slots % block].view(codes.dtype).double() * scale[page, head].double()[:, None]


def _scale64(largest, format):
    """By trial: the first power of two from below that is large enough."""
    e = LEAST_EXPONENT if largest == 0 else max(LEAST_EXPONENT, int(torch.log2(largest / LARGEST_CODE[format])) - 2)
    while float(largest) > LARGEST_CODE[format] * 2.0 ** e:
        e += 1
    return 2.0 ** e


def _round64(x, format):
    """Nearest code value, ties to even; |x| is at most the largest code."""
    if format == "int8":
        return torch.round(x)
    step = torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))).long() - 3  # four significant bits, 2^-9 and more
    power = [((1023 + e) << 52).view(torch.float64) for e in (-step, step)]  # exact, as a power function need not be
    return torch.round(x * power[0]) * power[1]


def _attend64(s):
    case, q = s["case"], s["q"].double()
    b, n, heads, d = q.shape
    h = case["kv_heads"]
    group = heads // h
    out = torch.zeros((b, n, heads, d), dtype=torch.float64, device="cuda")
    weights = torch.zeros((b, h, case["length"]), dtype=torch.float64, device="cuda")
    for i, (length, count) in enumerate(zip(_lengths(case), _counts(case))):
        pages, slots = s["table"][i].long(), torch.arange(length, device="cuda")
        for j in range(h):
            k = _slots64(s["k"], s["k_scale"], pages, slots, case["block"], j)
            v = _slots64(s["v"], s["v_scale"], pages, slots, case["block"], j)
            z = torch.einsum("ngd,sd->gns", q[i, :count, j * group:(j + 1) * group], k) / d ** 0.5
            if case["causal"]:
                last = length - count + torch.arange(count, device="cuda")
                z = torch.where(slots[None] <= last[:, None], z, float("-inf"))
            p = torch.softmax(z, -1)
            out[i, :count, j * group:(j + 1) * group] = torch.einsum("gns,sd->ngd", p, v)
            if case["weights"]:
                weights[i, j, :length] = s["weights_in"][i, j, :length].double() + p.sum((0, 1))
    return {"out": out, "weights": weights} if case["weights"] else {"out": out}


def _append64(s):
    case, format, blk = s["case"], s["case"]["format"], s["case"]["block"]
    result = {}
    for name in ("k", "v"):
        out = torch.zeros(s["k_out"].shape, dtype=torch.float64, device="cuda")
        new = s["new_" + name].double()
        for i, (length, count) in enumerate(zip(_lengths(case), _counts(case))):
            pages, start = s["table"][i].long(), length // blk * blk
            for j in range(case["kv_heads"]):
                x = new[i, :count, j]
                before = torch.arange(start, length, device="cuda")
                if len(before):
                    x = torch.cat([_slots64(s[name], s[name + "_scale"], pages, before, blk, j), x])
                for r in range(0, len(x), blk):
                    part = x[r:r + blk]
                    if r == 0 and len(before):
                        scale = max(_scale64(part[len(before):].abs().max(), format),
                                    float(s[name + "_scale"][pages[start // blk], j]))
                    else:
                        scale = _scale64(part.abs().max(), format)
                    out[i, r:r + blk, j][:len(part)] = _round64(part / scale, format) * scale
        result[name] = out
    return result


def _evict64(s):
    case, format, blk = s["case"], s["case"]["format"], s["case"]["block"]
    b, h, budget = s["kept"].shape
    kept_all = torch.full((b, h, budget), -1, dtype=torch.int32, device="cuda")
    weights = torch.zeros((b, h, budget), dtype=torch.float64, device="cuda")
    values = {m: torch.zeros(s["k_out"].shape, dtype=torch.float64, device="cuda") for m in ("k", "v")}
    lengths = _lengths(case)
    for i, length in enumerate(lengths):
        n = min(length, budget)
        pages = s["table"][i].long()
        for j in range(h):
            w = s["weights_in"][i, j, :length].double().cpu().tolist()
            middle = sorted(range(case["first"], length - case["last"]), key=lambda t: (-w[t], t)) if n < length else []
            ends = set(range(min(case["first"], length))) | set(range(max(0, length - case["last"]), length))
            chosen = range(length) if n == length else sorted(ends | set(middle[:n - len(ends)]))
            kept = torch.tensor(list(chosen), device="cuda")
            kept_all[i, j, :n] = kept.int()
            weights[i, j, :n] = s["weights_in"][i, j, kept].double()
            for m in ("k", "v"):
                x = _slots64(s[m], s[m + "_scale"], pages, kept, blk, j)
                room = torch.zeros((_blocks(n, blk) * blk, case["dim"]), dtype=torch.float64, device="cuda")
                room[:n] = x
                room = room.view(-1, blk, case["dim"])
                largest = room.abs().amax((1, 2)).cpu()
                scale = torch.tensor([_scale64(a, format) for a in largest], dtype=torch.float64, device="cuda")[:, None, None]
                values[m][i, :n, j] = (_round64(room / scale, format) * scale).view(-1, case["dim"])[:n]
    return {"kept": kept_all, "lengths": torch.tensor([min(n, budget) for n in lengths], dtype=torch.int32),
            "weights": weights, "k": values["k"], "v": values["v"]}


def _read64(s):
    case, result = s["case"], {}
    for name in ("k", "v"):
        out = torch.zeros(s["k_out"].shape, dtype=torch.float64, device="cuda")
        for i, length in enumerate(_lengths(case)):
            slots = torch.arange(length, device="cuda")
            for j in range(case["kv_heads"]):
                out[i, :length, j] = _slots64(s[name], s[name + "_scale"], s["table"][i].long(), slots, case["block"], j)
        result[name] = out
    return result


def exact(case, seed):
    if case["op"] == "append" and case["batch"] * case["kv_heads"] * _blocks(case["tokens"] + case["block"], case["block"]) > 20000:
        return None  # block by block on the host: too slow for very many blocks
    if case["op"] == "evict" and sum(_lengths(case)) * case["kv_heads"] > 3_000_000:
        return None  # sorted on the host: too slow for very many tokens
    s = prepare(case, seed)
    return {"attend": _attend64, "append": _append64, "evict": _evict64, "read": _read64}[case["op"]](s)
