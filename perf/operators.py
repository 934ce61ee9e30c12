"""Attention over observation histories: over whole prompts of packed environments, of new tokens over a paged cache of
keys / values, and the cache itself, written (in 32, 16 or 8 bits) and read back -- each in its plain form of elementary
torch operations, and (own = True) through the public entry points of the library."""
import math

import torch

own = False

DT = {"fp32": torch.float32, "bf16": torch.bfloat16}
PAGE = 64                     # tokens of a page where a case does not say


def listed():
    return [
        # the first observation of one robot: 64 tokens, the head shape of a 512-wide network -- latency
        {"name": "prompt_robot_1", "op": "prompt", "type": "fp32", "heads": 8, "kv": 8, "dim": 64, "B": 1, "lo": 64, "hi": 64, "past": 0},
        # the first observations of a fleet, ragged, some of one token
        {"name": "prompt_fleet_256", "op": "prompt", "type": "bf16", "heads": 8, "kv": 8, "dim": 64, "B": 256, "lo": 1, "hi": 191, "past": 0},
        # fp32 histories of a few environments, grouped heads
        {"name": "prompt_fp32_4", "op": "prompt", "type": "fp32", "heads": 8, "kv": 2, "dim": 64, "B": 4, "lo": 301, "hi": 1501, "past": 0},
        # a chunk of new observations behind the history read back from a cache
        {"name": "prompt_chunk_16", "op": "prompt", "type": "bf16", "heads": 16, "kv": 4, "dim": 128, "B": 16, "lo": 65, "hi": 257, "past": 2000},
        # whole episodes in one pass, the largest product
        {"name": "prompt_long_2", "op": "prompt", "type": "bf16", "heads": 32, "kv": 8, "dim": 128, "B": 2, "lo": 5003, "hi": 8192, "past": 0},
        # a control step of a batch: one new token an environment into an 8-bit cache, and back
        {"name": "store_step_64", "op": "store", "type": "bf16", "held": "mx8", "kv": 8, "dim": 64, "B": 64, "lo": 1, "hi": 1, "past": 700, "back": 0},
        # fp32 histories of odd lengths kept as they are, and read back with the tokens before them
        {"name": "store_fp32_16", "op": "store", "type": "fp32", "held": "fp32", "kv": 4, "dim": 32, "B": 16, "lo": 1, "hi": 701, "past": 300, "back": 300},
        # whole episodes into an 8-bit cache, and back
        {"name": "store_long_8", "op": "store", "type": "bf16", "held": "mx8", "kv": 8, "dim": 128, "B": 8, "lo": 9001, "hi": 16384, "past": 0, "back": 0},
        # one robot's control step on its history of eleven observations -- latency
        {"name": "paged_robot_1", "op": "paged", "type": "fp32", "held": "fp32", "heads": 8, "kv": 8, "dim": 64, "B": 1, "tokens": 1, "lo": 700, "hi": 700},
        # a control step of a fleet, ragged histories, grouped heads
        {"name": "paged_fleet_256", "op": "paged", "type": "bf16", "held": "bf16", "heads": 8, "kv": 2, "dim": 64, "B": 256, "tokens": 1, "lo": 1, "hi": 2001},
        # few environments with very long histories in 8 bits
        {"name": "paged_long_8", "op": "paged", "type": "bf16", "held": "mx8", "heads": 32, "kv": 8, "dim": 128, "B": 8, "tokens": 1, "lo": 20001, "hi": 131072},
        # the 64 observation tokens of width 768 that condition a network, pooled from each environment's 8-bit history
        {"name": "paged_observe_32", "op": "paged", "type": "bf16", "held": "mx8", "heads": 12, "kv": 4, "dim": 64, "B": 32, "tokens": 64, "lo": 501, "hi": 4000,
         "all": True, "out": "fp32"},
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    op = rng.choice(["prompt", "store", "paged"])
    kv = rng.choice([1, 2, 3, 4, 6, 8])
    case = {"op": op, "kv": kv, "dim": rng.choice([32, 64, 128])}
    if op != "store":
        case["heads"] = kv * rng.choice([g for g in (1, 2, 3, 4, 6, 8) if kv * g <= 32])
    case["type"] = rng.choice(["fp32", "bf16", "bf16"])
    if op == "prompt":
        case["B"] = _log_int(rng, 1, 256)
        case["hi"] = _log_int(rng, 1, min(8192, 32768 // case["B"]))
        case["past"] = rng.choice([0, 0, _log_int(rng, 1, min(8192, 32768 // case["B"]))])
        # no more products than the largest listed case has with every sequence as long as the longest, half of them in fp32
        while case["heads"] * case["dim"] * case["B"] * case["hi"] * (case["hi"] + case["past"]) > (1 << 38 if case["type"] == "bf16" else 1 << 37):
            case["hi"], case["past"] = case["hi"] * 3 // 4, case["past"] * 3 // 4
        case["lo"] = _log_int(rng, 1, case["hi"])
        case["all"] = rng.random() < 0.25
    elif op == "store":
        case["held"] = rng.choice([case["type"], "mx8", "mx8"])
        case["B"] = _log_int(rng, 1, 1024)
        case["hi"] = _log_int(rng, 1, max(2, min(16384, 65536 // case["B"])))
        case["lo"] = _log_int(rng, 1, case["hi"])
        case["past"] = rng.choice([0, rng.randint(1, 200)])
        case["back"] = rng.choice([0, case["past"]])
        case["page"] = rng.choice([16, 32, 64, 128, 256])
    else:
        case["held"] = rng.choice([case["type"], "mx8"])
        case["B"] = _log_int(rng, 1, 256)
        case["tokens"] = rng.choice([1, 1, 1, rng.randint(2, 64)])
        case["hi"] = _log_int(rng, case["tokens"], max(case["tokens"] + 1, min(65536, (262144 if case["tokens"] == 1 else 32768) // case["B"])))
        case["lo"] = _log_int(rng, 1, case["hi"])
        case["all"] = rng.random() < 0.3
        case["out"] = rng.choice([case["type"], "fp32"])
        case["page"] = rng.choice([16, 32, 64, 128, 256])
    return case


def _lengths(case):
    """lo .. hi, spread by the golden ratio; the longest is hi."""
    lo, hi, B = case["lo"], case["hi"], case["B"]
    return [hi] + [lo + int((hi - lo) * ((i * 0.6180339887498949) % 1.0)) for i in range(1, B)]


def _visible(nq, nk, every):
    if every:
        return nq * nk
    first = nk - nq + 1                                   # keys that the first query sees
    return sum(max(0, first + i) for i in range(nq)) if first < 0 else nq * first + nq * (nq - 1) // 2


def _held_bytes(held, dim):
    return {"fp32": 4 * dim, "bf16": 2 * dim, "mx8": dim + dim // 32}[held]


def work(case):
    n, dim, every = _lengths(case), case["dim"], bool(case.get("all"))
    size = 4 if case["type"] == "fp32" else 2
    if case["op"] == "prompt":
        q, k = sum(n), sum(n) + case["past"] * case["B"]
        pairs = sum(_visible(x, x + case["past"], every) for x in n)
        return {"bytes": size * dim * (2 * q * case["heads"] + 2 * k * case["kv"]), "flops": 4 * dim * case["heads"] * pairs}
    if case["op"] == "store":
        new, back = sum(n), sum(n) + case["back"] * case["B"]
        return {"bytes": 2 * case["kv"] * (new + back) * (size * dim + _held_bytes(case["held"], dim)), "flops": 0}
    t, out = case["tokens"], 4 if case.get("out", case["type"]) == "fp32" else 2
    pairs = sum(_visible(t, x, every) for x in n)
    return {"bytes": 2 * case["kv"] * sum(n) * _held_bytes(case["held"], dim) + case["B"] * t * case["heads"] * dim * (size + out),
            "flops": 4 * dim * case["heads"] * pairs}


def _ptr(n, dev):
    return torch.tensor([sum(n[:i]) for i in range(len(n) + 1)] if len(n) < 64 else [0] + torch.tensor(n).cumsum(0).tolist(),
                        dtype=torch.int32, device=dev)


def prepare(case, seed):
    dev = "cuda"
    g = torch.Generator(device=dev)
    g.manual_seed(seed * 1000003 + 17)
    n, dim, kv, B = _lengths(case), case["dim"], case["kv"], case["B"]
    dt = DT[case["type"]]
    normal = lambda *s: torch.randn(*s, generator=g, device=dev)  # noqa: E731
    # a few channels of keys are large, as learned keys have them; values are even
    channel = torch.exp(0.5 * normal(kv, dim))
    key = lambda rows: (normal(rows, kv, dim) * channel).to(dt)  # noqa: E731
    s = {"case": case, "scale": dim ** -0.5, "longest": max(n)}
    if case["op"] == "prompt":
        total = sum(n)
        nk = [x + case["past"] for x in n]
        s.update(q_ptr=_ptr(n, dev), k_ptr=_ptr(nk, dev), longest_k=max(nk), q=normal(total, case["heads"], dim).to(dt),
                 k=key(sum(nk)), v=normal(sum(nk), kv, dim).to(dt))
        return s
    page = case.get("page", PAGE)
    have = [x + case.get("past", 0) for x in n]
    columns = -(-max(have) // page)
    pages = B * columns
    s["table"] = torch.randperm(pages, generator=g, device=dev).to(torch.int32).reshape(B, columns).contiguous()
    shape = (pages, kv, page, dim)
    s["pool"] = []
    for large in (channel[:, None, :], 1.0):
        x = normal(*shape) * large
        if case["held"] == "mx8":
            s["pool"].append(_to_mx8(x))
        else:
            s["pool"].append((x.to(DT[case["held"]]), None))
        del x
    if case["op"] == "store":
        s.update(row_ptr=_ptr(n, dev), start=torch.full((B,), case["past"], dtype=torch.int32, device=dev),
                 k=key(sum(n)), v=normal(sum(n), kv, dim).to(dt), total=sum(n))
        back = [x + case["back"] for x in n]
        s.update(back_ptr=_ptr(back, dev), back_start=torch.full((B,), case["past"] - case["back"], dtype=torch.int32, device=dev),
                 back_total=sum(back))
        return s
    s.update(q=normal(B * case["tokens"], case["heads"], dim).to(dt), length=torch.tensor(n, dtype=torch.int32, device=dev))
    return s


# ---- plain forms


def _exponent(amax):
    """Byte of the power-of-two scale of a block whose largest magnitude is amax: the smallest with amax <= 448 * 2^e."""
    bits = amax.view(torch.int32)
    e = ((bits >> 23) & 255) - 8 + ((bits & 0x7FFFFF) > 0x600000).to(torch.int32)
    return e.clamp(16, 254)                       # what is far below 2^-111 is held as a part of that


def _power(byte):
    return (byte.to(torch.int32) << 23).view(torch.float32)


def _to_mx8(x):
    """x [..., dim] fp32 -> (e4m3 bits, scale bytes), blocks of 32."""
    b = x.reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    e = _exponent(b.abs().amax(-1))
    q = (b * _power(254 - e)[..., None]).to(torch.float8_e4m3fn)
    return q.reshape(x.shape).view(torch.uint8), e.to(torch.uint8)


def _values(pool, scale):
    """What a cache holds, in fp32."""
    if scale is None:
        return pool.float()
    x = pool.view(torch.float8_e4m3fn).float()
    return (x.reshape(*scale.shape, 32) * _power(scale)[..., None]).reshape(x.shape)


def _softmax_product(q, k, v, seen):
    """q [B, kv, G, nq, dim], k / v [B, kv, nk, dim], seen [B, nq, nk]: attention in fp32."""
    B, kv, G, nq, dim = q.shape
    s = torch.matmul(q.reshape(B, kv, G * nq, dim), k.transpose(-1, -2).contiguous()).reshape(B, kv, G, nq, -1)
    s.masked_fill_(~seen[:, None, None], -math.inf)
    top = s.amax(-1, keepdim=True)
    s.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    total = s.sum(-1, keepdim=True)
    o = torch.matmul(s.reshape(B, kv, G * nq, -1), v).reshape(B, kv, G, nq, dim)
    return o / torch.where(total == 0, 1.0, total)


def _seen(nq, nk, Lq, Lk, every):
    """[B, Lq, Lk]: which keys a query sees; nq, nk [B]."""
    i = torch.arange(Lq, device=nq.device)[None, :, None]
    j = torch.arange(Lk, device=nq.device)[None, None, :]
    last = nk[:, None, None] if every else nk[:, None, None] - nq[:, None, None] + 1 + i
    return (j < last) & (j < nk[:, None, None]) & (i < nq[:, None, None])


def _padded(x, ptr, longest):
    """Packed rows [rows, heads, dim] as [B, longest, heads, dim] in fp32, zeros behind each sequence."""
    at = ptr[:-1, None].long() + torch.arange(longest, device=x.device)
    return torch.where((at < ptr[1:, None])[..., None, None], x.float()[at.clamp(max=x.shape[0] - 1)], 0.0)


def _where(ptr, rows):
    """Sequence and place in it of every packed row."""
    r = torch.arange(rows, dtype=ptr.dtype, device=ptr.device)
    b = torch.searchsorted(ptr, r, right=True) - 1
    return b, r - ptr[b]


def _plain_prompt(s):
    case, q = s["case"], s["q"]
    G, kv, dim = case["heads"] // case["kv"], case["kv"], case["dim"]
    qp = _padded(q, s["q_ptr"], s["longest"]) * s["scale"]
    qp = qp.reshape(*qp.shape[:2], kv, G, dim).permute(0, 2, 3, 1, 4)
    kp, vp = (_padded(s[x], s["k_ptr"], s["longest_k"]).permute(0, 2, 1, 3).contiguous() for x in "kv")
    nq, nk = s["q_ptr"][1:] - s["q_ptr"][:-1], s["k_ptr"][1:] - s["k_ptr"][:-1]
    o = _softmax_product(qp, kp, vp, _seen(nq, nk, s["longest"], s["longest_k"], bool(case.get("all"))))
    o = o.permute(0, 3, 1, 2, 4).reshape(case["B"], -1, case["heads"], dim)
    return o[_where(s["q_ptr"], q.shape[0])].to(q.dtype)


def _slots(s, ptr, start, rows):
    """Page and place in it of every packed row."""
    b, at = _where(ptr, rows)
    at = at + start[b]
    page = s["pool"][0][0].shape[2]
    return s["table"][b, at // page].long(), at % page


def _plain_store(s):
    case = s["case"]
    into = _slots(s, s["row_ptr"], s["start"], s["total"])
    back = _slots(s, s["back_ptr"], s["back_start"], s["back_total"])

    def one(x, pool, scale):
        if scale is None:
            pool[into[0], :, into[1]] = x.to(pool.dtype)
            return pool[back[0], :, back[1]].to(DT[case["type"]])
        q, e = _to_mx8(x.float())
        pool[into[0], :, into[1]] = q
        scale[into[0], :, into[1]] = e
        return _values(pool[back[0], :, back[1]], scale[back[0], :, back[1]]).to(DT[case["type"]])

    return {"k": one(s["k"], *s["pool"][0]), "v": one(s["v"], *s["pool"][1])}


def _plain_paged(s):
    case = s["case"]
    B, t, kv, dim = case["B"], case["tokens"], case["kv"], case["dim"]
    G = case["heads"] // kv

    def gathered(pool, scale):
        x = _values(pool[s["table"].long()], None if scale is None else scale[s["table"].long()])   # [B, columns, kv, page, dim]
        return x.permute(0, 2, 1, 3, 4).reshape(B, kv, -1, dim)[:, :, :s["longest"]]

    q = (s["q"].float() * s["scale"]).reshape(B, t, kv, G, dim).permute(0, 2, 3, 1, 4)
    k, v = gathered(*s["pool"][0]), gathered(*s["pool"][1])
    nq = torch.full_like(s["length"], t)
    o = _softmax_product(q, k, v, _seen(nq, s["length"], t, s["longest"], bool(case.get("all"))))
    return o.permute(0, 3, 1, 2, 4).reshape(B * t, case["heads"], dim).to(DT[case.get("out", case["type"])])


# ---- the library's calls

_context = []


def _tsdp():
    """The context that a program has open for its networks."""
    if not _context:
        import tsdp_inputs as ti
        from paper_2512_15773_amd import Tsdp
        _context.append(Tsdp.from_workload(ti.C1))
    return _context[0]


def _cache(s):
    """The cache object that a program keeps beside its pools."""
    if "cache" not in s:
        from paper_2512_15773_amd import KvCache
        (k, k_scale), (v, v_scale) = s["pool"]
        s["cache"] = KvCache(k, v, s["table"], k_scale, v_scale)
    return s["cache"]


def run(state):
    s, case = state, state["case"]
    op = case["op"]
    if not own:
        return {"prompt": _plain_prompt, "store": _plain_store, "paged": _plain_paged}[op](s)
    ctx = _tsdp()
    if op == "prompt":
        return ctx.tsdp_attend_prompt(s["q"], s["k"], s["v"], s["q_ptr"], s["k_ptr"], causal=not case.get("all"), scale=s["scale"])
    cache = _cache(s)
    if op == "store":
        ctx.tsdp_cache_write(cache, s["row_ptr"], s["start"], s["k"], s["v"])
        k, v = ctx.tsdp_cache_read(cache, s["back_ptr"], s["back_start"], s["back_total"], DT[case["type"]])
        return {"k": k, "v": v}
    if "scratch" not in s:
        s["scratch"] = ctx.alloc_scratch(cache, case["heads"], case["tokens"], s["longest"])
    return ctx.tsdp_attend_paged(s["q"], cache, s["length"], s["longest"], tokens=case["tokens"], causal=not case.get("all"),
                                 scale=s["scale"], out_dtype=DT[case.get("out", case["type"])], scratch=s["scratch"])


# ---- the definitions in 64 bits


def _exact_attention(q, k, v, scale, every):
    """One sequence: q [nq, heads, dim], k / v [nk, kv, dim] in 64 bits."""
    nq, heads, dim = q.shape
    nk, kv = k.shape[:2]
    out = torch.zeros(nq, heads, dim, dtype=torch.float64, device=q.device)
    for lo in range(0, nq, 2048):
        hi = min(nq, lo + 2048)
        last = torch.arange(lo, hi, device=q.device) + (nk - nq + 1)
        if every:
            last = torch.full_like(last, nk)
        hidden = torch.arange(nk, device=q.device)[None] >= last[:, None]
        for h in range(heads):
            x = k[:, h // (heads // kv)]
            score = torch.mm(q[lo:hi, h], x.t().contiguous()) * scale
            score[hidden] = -math.inf
            weight = torch.softmax(score, -1)
            weight[(last <= 0)] = 0.0
            out[lo:hi, h] = torch.mm(weight, v[:, h // (heads // kv)])
    return out


def _exact_mx8(x):
    """The values that an 8-bit cache holds of x [..., dim], in 64 bits."""
    b = x.reshape(*x.shape[:-1], -1, 32)
    amax = b.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(amax / 448.0).clamp(min=-111.0))
    e = torch.where(amax > 448.0 * torch.exp2(e), e + 1, e)                 # log2 next to a whole number
    e = torch.where((amax <= 448.0 * torch.exp2(e - 1)) & (e > -111), e - 1, e)
    y = b * torch.exp2(-e)
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return (torch.round(y / step) * step * torch.exp2(e)).reshape(x.shape)


def exact(case, seed):
    s = prepare(case, seed)
    n, every = _lengths(case), bool(case.get("all"))
    if case["op"] == "prompt":
        q_at, k_at, out = 0, 0, []
        for x in n:
            y = x + case["past"]
            out.append(_exact_attention(s["q"][q_at:q_at + x].double(), s["k"][k_at:k_at + y].double(), s["v"][k_at:k_at + y].double(),
                                        s["scale"], every))
            q_at, k_at = q_at + x, k_at + y
        return torch.cat(out)
    table = s["table"].cpu()

    def held(which, b, lo, hi):
        """Tokens lo .. hi - 1 of environment b as the pools hold them."""
        pool, scale = s["pool"][which]
        page = pool.shape[2]
        at = torch.arange(lo, hi)
        p, r = table[b, at // page].long().to(pool.device), (at % page).to(pool.device)
        if scale is None:
            return pool[p, :, r].double()
        x = pool[p, :, r]
        sign, power, fraction = (x >> 7).double(), ((x >> 3) & 15).double(), (x & 7).double()
        value = torch.where(power > 0, (1 + fraction / 8) * torch.exp2(power - 7), fraction * 2.0 ** -9) * (1 - 2 * sign)
        return value * torch.exp2(scale[p, :, r].double() - 127).repeat_interleave(32, -1)

    if case["op"] == "store":
        at, out = 0, {"k": [], "v": []}
        for b, x in enumerate(n):
            for which, name in enumerate("kv"):
                new = s[name][at:at + x].double()
                if case["held"] == "mx8":
                    new = _exact_mx8(new)
                if case["back"]:
                    new = torch.cat([held(which, b, case["past"] - case["back"], case["past"]), new])
                out[name].append(new)
            at += x
        return {name: torch.cat(x) for name, x in out.items()}
    t = case["tokens"]
    return torch.cat([_exact_attention(s["q"][b * t:b * t + t].double(), held(0, b, 0, x), held(1, b, 0, x), s["scale"], every)
                      for b, x in enumerate(n)])
