"""Operators for serving a batch from a paged 8-bit key/value cache: the cases that are measured, their plain forms and
their definitions in 64 bits.

Cache: codes int8 [n_pages][Hkv][page][D] for keys and for values, one float32 scale per 32 positions of a page and head
([n_pages][Hkv][page / 32]); a value is code * scale.  A request b holds the pages table[b][0], table[b][1], ... and its
length lens[b]; the new tokens of a step are rows row_start[b] .. row_start[b + 1] - 1 of the step's arrays, and they are
the request's last positions.

    plan    pages, lengths, row and position maps of a step, from the requests' lengths
    rope    rotary positions of a step's rows
    append  new keys and values into the cache, quantised
    attn    attention of the new tokens over the cache
"""
import math
import random

import torch

own = False

BLOCK = 32   # positions that share a scale
DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
SCRATCH_BYTES = 1 << 23   # what the attention asks for, zero before its first use


# ---- cases ------------------------------------------------------------------------------------------------------
def listed():
    return [
        # one request of a 7B backbone (32 heads of their own) early in an episode: a control loop that waits for it
        dict(name="attn one token 7B L512", op="attn", batch=1, longest=512, ragged=False, new=1, kv=32, group=1, dim=128, page=64, dtype="f16"),
        # a full batch of equal contexts, four query heads per key/value head
        dict(name="attn batch 32 L4096 4x8", op="attn", batch=32, longest=4096, ragged=False, new=1, kv=8, group=4, dim=128, page=64, dtype="f16"),
        # requests of all ages, idle slots among them, a few tokens each (checked drafts)
        dict(name="attn ragged 61 to 16384", op="attn", batch=61, longest=16384, ragged=True, new=3, kv=8, group=4, dim=128, page=128, dtype="bf16"),
        # one long context, eight heads of 256 on one key/value head (the 2B backbone)
        dict(name="attn 2B one L100001", op="attn", batch=1, longest=100001, ragged=False, new=1, kv=1, group=8, dim=256, page=256, dtype="bf16"),
        # small heads, several new tokens, short contexts
        dict(name="attn heads of 64", op="attn", batch=17, longest=1000, ragged=True, new=5, kv=10, group=1, dim=64, page=32, dtype="f16"),
        # a decode step of a batch: one new token per request
        dict(name="append batch 64", op="append", batch=64, longest=900, ragged=True, new=1, kv=8, dim=128, page=64, dtype="f16"),
        # a prompt of one request, every head with keys and values of its own
        dict(name="append prompt 4000 7B", op="append", batch=1, longest=4000, ragged=False, new=4000, kv=32, dim=128, page=64, dtype="bf16"),
        # chunks of several prompts into contexts that are under way
        dict(name="append chunks 2B", op="append", batch=9, longest=2500, ragged=True, new=333, kv=1, dim=256, page=128, dtype="f16"),
        # a decode step's queries and keys out of the projections' float32 sums, half of each head rotated
        dict(name="rope decode 45 part", op="rope", rows=45, heads=40, extra=8, dim=128, rot=64, layout="pairs", scaling="linear", factor=4.0, far=8000, src="f32", dst="f16"),
        # a prompt far into a context that was stretched by parts
        dict(name="rope prompt 4000 parts", op="rope", rows=4000, heads=40, extra=8, dim=128, rot=128, layout="half", scaling="parts", factor=8.0, far=120000, src="bf16", dst="bf16"),
        # a decode step of a small batch
        dict(name="plan batch 16", op="plan", batch=16, longest=2000, new=1, rows=64, page=64, ended=0),
        # prompts, decode steps and ended requests of a large batch in one step
        dict(name="plan batch 1000", op="plan", batch=1000, longest=20000, new=30, rows=4096, page=32, ended=50),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["attn", "attn", "append", "rope", "plan"])
    if op == "attn":
        dim, kv, group = rng.choice([64, 128, 256]), rng.choice([1, 2, 4, 8, 10, 32]), rng.choice([1, 2, 4, 7, 8, 16])
        batch = _log(rng, 1, 64)
        most = 32 * 4096 * 8 * 128 // (batch * kv * dim * (2 if group > 4 else 1))   # no more than the full batch's bytes
        longest = _log(rng, 1, max(2, min(100000, most)))
        return dict(op=op, batch=batch, longest=longest, ragged=rng.random() < 0.6, new=rng.choice([1, 1, 1, 2, 5, 8]), kv=kv, group=group, dim=dim,
                    page=rng.choice([32, 64, 128, 256, 1024]), dtype=rng.choice(["f16", "bf16"]))
    if op == "append":
        dim, kv = rng.choice([64, 128, 256]), rng.choice([1, 2, 4, 8, 10, 32])
        batch = _log(rng, 1, 64)
        new = _log(rng, 1, max(2, min(4000 // batch, 4000 * 32 * 128 // (batch * kv * dim))))
        return dict(op=op, batch=batch, longest=min(4000, new + _log(rng, 1, 1000)), ragged=rng.random() < 0.6, new=new, kv=kv, dim=dim,
                    page=rng.choice([32, 64, 128, 256]), dtype=rng.choice(["f16", "bf16"]))
    if op == "rope":
        dim = rng.choice([64, 80, 128, 256])
        scaling = rng.choice(["none", "linear", "base", "parts"])
        src, dst = rng.choice([("f16", "f16"), ("bf16", "bf16"), ("f32", "f16"), ("f32", "bf16"), ("f32", "f32")])
        heads = rng.choice([2, 9, 16, 40, 64])
        return dict(op=op, rows=_log(rng, 1, max(2, min(4000, 4000 * 40 * 64 // (heads * dim)))), heads=heads, extra=rng.choice([0, 1, 4]), dim=dim,
                    rot=rng.choice([dim, dim, dim // 2, dim // 4 * 2 - 2]), layout=rng.choice(["half", "pairs"]), scaling=scaling,
                    factor=1.0 if scaling == "none" else round(rng.uniform(1.5, 32.0), 2), far=_log(rng, 1, 1000000), src=src, dst=dst)
    batch = _log(rng, 1, 1000)
    return dict(op=op, batch=batch, longest=_log(rng, 1, 20000), new=rng.randint(1, max(1, min(100, 4096 // batch))), rows=4096, page=rng.choice([32, 64, 128, 1024]),
                ended=rng.choice([0, 0, batch // 10]))


# ---- shapes that follow from a case alone ------------------------------------------------------------------------
def _lens(case):
    """Lengths (new tokens included) and new tokens of the requests."""
    rng = random.Random("%(batch)d %(longest)d %(new)d" % case)
    lens = []
    for b in range(case["batch"]):
        if not case["ragged"] or b == 0:
            lens.append(case["longest"])
        elif b % 8 == 5:
            lens.append(0)   # a slot without a request
        else:
            lens.append(_log(rng, 1, case["longest"]))
    new = [min(case["new"], n) if case["ragged"] is False or rng.random() < 0.7 else rng.randint(0, min(case["new"], n)) for n in lens]
    new[0] = min(case["new"], lens[0])
    return lens, new


def _pages(lens, page):
    return [-(-n // page) for n in lens]


def _plan_numbers(case):
    """Lengths before the step, and new tokens (-1: the request has ended)."""
    rng = random.Random("%(batch)d %(longest)d %(new)d %(ended)d" % case)
    lens = [0 if b % 9 == 4 else _log(rng, 1, case["longest"]) for b in range(case["batch"])]
    ended = set(rng.sample(range(case["batch"]), case["ended"]))
    room, new = case["rows"], []
    for b in range(case["batch"]):
        if b in ended:
            new.append(-1)
            continue
        # most requests decode one token, a few bring a prompt
        n = 1 if rng.random() < 0.9 else rng.randint(0, case["new"])
        n = min(n, room - (case["batch"] - 1 - b) if room > case["batch"] - b else min(1, room))
        new.append(n)
        room -= n
    return lens, new


def work(case):
    op = case["op"]
    if op == "attn":
        lens, new = _lens(case)
        kv, D, rows = case["kv"], case["dim"], sum(new)
        read = sum(lens[b] for b in range(len(lens)) if new[b])
        seen = sum(new[b] * lens[b] - new[b] * (new[b] - 1) // 2 for b in range(len(lens)))
        return {"bytes": read * kv * (2 * D + 2 * 4 / BLOCK) + 2 * rows * kv * case["group"] * D * 2, "flops": 4 * D * kv * case["group"] * seen}
    if op == "append":
        _, new = _lens(case)
        n = sum(new) * case["kv"] * case["dim"] * 2
        return {"bytes": n * 2 + n + 4 * n // (case["dim"] * BLOCK), "flops": 3 * n}
    if op == "rope":
        n = case["rows"] * case["heads"] * case["dim"]
        size = {"f16": 2, "bf16": 2, "f32": 4}
        return {"bytes": n * (size[case["src"]] + size[case["dst"]]) + 4 * case["rows"], "flops": 3 * n * case["rot"] / case["dim"]}
    lens, new = _plan_numbers(case)
    moved = sum(abs(-(-max(0, n + m if m >= 0 else 0) // case["page"]) - -(-n // case["page"])) for n, m in zip(lens, new))
    return {"bytes": 4 * (4 * case["batch"] + case["rows"] + 2 * moved), "flops": 4 * (case["batch"] + case["rows"])}


# ---- inputs -----------------------------------------------------------------------------------------------------
def _normal(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda", dtype=torch.float32)


def _up11(x):
    """The next float32 of 11 significant bits that is not below x >= 0."""
    return ((x.contiguous().view(torch.int32) + 0x1FFF) & ~0x1FFF).view(torch.float32)


def _cache(gen, n_pages, kv, page, dim):
    """Codes and scales of a cache in use: channels of unequal size, as keys have them."""
    x = _normal(gen, n_pages, kv, page // BLOCK, BLOCK, dim) * (0.3 + torch.rand(kv, 1, 1, dim, generator=gen, device="cuda") * 1.7)
    scale = _up11(x.abs().amax((3, 4)) / 127)
    codes = torch.round(x / scale[..., None, None]).to(torch.int8).view(n_pages, kv, page, dim)
    return codes, scale


def _table(gen, pages, spare):
    """A table of distinct pages in no order; -1 where a request holds none."""
    n = sum(pages)
    order = torch.randperm(n + spare, generator=gen, device="cuda").to(torch.int32)
    held = torch.tensor(pages, device="cuda")
    at = torch.cumsum(held, 0) - held
    col = torch.arange(max(1, max(pages)), device="cuda")
    t = order[(at[:, None] + col).clamp(max=n + spare - 1)]
    return torch.where(col < held[:, None], t, torch.full_like(t, -1)).contiguous()


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    op = case["op"]
    s = {"case": case}
    if op in ("attn", "append"):
        lens, new = _lens(case)
        pages = _pages(lens, case["page"])
        s["lens"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
        s["row_start"] = torch.tensor([0] + [sum(new[: b + 1]) for b in range(len(new))], dtype=torch.int32, device="cuda")
        s["table"] = _table(gen, pages, 2)
        n_pages, rows = sum(pages) + 2, sum(new) + (2 if case["ragged"] else 0)   # rows behind the last request's stay as they are
        s["k"], s["ks"] = _cache(gen, n_pages, case["kv"], case["page"], case["dim"])
        s["v"], s["vs"] = _cache(gen, n_pages, case["kv"], case["page"], case["dim"])
        dt = DTYPES[case["dtype"]]
        if op == "attn":
            heads = case["kv"] * case["group"]
            s["q"] = _normal(gen, rows, heads, case["dim"]).to(dt)
            s["out"] = torch.zeros(rows, heads, case["dim"], dtype=dt, device="cuda")
            s["scratch"] = torch.zeros(SCRATCH_BYTES, dtype=torch.uint8, device="cuda")
        else:
            # the rows of a fused projection's output: keys, then values, of each token
            kv = _normal(gen, rows, 2, case["kv"], case["dim"]) * (0.3 + torch.rand(2, case["kv"], case["dim"], generator=gen, device="cuda") * 1.7)
            kv = kv.to(dt)
            s["new_k"], s["new_v"] = kv[:, 0], kv[:, 1]
    elif op == "rope":
        x = _normal(gen, case["rows"], case["heads"] + case["extra"], case["dim"]).to(DTYPES[case["src"]])
        s["x"] = x[:, : case["heads"]]   # the values of a fused projection lie between the rows
        s["pos"] = torch.randint(0, case["far"] + 1, (case["rows"],), generator=gen, device="cuda", dtype=torch.int32)
        s["pos"][case["rows"] - case["rows"] // 16:] = -1   # a padded step: these rows are nobody's
        s["out"] = torch.zeros(case["rows"], case["heads"], case["dim"], dtype=DTYPES[case["dst"]], device="cuda")
    else:
        lens, new = _plan_numbers(case)
        P = case["page"]
        held = _pages(lens, P)
        need = sum(max(0, -(-(n + m) // P) - -(-n // P)) for n, m in zip(lens, new) if m >= 0)
        wide = max([-(-(n + max(m, 0)) // P) for n, m in zip(lens, new)] + [1]) + 1
        t = torch.full((len(lens), wide), -1, dtype=torch.int32, device="cuda")
        held_t = _table(gen, held, need + 5)
        t[:, : held_t.shape[1]] = held_t
        s["table"] = t
        free = torch.ones(sum(held) + need + 5, dtype=torch.bool, device="cuda")
        free[t[t >= 0].long()] = False
        free = torch.nonzero(free)[:, 0]
        s["free"] = torch.full((sum(held) + need + 5,), -1, dtype=torch.int32, device="cuda")
        s["free"][: need + 5] = free[torch.randperm(need + 5, generator=gen, device="cuda")].to(torch.int32)
        s["n_free"] = torch.tensor([need + 5], dtype=torch.int32, device="cuda")
        s["lens"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
        s["new"] = torch.tensor(new, dtype=torch.int32, device="cuda")
        s["lens_out"], s["n_free_out"] = torch.zeros_like(s["lens"]), torch.zeros_like(s["n_free"])
        s["row_start"] = torch.zeros(len(lens) + 1, dtype=torch.int32, device="cuda")
        s["pos"] = torch.zeros(case["rows"], dtype=torch.int32, device="cuda")
    return s


# ---- the framework's calls --------------------------------------------------------------------------------------
def _own(s):
    from paper_2605_24011_b200 import aq
    case, op = s["case"], s["case"]["op"]
    if op == "rope":
        if "rope" not in s:   # a program makes it once
            s["rope"] = aq.aq_rope_setup(case["rot"], layout=case["layout"], theta=10000.0, scaling=case["scaling"], factor=case["factor"], trained=4096)
        return aq.aq_rope_rows(s["rope"], s["x"], s["pos"], s["out"])
    if op == "plan":
        aq.aq_kv8_plan(s["lens"], s["new"], s["table"], s["free"], s["n_free"], case["page"], s["lens_out"], s["n_free_out"], s["row_start"], s["pos"])
        return s["lens_out"], s["n_free_out"], s["row_start"], s["pos"], s["table"], s["free"]
    if "cache" not in s:   # what a program keeps of a layer and of a step
        s["cache"] = aq.Kv8Cache(s["k"], s["v"], s["ks"], s["vs"])
        s["batch"] = aq.Kv8Batch(s["lens"], s["table"], s["row_start"])
    if op == "attn":
        return aq.aq_kv8_attn(s["cache"], s["batch"], s["q"], s["out"], s["scratch"])
    aq.aq_kv8_append(s["cache"], s["batch"], s["new_k"], s["new_v"])
    return _values(s["k"], s["ks"]), _values(s["v"], s["vs"]), s["ks"], s["vs"]


def _values(codes, scale):
    """What the codes stand for."""
    n, kv, page, dim = codes.shape
    return codes.reshape(n, kv, page // BLOCK, BLOCK * dim) * scale[..., None]


# ---- plain forms ------------------------------------------------------------------------------------------------
def _rows(s, count):
    """Of each of `count` rows: its request, its position (-1 for a row behind the last request's)."""
    t = torch.arange(count, device="cuda", dtype=torch.int32)
    b = (torch.searchsorted(s["row_start"], t, right=True) - 1).clamp(max=s["lens"].numel() - 1)
    pos = s["lens"][b] - s["row_start"][b + 1] + t
    return b, torch.where(t < s["row_start"][-1], pos, torch.full_like(pos, -1)).long()


def _plain_attn(s):
    case = s["case"]
    kv, G, D, P = case["kv"], case["group"], case["dim"], case["page"]
    table = s["table"].clamp(min=0).long()
    B, L = table.shape[0], table.shape[1] * P

    def gathered(codes, scale):   # [B][kv][L][D]
        x = codes[table].float().view(B, -1, kv, P // BLOCK, BLOCK, D) * scale[table][..., None, None]
        return x.view(B, -1, kv, P, D).transpose(1, 2).reshape(B, kv, L, D)

    n = max(1, min(case["new"], case["longest"]))
    t = s["row_start"][:-1].long()[:, None] + torch.arange(n, device="cuda")   # the row of request b's token i
    mine = t < s["row_start"][1:].long()[:, None]
    t = t.clamp(max=s["q"].shape[0] - 1)
    q = s["q"][t].float().view(B, n, kv, G, D).permute(0, 2, 1, 3, 4).reshape(B, kv, n * G, D)
    last = s["lens"].long()[:, None] - s["row_start"][1:].long()[:, None] + t   # [B][n]
    sees = torch.arange(L, device="cuda") <= last[..., None]                       # [B][n][L]
    x = (q @ gathered(s["k"], s["ks"]).transpose(2, 3)) * (1.0 / math.sqrt(D))
    x = x.view(B, kv, n, G, L).masked_fill(~sees[:, None, :, None, :], -math.inf)
    top = x.amax(-1, keepdim=True)
    x = torch.exp(x - torch.where(top == -math.inf, torch.zeros_like(top), top))
    total = x.sum(-1, keepdim=True)
    x = x / torch.where(total == 0, torch.ones_like(total), total)
    o = x.view(B, kv, n * G, L) @ gathered(s["v"], s["vs"])
    o = o.view(B, kv, n, G, D).permute(0, 2, 1, 3, 4).reshape(B, n, kv * G, D)
    out = s["out"].clone()
    out[t[mine]] = o[mine].to(out.dtype)
    return out


def _plain_append(s):
    case = s["case"]
    kv, D, P = case["kv"], case["dim"], case["page"]
    b, pos = _rows(s, s["new_k"].shape[0])
    real = pos >= 0
    b, pos = b[real], pos[real]
    page = s["table"][b, pos // P].long()
    block, slot = page * (P // BLOCK) + pos % P // BLOCK, pos % BLOCK
    n = s["k"].shape[0] * (P // BLOCK)
    first = torch.full((n,), BLOCK, device="cuda").scatter_reduce(0, block, slot, "amin")   # BLOCK: not touched
    put = []
    for codes, scale, new in ((s["k"], s["ks"], s["new_k"]), (s["v"], s["vs"], s["new_v"])):
        x = new[real].float()                                                              # [rows][kv][D]
        codes = codes.reshape(-1, kv, P // BLOCK, BLOCK, D).transpose(1, 2).reshape(n, kv, BLOCK, D)
        old = scale.transpose(1, 2).reshape(n, kv)
        was = torch.where(first[:, None] == 0, torch.zeros_like(old), old)
        most = torch.zeros(n, kv, device="cuda").scatter_reduce(0, block[:, None].expand(-1, kv), x.abs().amax(2), "amax")
        need = _up11(most / 127)
        now = torch.where(need <= was, was, torch.maximum(need, _up11(1.25 * was)))
        now = torch.where(first[:, None] < BLOCK, now, old)
        fit = torch.where(now > 0, now, torch.ones_like(now))
        again = torch.round(codes.float() * was[..., None, None] / fit[..., None, None]).to(torch.int8)
        older = (torch.arange(BLOCK, device="cuda") < first[:, None]) & (first[:, None] < BLOCK)
        codes = torch.where(older[:, None, :, None] & (now > was)[..., None, None], again, codes)
        codes = codes.transpose(1, 2).contiguous()                                          # [block][slot][kv][D]
        codes[block, slot] = torch.round(x / fit[block][..., None]).to(torch.int8)
        codes = codes.transpose(1, 2).reshape(-1, P // BLOCK, kv, BLOCK, D).transpose(1, 2).reshape(-1, kv, P, D)
        now = now.reshape(-1, P // BLOCK, kv).transpose(1, 2).contiguous()
        put += [(codes, now)]
    (k, ks), (v, vs) = put
    return _values(k, ks), _values(v, vs), ks, vs


def _turns(case):
    """Radians per position of each pair, and the factor of the rotated values, in 64 bits."""
    r, s = case["rot"], case["factor"]
    i = torch.arange(r // 2, device="cuda", dtype=torch.float64)
    theta = 10000.0 * (s ** (r / (r - 2)) if case["scaling"] == "base" and r > 2 else 1.0)
    f = theta ** (-2 * i / r)
    if case["scaling"] == "linear":
        return f / s, 1.0
    if case["scaling"] == "parts":
        made = 4096 * f / (2 * math.pi)   # rotations over the length the model was trained on
        keep = ((made - 1.0) / (32.0 - 1.0)).clamp(0, 1)
        return f * keep + f / s * (1 - keep), 0.1 * math.log(s) + 1
    return f, 1.0


def _plain_rope(s):
    case = s["case"]
    f, m = _turns(case)
    angle = s["pos"].double()[:, None] * f
    c, w = (torch.cos(angle) * m).float()[:, None], (torch.sin(angle) * m).float()[:, None]
    x, r = s["x"].float(), case["rot"]
    half = case["layout"] == "half"
    a, b = (x[..., : r // 2], x[..., r // 2: r]) if half else (x[..., 0:r:2], x[..., 1:r:2])
    a, b = a * c - b * w, b * c + a * w
    turned = torch.cat((a, b), -1) if half else torch.stack((a, b), -1).flatten(-2)
    out = torch.cat((turned, x[..., r:]), -1).to(s["out"].dtype)
    return torch.where((s["pos"] >= 0)[:, None, None], out, s["out"])


def _plain_plan(s):
    P, lens, new = s["case"]["page"], s["lens"], s["new"]
    held = (lens + P - 1) // P
    gone = new < 0
    length = torch.where(gone, torch.zeros_like(lens), lens + new)
    more = torch.where(gone, torch.zeros_like(lens), (length + P - 1) // P - held)
    back = torch.where(gone, held, torch.zeros_like(held))
    col = torch.arange(s["table"].shape[1], device="cuda", dtype=torch.int32)
    # pages of ended requests go on the stack, in the order of the requests and their pages
    at = s["n_free"] + (torch.cumsum(back, 0) - back)[:, None] + col
    give = col < back[:, None]
    free = torch.cat((s["free"], s["free"].new_zeros(1)))
    free = free.scatter(0, torch.where(give, at, at.new_tensor(s["free"].numel())).long().flatten(), s["table"].flatten())[:-1]
    # and requests that grow take theirs from its top, in the same order
    top = s["n_free"] + back.sum()
    at = top - 1 - ((torch.cumsum(more, 0) - more)[:, None] + col - held[:, None])
    take = (col >= held[:, None]) & (col < (held + more)[:, None])
    table = torch.where(take, free[torch.where(take, at, torch.zeros_like(at)).long()], s["table"])
    count = new.clamp(min=0)
    row_start = torch.cat((count.new_zeros(1), torch.cumsum(count, 0))).to(torch.int32)
    t = torch.arange(s["pos"].numel(), device="cuda", dtype=torch.int32)
    b = (torch.searchsorted(row_start, t, right=True) - 1).clamp(max=lens.numel() - 1)
    pos = torch.where(t < row_start[-1], lens[b] + t - row_start[b], torch.full_like(t, -1))
    return length, (top - more.sum()).to(torch.int32), row_start, pos, table, free


def run(state):
    if own:
        return _own(state)
    return {"attn": _plain_attn, "append": _plain_append, "rope": _plain_rope, "plan": _plain_plan}[state["case"]["op"]](state)


# ---- definitions in 64 bits -------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    return {"attn": _exact_attn, "append": _exact_append, "rope": _exact_rope, "plan": lambda s: None}[case["op"]](s)


def _exact_attn(s):
    case = s["case"]
    G, D, P = case["group"], case["dim"], case["page"]
    out = s["out"].double()
    start = s["row_start"].tolist()
    for b, L in enumerate(s["lens"].tolist()):
        rows = start[b + 1] - start[b]
        if not rows or not L:
            continue
        pages = s["table"][b, : -(-L // P)].long()
        for h in range(case["kv"]):
            K = (s["k"][pages, h].double() * s["ks"][pages, h].double().repeat_interleave(BLOCK, 1)[..., None]).view(-1, D)[:L]
            V = (s["v"][pages, h].double() * s["vs"][pages, h].double().repeat_interleave(BLOCK, 1)[..., None]).view(-1, D)[:L]
            for i in range(rows):
                upto = L - rows + i + 1
                q = s["q"][start[b] + i, h * G: (h + 1) * G].double()
                out[start[b] + i, h * G: (h + 1) * G] = torch.softmax(q @ K[:upto].T / math.sqrt(D), -1) @ V[:upto]
    return out


def _exact_up11(x):
    m, e = torch.frexp(x)
    return torch.ldexp(torch.ceil(m * 2048) / 2048, e)


def _exact_append(s):
    case = s["case"]
    P = case["page"]
    start = s["row_start"].tolist()
    caches = [[s["k"].double(), s["ks"].double(), s["new_k"].double()], [s["v"].double(), s["vs"].double(), s["new_v"].double()]]
    for b, L in enumerate(s["lens"].tolist()):
        p, row, pages = L - (start[b + 1] - start[b]), start[b], s["table"][b].tolist()
        while p < L:   # a block of 32 positions at a time
            upto = min(L, (p // BLOCK + 1) * BLOCK)
            page, j, lo, at = pages[p // P], p % P // BLOCK, p % BLOCK, p % P - p % BLOCK
            for codes, scale, new in caches:
                x = new[row: row + upto - p]                                 # [positions][kv][D]
                was = scale[page, :, j] if lo else torch.zeros_like(scale[page, :, j])
                need = _exact_up11(x.abs().amax((0, 2)) / 127)
                now = torch.where(need <= was, was, torch.maximum(need, _exact_up11(was * 1.25)))
                fit = torch.where(now > 0, now, 1.0)[:, None, None]
                if lo:
                    codes[page, :, at: at + lo] = torch.round(codes[page, :, at: at + lo] * was[:, None, None] / fit)
                codes[page, :, at + lo: at + lo + upto - p] = torch.round(x.transpose(0, 1) / fit)
                scale[page, :, j] = now
            row, p = row + upto - p, upto
    values = [(c.view(*sc.shape, -1) * sc[..., None]) for c, sc, _ in caches]
    return values[0], values[1], caches[0][1], caches[1][1]


def _exact_rope(s):
    case = s["case"]
    r, factor = case["rot"], case["factor"]
    out = s["out"].double()
    x = s["x"].double()
    real = (s["pos"] >= 0).nonzero()[:, 0]
    out[real] = x[real]
    for i in range(r // 2):
        base, m = 10000.0, 1.0
        if case["scaling"] == "base" and r > 2:
            base *= factor ** (r / (r - 2))
        f = math.exp(-2.0 * i / r * math.log(base))
        if case["scaling"] == "linear":
            f /= factor
        elif case["scaling"] == "parts":
            keep = min(1.0, max(0.0, (4096 * f / (2 * math.pi) - 1) / 31))
            f, m = f * keep + f / factor * (1 - keep), 0.1 * math.log(factor) + 1
        turn = torch.polar(torch.full((real.numel(),), m, dtype=torch.float64, device="cuda"), s["pos"][real].double() * f)
        u, w = (i, i + r // 2) if case["layout"] == "half" else (2 * i, 2 * i + 1)
        z = torch.complex(x[real, :, u], x[real, :, w]) * turn[:, None]
        out[real, :, u], out[real, :, w] = z.real, z.imag
    return out
