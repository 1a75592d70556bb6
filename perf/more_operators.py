"""A caller's own paged cache, case by case: what is computed, in plain form and through the library.

A program that drives a model layer by layer (a reply that goes on after a tool's answer, a draft that is checked, a
prompt that is taken in pieces, one token for each of many sequences) keeps keys and values in pages and runs two
operators over a ragged batch of new tokens, a chunk for each sequence:

  append_kv          queries and keys [rows][heads][hd] are rotated by their positions; keys and values go to the
                     sequences' pages, rounded to the cache's format
  chunk_attention    row i of a sequence's chunk attends the keys 0 .. kv_len - chunk + i of its pages

`own` False: elementary torch operations; True: the calls of paper_2602_02192_b200.binding.
"""
import math
import random

import torch

own = False

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
PAGE = 16                       # tokens of a page; a page is [kv heads][K, V][16][hd]


# ---- cases ------------------------------------------------------------------------------------
def _case(name, op, S, chunk, context, heads, cache="bf16", given="", lens=0, idle=0, spare=0, theta=1e4):
    """S sequences with chunk = (shortest, longest) new tokens over context = (shortest, longest) cached ones; heads =
    (query heads, kv heads, head size); given: the type of q, k and v before the append ("": as the cache); lens: which
    lengths of these ranges; idle: sequences without new tokens; spare: rows behind the last sequence, not to be touched."""
    return {"name": name, "op": op, "S": S, "chunk_lo": chunk[0], "chunk_hi": chunk[1], "context_lo": context[0],
            "context_hi": context[1], "Hq": heads[0], "Hkv": heads[1], "hd": heads[2], "cache": cache,
            "given": given or cache, "lens": lens, "idle": idle, "spare": spare, "theta": theta}


TINY, H8B, H32B = (4, 2, 64), (32, 8, 128), (64, 8, 128)     # the two-layer, the 8B and the 32B shape


def listed():
    return [
        # one token of one conversation: latency
        _case("append_one_token", "append_kv", 1, (1, 1), (700, 700), H8B),
        # a decode step of 32 prompts x 8 samples, from the fp32 projection
        _case("append_decode_step", "append_kv", 256, (1, 1), (512, 2559), H8B, given="fp32", lens=1),
        # tools' answers of odd lengths in a few conversations, some of them waiting, half-precision cache
        _case("append_turns", "append_kv", 23, (1, 200), (0, 5000), H8B, cache="fp16", given="fp32", lens=2, idle=3, spare=37),
        # a batch of prompts of the 32B shape
        _case("append_prompts", "append_kv", 16, (1024, 1024), (0, 0), H32B, theta=1e6),
        # one token over a short cache: latency
        _case("attend_one_token", "chunk_attention", 1, (1, 1), (700, 700), H8B),
        # one token over a very long cache
        _case("attend_one_far_token", "chunk_attention", 1, (1, 1), (131000, 131000), H8B),
        # a decode step of 32 prompts x 8 samples whose caches are their own
        _case("attend_decode_step", "chunk_attention", 256, (1, 1), (512, 2559), H8B, lens=1),
        # drafts of a few tokens, checked at once
        _case("attend_drafts", "chunk_attention", 48, (2, 9), (300, 6000), H8B, lens=3),
        # tools' answers of odd lengths, some conversations waiting; five query heads to a kv head of 64
        _case("attend_turns_odd", "chunk_attention", 37, (1, 300), (0, 4000), (10, 2, 64), cache="fp16", lens=4, idle=4, spare=29),
        # the same on the 8B shape
        _case("attend_turns", "chunk_attention", 40, (16, 400), (200, 5000), H8B, lens=5),
        # a batch of prompts of the 32B shape
        _case("attend_prompts", "chunk_attention", 8, (1024, 1024), (0, 0), H32B, cache="fp16"),
        # 2048 tokens of a long document that is taken in pieces
        _case("attend_document", "chunk_attention", 1, (2048, 2048), (14336, 14336), H8B),
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, even over the logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    op = rng.choice(["append_kv", "chunk_attention", "chunk_attention"])
    Hkv = rng.choice([1, 2, 4, 8, 8, 8])
    heads = (Hkv * rng.choice([1, 2, 3, 4, 4, 5, 7, 8]), Hkv, rng.choice([64, 128, 128]))
    cache = rng.choice(["bf16", "bf16", "fp16"])
    common = {"cache": cache, "lens": rng.randint(10, 10**6), "idle": rng.choice([0, 0, 1, 3]), "spare": rng.choice([0, 0, 1, 50])}
    if op == "append_kv":
        S = _spread(rng, 1, 256)
        longest = _spread(rng, 1, max(1, 8192 // S))
        c = _case("", op, S, (rng.choice([1, longest]), longest), (0, _spread(rng, 1, 100000 if S < 16 else 8000)), heads,
                  given=rng.choice(["fp32", cache, "bf16", "fp16"]), theta=rng.choice([1e4, 1e6, 5e5]), **common)
    else:
        S = _spread(rng, 1, 256)
        longest = _spread(rng, 1, max(1, 4096 // S)) if rng.random() < 0.7 else 1
        # no more scores than the longest listed chunk has, no more cache than the decode step reads
        most = min((1 << 30) // (S * longest * heads[0]), (1 << 19) // S, 120000) - longest
        context = _spread(rng, 1, max(1, most))
        c = _case("", op, S, (rng.choice([1, longest]), longest), (rng.choice([0, context // 2, context]), context), heads, **common)
    del c["name"]
    return c


def _lengths(case):
    """New and cached tokens of every sequence."""
    rng = random.Random(case["lens"])
    new = [rng.randint(case["chunk_lo"], case["chunk_hi"]) for _ in range(case["S"])]
    old = [rng.randint(case["context_lo"], case["context_hi"]) for _ in range(case["S"])]
    for _ in range(min(case["idle"], case["S"] - 1)):
        new[rng.randrange(1, case["S"])] = 0
    return new, old


# ---- inputs -----------------------------------------------------------------------------------
def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 7919 + 13)
    new, old = _lengths(case)
    S, Hq, Hkv, hd, rows = case["S"], case["Hq"], case["Hkv"], case["hd"], sum(new) + case["spare"]
    appends = case["op"] == "append_kv"
    # an append touches the pages of its new tokens alone: the pages before them are one and the same here
    first = [o // PAGE if appends else 0 for o in old]
    count = [-(-(o + n) // PAGE) for o, n in zip(old, new)]
    need = sum(max(0, c - f) for c, f in zip(count, first)) + 1
    order = torch.randperm(need - 1, generator=g, device="cuda", dtype=torch.int32).cpu() + 1
    width = max(max(count), 1)
    table, at = torch.zeros((S, width), dtype=torch.int32), 0
    for i in range(S):
        n = max(0, count[i] - first[i])
        table[i, first[i]:first[i] + n] = order[at:at + n]
        at += n
    starts = torch.tensor([0] + new, dtype=torch.int32).cumsum(0, dtype=torch.int32).cuda()
    lens = torch.tensor([o + n for o, n in zip(old, new)], dtype=torch.int32).cuda()
    pool = torch.empty((need, Hkv, 2, PAGE, hd), dtype=DTYPES[case["cache"]], device="cuda").normal_(generator=g)
    s = {"case": case, "starts": starts, "lens": lens, "table": table.cuda(), "pool": pool, "rows": rows, "longest": max(new)}
    if appends:          # one projection's rows, cut
        whole = torch.empty((rows, (Hq + 2 * Hkv) * hd), device="cuda").normal_(generator=g).to(DTYPES[case["given"]])
        q, k, v = whole.split((Hq * hd, Hkv * hd, Hkv * hd), dim=1)
        s["q"], s["k"], s["v"] = q.view(rows, Hq, hd), k.view(rows, Hkv, hd), v.view(rows, Hkv, hd)
        s["out"] = torch.zeros((rows, Hq, hd), dtype=DTYPES[case["cache"]], device="cuda")
    else:                # some heads look at few keys, some at many
        q = torch.empty((rows, Hq, hd), device="cuda").normal_(generator=g)
        q *= 0.3 + 2.7 * torch.rand((rows, Hq, 1), generator=g, device="cuda")
        s["q"] = q.to(DTYPES[case["cache"]])
        s["out"] = torch.zeros_like(s["q"])
    if own:              # the tables of the batch, named once for all layers
        from paper_2602_02192_b200 import binding
        s["chunks"] = binding.KVChunks(s["starts"], s["lens"], s["table"], rows, max(new))
    return s


# ---- plain forms ------------------------------------------------------------------------------
def _places(s):
    """For every row of the sequences: its sequence and its position."""
    rows = torch.arange(s["rows"] - s["case"]["spare"], device="cuda", dtype=torch.int32)
    seq = torch.searchsorted(s["starts"][1:].contiguous(), rows, right=True)
    return rows.long(), seq, (s["lens"][seq] - s["starts"][seq + 1] + rows).long()


def _append_kv(s):
    case, (rows, seq, pos) = s["case"], _places(s)
    half = case["hd"] // 2
    speed = float(case["theta"]) ** (torch.arange(half, device="cuda", dtype=torch.float64) * (-2.0 / case["hd"]))
    angle = pos.double()[:, None] * speed                       # far positions lose their angle in 32 bits
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]

    def rotated(x):
        a, b = x[:len(rows), :, :half].float(), x[:len(rows), :, half:].float()
        return torch.cat([a * cos - b * sin, b * cos + a * sin], dim=2)

    page, slot = s["table"][seq, pos // PAGE].long(), pos % PAGE
    s["pool"][page, :, 0, slot] = rotated(s["k"]).to(s["pool"].dtype)
    s["pool"][page, :, 1, slot] = s["v"][:len(rows)].to(s["pool"].dtype)
    s["out"][:len(rows)] = rotated(s["q"]).to(s["out"].dtype)
    return {"q": s["out"], "pool": s["pool"]}


def _chunk_attention(s):
    """All sequences at once, padded to the longest chunk and the longest cache."""
    case, (rows, seq, pos) = s["case"], _places(s)
    S, Hq, Hkv, hd, longest = case["S"], case["Hq"], case["Hkv"], case["hd"], s["longest"]
    at = rows - s["starts"][seq].long()                          # place in the chunk
    q = torch.zeros((S, longest, Hq, hd), device="cuda")
    q[seq, at] = s["q"][:len(rows)].float()
    last = torch.full((S, longest), -1, dtype=torch.long, device="cuda")
    last[seq, at] = pos
    kv = s["pool"][s["table"].long()]                            # [S][pages][kv heads][K, V][16][hd]
    k = kv[:, :, :, 0].permute(0, 2, 1, 3, 4).reshape(S, Hkv, -1, hd).float()
    v = kv[:, :, :, 1].permute(0, 2, 1, 3, 4).reshape(S, Hkv, -1, hd).float()
    del kv
    # query heads of a kv head side by side: [S][kv heads][longest x heads a kv head][hd]
    q = q.view(S, longest, Hkv, Hq // Hkv, hd).permute(0, 2, 1, 3, 4).reshape(S, Hkv, -1, hd)
    p = torch.matmul(q, k.transpose(2, 3)).div_(math.sqrt(hd)).view(S, Hkv, longest, Hq // Hkv, -1)
    seen = torch.arange(k.shape[2], device="cuda") <= last[:, :, None]
    p.masked_fill_(~seen[:, None, :, None, :], -math.inf)
    top = p.amax(dim=-1, keepdim=True)
    p.sub_(torch.where(torch.isneginf(top), torch.zeros_like(top), top)).exp_()
    total = p.sum(dim=-1, keepdim=True)
    o = torch.matmul(p.view(S, Hkv, -1, k.shape[2]), v).view(S, Hkv, longest, Hq // Hkv, hd) / total.clamp(min=1e-37)
    s["out"][:len(rows)] = o.permute(0, 2, 1, 3, 4).reshape(S, longest, Hq, hd)[seq, at].to(s["out"].dtype)
    return s["out"]


def run(state):
    s = state
    if own:
        from paper_2602_02192_b200 import binding
        if s["case"]["op"] == "append_kv":
            binding.echo_append_kv(s["chunks"], s["q"], s["k"], s["v"], s["pool"], s["case"]["theta"], out=s["out"])
            return {"q": s["out"], "pool": s["pool"]}
        return binding.echo_chunk_attention(s["chunks"], s["q"], s["pool"], out=s["out"])
    if s["case"]["op"] == "append_kv":
        return _append_kv(s)
    return _chunk_attention(s)


def work(case):
    new, old = _lengths(case)
    Hq, Hkv, hd, tokens = case["Hq"], case["Hkv"], case["hd"], sum(new)
    if case["op"] == "append_kv":
        given = 4 if case["given"] == "fp32" else 2
        return {"bytes": tokens * hd * (Hq + 2 * Hkv) * (given + 2) + 4 * tokens, "flops": 3 * tokens * hd * (Hq + Hkv)}
    keys = sum(o + n for o, n in zip(old, new) if n)
    pairs = sum(n * o + n * (n + 1) // 2 for o, n in zip(old, new))
    return {"bytes": 4 * keys * Hkv * hd + 4 * tokens * Hq * hd + keys // 4, "flops": 4 * pairs * Hq * hd}


# ---- the definitions in 64 bits ---------------------------------------------------------------
def exact(case, seed):
    global own
    was, own = own, False
    s = prepare(case, seed)
    own = was
    new, old = _lengths(case)
    Hkv, hd, group, pool = case["Hkv"], case["hd"], case["Hq"] // case["Hkv"], s["pool"].double()
    out, row = s["out"].double(), 0
    if case["op"] == "append_kv":
        i = torch.arange(hd // 2, dtype=torch.float64, device="cuda")
        rate = torch.exp(-2 * i / hd * math.log(case["theta"]))

        def turn(x, position):
            z = torch.complex(x[..., : hd // 2].double(), x[..., hd // 2:].double())
            phase = position.double()[:, None, None] * rate
            z = z * torch.polar(torch.ones_like(phase), phase)
            return torch.cat([z.real, z.imag], dim=-1)

        for b in range(case["S"]):
            if new[b] == 0:
                continue
            here = torch.arange(old[b], old[b] + new[b], device="cuda")
            part = slice(row, row + new[b])
            pages = s["table"][b].long()[here // PAGE]
            out[part] = turn(s["q"][part], here)
            pool[pages, :, 0, here % PAGE] = turn(s["k"][part], here)
            pool[pages, :, 1, here % PAGE] = s["v"][part].double()
            row += new[b]
        return {"q": out, "pool": pool}
    for b in range(case["S"]):
        n, whole = new[b], new[b] + old[b]
        if n == 0:
            continue
        pages = s["table"][b, : -(-whole // PAGE)].long()
        kv = s["pool"][pages].transpose(0, 1)                    # [kv heads][pages][K, V][16][hd]
        for h in range(Hkv):
            k = kv[h, :, 0].reshape(-1, hd)[:whole].double()
            v = kv[h, :, 1].reshape(-1, hd)[:whole].double()
            q = s["q"][row:row + n, h * group:(h + 1) * group].double()
            z = torch.einsum("ngd,kd->ngk", q, k) * hd ** -0.5
            z += torch.triu(torch.full((n, whole), -math.inf, dtype=torch.float64, device="cuda"), old[b] + 1)[:, None]
            out[row:row + n, h * group:(h + 1) * group] = torch.softmax(z, dim=-1) @ v
        row += n
    return out
