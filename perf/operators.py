"""Cases that measure the streaming operators: rotary positions with the append to a paged
K/V cache, attention over whole packed prompts, and attention of a chunk of new tokens
(single tokens included) over the paged cache.

``run`` computes each operator in its plain form (elementary torch operations in 32 bits), or,
where ``own`` is true, through the library's entry points.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


# ---------------------------------------------------------------- cases
def listed():
    return [
        # 64 running sequences, one new token each, before every layer's attention: latency
        dict(name="append_tokens", op="append", dtype="bf16", d=64, hq=16, hkv=4, batch=64, q_lo=1, q_hi=1,
             kv_lo=1374, kv_hi=10992, page=64, rot=64, interleaved=False, layout="packed"),
        # a prompt of 32 views of 1,374 tokens written into the cache, a quarter of the head rotated
        dict(name="append_prompt", op="append", dtype="fp16", d=128, hq=16, hkv=8, batch=1, q_lo=43968, q_hi=43968,
             kv_lo=43968, kv_hi=43968, page=16, rot=32, interleaved=True, layout="split"),
        # short packed prompts of odd lengths, the smallest one token
        dict(name="prompt_short", op="prompt", dtype="bf16", d=64, hq=16, hkv=16, batch=5, q_lo=1, q_hi=261, block=1),
        # eight views of 1,374 tokens, each seeing itself and the views before it
        dict(name="prompt_views", op="prompt", dtype="bf16", d=64, hq=16, hkv=16, batch=1, q_lo=10992, q_hi=10992,
             block=1374),
        # packed prompts of several lengths with wider, grouped heads
        dict(name="prompt_packed", op="prompt", dtype="fp16", d=128, hq=16, hkv=2, batch=6, q_lo=517, q_hi=8191, block=1),
        # the longest prompt: 32 views of 1,374 tokens, token by token
        dict(name="prompt_long", op="prompt", dtype="bf16", d=64, hq=16, hkv=4, batch=1, q_lo=43968, q_hi=43968, block=1),
        # one sequence, one token, a short context: latency
        dict(name="token_single", op="paged", dtype="bf16", d=64, hq=16, hkv=4, batch=1, q_lo=1, q_hi=1, kv_lo=1375,
             kv_hi=1375, page=64, block=1),
        # a serving batch of single tokens over contexts of all lengths
        dict(name="token_batch", op="paged", dtype="bf16", d=64, hq=16, hkv=4, batch=64, q_lo=1, q_hi=1, kv_lo=97,
             kv_hi=16381, page=32, block=1),
        # single tokens over 100 views of 1,374 tokens, small pages
        dict(name="token_long", op="paged", dtype="fp16", d=128, hq=32, hkv=4, batch=4, q_lo=1, q_hi=1, kv_lo=130003,
             kv_hi=137400, page=16, block=1),
        # one new view over the 31 views in the cache
        dict(name="chunk_view", op="paged", dtype="bf16", d=64, hq=16, hkv=4, batch=1, q_lo=1374, q_hi=1374,
             kv_lo=43968, kv_hi=43968, page=64, block=1374),
        # a mixed batch: chunks of prompts beside short ones, over contexts of several lengths
        dict(name="chunk_mixed", op="paged", dtype="bf16", d=128, hq=16, hkv=2, batch=12, q_lo=3, q_hi=509, kv_lo=600,
             kv_hi=20001, page=128, block=1),
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        c = dict(op=rng.choice(("append", "prompt", "paged", "paged")), dtype=rng.choice(("bf16", "fp16")),
                 d=rng.choice((64, 128)))
        c["hkv"] = rng.choice((1, 2, 3, 4, 8, 16))
        c["hq"] = c["hkv"] * rng.choice([g for g in (1, 2, 3, 4, 6, 8) if g * c["hkv"] <= 32])
        c["batch"] = _spread(rng, 1, 64)
        if c["op"] == "prompt":
            c["q_hi"] = _spread(rng, 2, 30000)
            c["q_lo"] = rng.choice((c["q_hi"], _spread(rng, 1, c["q_hi"])))
            c["block"] = rng.choice((0, 1, 1, 1, 261, 1374))
        else:
            c["page"] = rng.choice((16, 32, 64, 128))
            c["kv_hi"] = _spread(rng, 16, 140000)
            c["kv_lo"] = rng.choice((c["kv_hi"], _spread(rng, 1, c["kv_hi"])))
            c["q_hi"] = 1 if rng.random() < 0.4 else _spread(rng, 1, min(4000, c["kv_lo"]))
            c["q_lo"] = rng.choice((c["q_hi"], _spread(rng, 1, c["q_hi"])))
            if c["op"] == "append":
                c["rot"] = rng.choice((c["d"], c["d"] // 2, 32))
                c["interleaved"] = rng.random() < 0.5
                c["layout"] = rng.choice(("packed", "split"))
            else:
                c["block"] = rng.choice((0, 1, 1, 1, 261))
        w, cache = work(c), sum(_kv_lens(c)) * c["hkv"] * c["d"] * 4
        padded = c["batch"] * c["q_hi"] * c["hq"] * max(_kv_lens(c)) if c["op"] != "append" else 0
        if w["flops"] <= 3.9e12 and w["bytes"] <= 1.1e9 and cache <= 2.2e9 and padded <= 3.0e10:
            return c


def _lens(n, lo, hi):
    """n lengths from lo to hi, evenly spread over the logarithm, in a mixed order."""
    at = [lo if n == 1 else int(round(lo * (hi / lo) ** (i / (n - 1)))) for i in range(n)]
    step = next(s for s in (7, 11, 13, 17) if math.gcd(s, n) == 1)
    return [at[(i * step) % n] for i in range(n)] if lo != hi else [hi] * n


def _q_lens(c):
    return _lens(c["batch"], c["q_lo"], c["q_hi"])


def _kv_lens(c):
    """Lengths after the append: a chunk is never longer than its sequence."""
    if c["op"] == "prompt":
        return _q_lens(c)
    return [max(a, b) for a, b in zip(_lens(c["batch"], c["kv_lo"], c["kv_hi"]), _q_lens(c))]


def _pairs(c):
    """(query, visible key) pairs of one head."""
    n = 0
    for ql, kl in zip(_q_lens(c), _kv_lens(c)):
        b = c["block"]
        if b == 0:
            n += ql * kl
        else:
            full, rest = divmod(ql, b)  # rows of whole blocks, rows of the last, cut one
            n += ql * (kl - ql) + b * b * full * (full + 1) // 2 + rest * ql
    return n


def work(c):
    T, K = sum(_q_lens(c)), sum(_kv_lens(c))
    if c["op"] == "append":
        # q, k and v read once; rotated q, and k and v in the cache, written once
        values = 2 * T * (c["hq"] + 2 * c["hkv"]) * c["d"]
        return {"bytes": 2 * values, "flops": 3 * T * (c["hq"] + c["hkv"]) * c["rot"]}
    # q, and the visible keys and values, read once; outputs and the rows' log-sums written once
    return {"bytes": 2 * c["d"] * (2 * T * c["hq"] + 2 * K * c["hkv"]) + 4 * T * c["hq"],
            "flops": 4 * _pairs(c) * c["hq"] * c["d"]}


# ---------------------------------------------------------------- inputs
def _inv_freq(rot):
    """Radians per position of each rotated pair, base 10,000, in 64 bits."""
    return [10000.0 ** (-2.0 * i / rot) for i in range(rot // 2)]


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt, d, hq, hkv = DTYPES[c["dtype"]], c["d"], c["hq"], c["hkv"]
    ql, kl = _q_lens(c), _kv_lens(c)
    B, T = len(ql), sum(ql)

    def randn(*shape):
        return torch.randn(*shape, generator=g, device="cuda", dtype=dt)

    s = dict(case=c, ql=ql, kl=kl, T=T)
    s["cu"] = torch.tensor([sum(ql[:i]) for i in range(B + 1)], dtype=torch.int32).cuda()
    if c["op"] == "prompt" or (c["op"] == "append" and c["layout"] == "packed"):
        qkv = randn(T, hq + 2 * hkv, d)  # a projection's output: q, k and v are slices of it
        s["q"], s["k"], s["v"] = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    else:
        s["q"] = randn(T, hq, d)
        if c["op"] == "append":
            s["k"], s["v"] = randn(T, hkv, d), randn(T, hkv, d)
    s["out"] = torch.empty(T, hq, d, dtype=dt, device="cuda")
    if c["op"] != "append":
        s["lse"] = torch.empty(T, hq, dtype=torch.float32, device="cuda")
    if c["op"] != "prompt":
        ps = c["page"]
        need = [-(-n // ps) for n in kl]
        total = sum(need) + 3  # a pool has pages that nobody holds
        order = torch.randperm(total, generator=g, device="cuda").to(torch.int32)
        table = torch.zeros(B, max(need), dtype=torch.int32, device="cuda")
        at = 0
        for b, n in enumerate(need):
            table[b, :n] = order[at:at + n]
            at += n
        s["table"] = table
        s["kv_len"] = torch.tensor(kl, dtype=torch.int32).cuda()
        s["k_pages"], s["v_pages"] = randn(total, hkv, ps, d), randn(total, hkv, ps, d)
    if c["op"] == "append":
        s["pos"] = torch.cat([torch.arange(n - m, n, dtype=torch.int32) for m, n in zip(ql, kl)]).cuda()
        # turns per position as 64-bit fractions of a turn
        s["turns"] = torch.tensor([int(f / (2 * math.pi) * 2.0 ** 64) for f in _inv_freq(c["rot"])],
                                  dtype=torch.int64).cuda()
    if own:
        import paper_2609_23733_gb300 as vp

        s["vp"] = vp
        s["dims"] = vp.attn_dims(hq, hkv, d, dtype=dt, block=c.get("block", 1))
        if c["op"] != "prompt":
            s["kv"] = vp.paged_kv(s["k_pages"], s["v_pages"], s["table"])
        if c["op"] == "append":
            s["rope"] = vp.rope_options(s["turns"], interleaved=c["interleaved"])
        else:
            s["ws"] = vp.attn_workspace(s["dims"], T, B)
    return s


# ---------------------------------------------------------------- the operators
def run(s):
    c = s["case"]
    if own:
        vp = s["vp"]
        if c["op"] == "append":
            vp.vp_rope_append(s["dims"], s["rope"], s["q"], s["k"], s["v"], s["cu"], s["kv_len"], s["pos"], s["kv"],
                              q_out=s["out"])
            return {"q": s["out"], "k_pages": s["k_pages"], "v_pages": s["v_pages"]}
        if c["op"] == "prompt":
            vp.vp_prompt_attention(s["dims"], s["q"], s["k"], s["v"], s["cu"], s["out"], s["lse"], s["ws"])
        else:
            vp.vp_paged_attention(s["dims"], s["q"], s["cu"], s["kv_len"], s["kv"], s["out"], s["lse"], s["ws"])
        return {"out": s["out"], "lse": s["lse"]}
    if c["op"] == "append":
        return _plain_append(s)
    return _plain_attention(s)


def _owners(s):
    """The sequence of each packed token, and its place among that sequence's new tokens."""
    B = len(s["ql"])
    cu = s["cu"].long()
    seq = torch.repeat_interleave(torch.arange(B, device="cuda"), cu[1:] - cu[:-1], output_size=s["T"])
    return seq, torch.arange(s["T"], device="cuda") - cu[seq]


def _rotate(x, cos, sin, rot, interleaved):
    """x [T][heads][d] in 32 bits with its first `rot` channels turned; cos, sin [T][1][rot / 2]."""
    if interleaved:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        turned = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        turned = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
    return turned if rot == x.shape[-1] else torch.cat((turned, x[..., rot:]), -1)


def _plain_append(s):
    c = s["case"]
    # the angle's fraction of a turn: a product of whole numbers that wraps at one turn
    turn = (s["pos"].long()[:, None] * s["turns"]) >> 32
    angle = turn.float() * (2 * math.pi / 2.0 ** 32)
    cos, sin = angle.cos()[:, None], angle.sin()[:, None]
    s["out"].copy_(_rotate(s["q"].float(), cos, sin, c["rot"], c["interleaved"]))
    k = _rotate(s["k"].float(), cos, sin, c["rot"], c["interleaved"]).to(s["k"].dtype)
    seq, i = _owners(s)
    cu = s["cu"].long()
    slot = s["kv_len"].long()[seq] - (cu[1:] - cu[:-1])[seq] + i
    page = s["table"][seq, slot // c["page"]].long()
    s["k_pages"][page, :, slot % c["page"]] = k
    s["v_pages"][page, :, slot % c["page"]] = s["v"]
    return {"q": s["out"], "k_pages": s["k_pages"], "v_pages": s["v_pages"]}


def _plain_attention(s):
    c = s["case"]
    d, hq, hkv = c["d"], c["hq"], c["hkv"]
    grp, B, T = hq // hkv, len(s["ql"]), s["T"]
    lq, lk, block = max(s["ql"]), max(s["kl"]), c["block"]
    seq, i = _owners(s)
    # every sequence padded to the longest
    q = torch.zeros(B, lq, hkv, grp, d, device="cuda")
    q[seq, i] = s["q"].float().view(T, hkv, grp, d)
    q = q.permute(0, 2, 1, 3, 4)  # [B][hkv][lq][grp][d]
    if c["op"] == "prompt":
        k, v = (torch.zeros(B, lk, hkv, d, device="cuda") for _ in range(2))
        k[seq, i], v[seq, i] = s["k"].float(), s["v"].float()
        k, v = k.transpose(1, 2), v.transpose(1, 2)
    else:
        k, v = (x[s["table"].long()].float().transpose(1, 2).flatten(2, 3)[:, :, :lk]
                for x in (s["k_pages"], s["v_pages"]))
    cu = s["cu"].long()
    n_q = cu[1:] - cu[:-1]
    n_k = n_q if c["op"] == "prompt" else s["kv_len"].long()
    out = torch.empty(B, hkv, lq, grp, d, device="cuda")
    lse = torch.empty(B, hkv, lq, grp, device="cuda")
    # as many rows at a time as the scores' memory allows
    rows = max(1, min(lq, 2 ** 31 // (B * hq * lk)))
    for r in range(0, lq, rows):
        e = min(lq, r + rows)
        # the last key that any of these rows sees
        hi = lk if block == 0 else max(1, max(b - a + min(a, ((e - 1) // block + 1) * block)
                                              for a, b in zip(s["ql"], s["kl"])))
        at = torch.arange(r, e, device="cuda")
        seen = n_k[:, None].expand(B, e - r)
        if block:
            seen = seen - n_q[:, None] + torch.minimum(n_q[:, None], (at // block + 1) * block)
        hidden = torch.arange(hi, device="cuda") >= seen[:, :, None]  # [B][rows][hi]
        x = torch.matmul(q[:, :, r:e].flatten(2, 3) / math.sqrt(d), k[:, :, :hi].transpose(2, 3))
        x = x.view(B, hkv, e - r, grp, hi).masked_fill_(hidden[:, None, :, None], -math.inf)
        top = x.amax(-1, keepdim=True).clamp_min_(-1e30)
        x = x.sub_(top).exp_()
        total = x.sum(-1, keepdim=True)
        y = torch.matmul(x.flatten(2, 3), v[:, :, :hi]).view(B, hkv, e - r, grp, d)
        out[:, :, r:e] = y / total.clamp_min(1e-30)
        lse[:, :, r:e] = (top + total.log())[..., 0]
    s["out"].copy_(out.permute(0, 2, 1, 3, 4)[seq, i].flatten(1, 2))
    s["lse"].copy_(lse.permute(0, 2, 1, 3)[seq, i].flatten(1, 2))
    return {"out": s["out"], "lse": s["lse"]}


# ---------------------------------------------------------------- the definitions in 64 bits
def exact(case, seed):
    c = case
    if c["op"] != "append" and 4 * _pairs(c) * c["hq"] * c["d"] > 5e12:
        return None
    s = prepare(case, seed)
    return _exact_append(s) if c["op"] == "append" else _exact_attention(s)


def _exact_append(s):
    c, rot = s["case"], s["case"]["rot"]
    f = torch.tensor(_inv_freq(rot), dtype=torch.float64, device="cuda")
    turn = torch.polar(torch.ones(s["T"], 1, rot // 2, dtype=torch.float64, device="cuda"),
                       (s["pos"].double()[:, None] * f)[:, None])

    def turned(x):  # each pair as a complex number times e^(i angle)
        x = x.double().clone()
        first, second = (slice(0, rot, 2), slice(1, rot, 2)) if c["interleaved"] else (slice(0, rot // 2), slice(rot // 2, rot))
        z = torch.complex(x[..., first].contiguous(), x[..., second].contiguous()) * turn
        x[..., first], x[..., second] = z.real, z.imag
        return x

    k, v = turned(s["k"]), s["v"].double()
    kp, vp = s["k_pages"].double(), s["v_pages"].double()
    t = 0
    for b, (m, n) in enumerate(zip(s["ql"], s["kl"])):
        slot = torch.arange(n - m, n, device="cuda")
        page = s["table"][b].long()[slot // c["page"]]
        kp[page, :, slot % c["page"]] = k[t:t + m]
        vp[page, :, slot % c["page"]] = v[t:t + m]
        t += m
    return {"q": turned(s["q"]), "k_pages": kp, "v_pages": vp}


def _exact_attention(s):
    c = s["case"]
    grp = c["hq"] // c["hkv"]
    out = torch.zeros(s["T"], c["hq"], c["d"], dtype=torch.float64, device="cuda")
    lse = torch.full((s["T"], c["hq"]), -math.inf, dtype=torch.float64, device="cuda")
    t = 0
    for b, (m, n) in enumerate(zip(s["ql"], s["kl"])):
        for h in range(c["hkv"]):
            if c["op"] == "prompt":
                k, v = s["k"][t:t + n, h].double(), s["v"][t:t + n, h].double()
            else:
                pages = s["table"][b, :-(-n // c["page"])].long()
                k, v = (x[pages, h].flatten(0, 1)[:n].double() for x in (s["k_pages"], s["v_pages"]))
            step = max(1, 2 ** 27 // (n * grp))
            for r in range(0, m, step):
                i = torch.arange(r, min(m, r + step), device="cuda")
                last = torch.full_like(i, n) if c["block"] == 0 else \
                    n - m + torch.clamp((i // c["block"] + 1) * c["block"], max=m)
                hi = int(last.max())
                for j in range(grp):
                    x = s["q"][t + i, h * grp + j].double() @ k[:hi].T / math.sqrt(c["d"])
                    x = x.masked_fill(torch.arange(hi, device="cuda") >= last[:, None], -math.inf)
                    total = torch.logsumexp(x, -1)
                    lse[t + i, h * grp + j] = total
                    out[t + i, h * grp + j] = torch.exp(x - total[:, None]) @ v[:hi]
        t += m
    return {"out": out, "lse": lse}
