"""Operators of a decoding step over a paged cache of 8-bit values, as a program that serves several sequences calls them.

A case is one call with its inputs in device memory.  `op` says which:

  append   new tokens' keys and values into the cache, keys and queries turned to their positions (astra_cache_append)
  attend   the new tokens' queries over everything cached for their sequences (astra_cache_attention)
  w4       products of a few tokens with weights of 4 bits and a scale per group (astra_w4_linear)

A cache page holds `page` tokens; keys and values are e4m3 with one scale per page and KV head, a power of two.  Models are
those of the repository's workloads (Llama-3-8B and GPT-2-small heads) and one with heads of 256.
"""
import math
import random

import torch

own = False

DEV = "cuda"

MODELS = {
    "llama": dict(hq=32, hkv=8, dh=128, rope=500000.0),
    "gpt2": dict(hq=12, hkv=12, dh=64, rope=0.0),
    "wide": dict(hq=16, hkv=4, dh=256, rope=10000.0),
}


def _append(model, dtype, seqs, cached, new, page, ahead=0, pad=0, mix=0):
    return dict(MODELS[model], op="append", dtype=dtype, seqs=seqs, cached=cached, new=new, page=page, ahead=ahead, pad=pad, mix=mix)


def _attend(model, dtype, seqs, cached, new, page, prior=False, gone=0.0, pad=0, mix=0):
    return dict(MODELS[model], op="attend", dtype=dtype, seqs=seqs, cached=cached, new=new, page=page, prior=prior, gone=gone, pad=pad, mix=mix)


def _w4(dtype, tokens, n_in, n_out, group, zeros=False, bias=False, y32=False):
    return dict(op="w4", dtype=dtype, tokens=tokens, n_in=n_in, n_out=n_out, group=group, zeros=zeros, bias=bias, y32=y32)


def listed():
    return [
        # the smallest write: one sequence's next token, far behind what the other devices hold of its context
        dict(_append("llama", "bf16", 1, 1024, 1, 64, ahead=98304), name="append_token"),
        # a server's step: 64 sequences of different lengths, one token each
        dict(_append("llama", "bf16", 64, 8192, 1, 64, mix=1), name="append_batch"),
        # prompts: ragged chunks of six sequences, some of them into pages that already hold tokens
        dict(_append("llama", "bf16", 6, 2048, 1531, 64, mix=2), name="append_prompts"),
        # a device's own part of an Astra step: its 1025 tokens here, the other devices' joined from their result
        dict(_attend("llama", "bf16", 1, 1024, 1, 64, prior=True), name="attend_token"),
        # one long context
        dict(_attend("llama", "bf16", 1, 131071, 1, 64), name="attend_long"),
        # a server's step: 64 ragged sequences
        dict(_attend("llama", "bf16", 64, 8192, 1, 64, mix=1), name="attend_batch"),
        # chunks of four prompts, up to 256 tokens each, over what is cached of them
        dict(_attend("llama", "bf16", 4, 2048, 256, 32, mix=3), name="attend_chunk"),
        # a small fp32 model checking a few drafted tokens per sequence
        dict(_attend("gpt2", "f32", 8, 1021, 5, 16, mix=4), name="attend_f32"),
        # queries, keys and values of one token of a large model
        dict(_w4("bf16", 1, 4096, 6144, 128), name="w4_token"),
        # a small model's projection in fp32, three tokens
        dict(_w4("f32", 3, 768, 2304, 32, bias=True, y32=True), name="w4_f32"),
        # the second MLP product of eight sequences, onto an fp32 stream
        dict(_w4("bf16", 8, 14336, 4096, 128, y32=True), name="w4_down"),
        # the first MLP product of 64 sequences, with zero points
        dict(_w4("bf16", 64, 4096, 28672, 64, zeros=True), name="w4_batch"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("append", "attend", "attend", "w4"))
    mix = rng.randrange(1, 1 << 20)
    if op == "w4":
        tokens = rng.choice((1, 1, 2, 4, _log_int(rng, 1, 64), _log_int(rng, 1, 64)))
        group = rng.choice((32, 64, 128))
        n_in = group * rng.randint(max(1, 256 // group), 14336 // group)
        return _w4(rng.choice(("bf16", "bf16", "f32")), tokens, n_in, _log_int(rng, 200, 28672 if n_in <= 4096 else 4096), group, rng.random() < 0.5,
                   rng.random() < 0.3, rng.random() < 0.3)
    model = rng.choice(("llama", "llama", "gpt2", "wide"))
    dtype = rng.choice(("bf16", "bf16", "f32")) if model != "llama" else "bf16"
    page = rng.choice((16, 32, 64, 64, 128))
    pad = rng.choice((0, 0, 3))
    if op == "append":
        kind = rng.choice(("step", "drafts", "prompts"))
        if kind == "prompts":
            seqs = rng.randint(1, 8)
            return _append(model, dtype, seqs, _log_int(rng, 1, 2048), _log_int(rng, 30, 6000 // seqs), page, rng.choice((0, 2565)), pad, mix)
        return _append(model, dtype, _log_int(rng, 1, 64), _log_int(rng, 1, 8192), 1 if kind == "step" else rng.randint(2, 8), page, rng.choice((0, 98304)), pad, mix)
    kind = rng.choice(("step", "step", "drafts", "chunk"))
    if kind == "chunk":
        seqs = rng.randint(1, 4)
        return _attend(model, dtype, seqs, _log_int(rng, 1, 2048), _log_int(rng, 9, 256), page, False, 0.0, pad, mix)
    seqs = _log_int(rng, 1, 64)
    most = {"llama": 300000, "gpt2": 400000, "wide": 300000}[model] // seqs
    return _attend(model, dtype, seqs, _log_int(rng, 1, min(most, 131000)), 1 if kind == "step" else rng.randint(2, 8), page, rng.random() < 0.3,
                   rng.choice((0.0, 0.0, 0.03)), pad, mix)


# ---- inputs --------------------------------------------------------------------------------------------------------
def _lengths(case):
    """Cached and new tokens of every sequence; the case says all of it, its seed nothing."""
    if not case["mix"]:
        return [case["cached"]] * case["seqs"], [case["new"]] * case["seqs"]
    r = random.Random(case["mix"])
    cached = [r.randint(case["cached"] // 16, case["cached"]) for _ in range(case["seqs"])]
    if case["seqs"] > 2:
        cached[r.randrange(case["seqs"])] = 0                      # a sequence that has just begun
    new = [r.randint(1, case["new"]) for _ in range(case["seqs"])]
    return cached, new


class _Draws:
    def __init__(self, seed, dtype):
        self.g = torch.Generator(device=DEV)
        self.g.manual_seed(seed)
        self.dt = torch.bfloat16 if dtype == "bf16" else torch.float32

    def normal(self, shape, std=1.0):
        return (torch.randn(shape, generator=self.g, device=DEV) * std).to(self.dt)

    def pool(self, pages, hkv, page, dh):
        """A cache as earlier calls left it: a page's values fill the upper part of the type's range, scales differ between heads and pages."""
        codes = torch.empty((pages, hkv, page, dh), dtype=torch.uint8, device=DEV)
        for at in range(0, pages, 512):
            part = codes[at:at + 512]
            part.copy_((torch.randn(part.shape, generator=self.g, device=DEV) * 83.0).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8))
        e = torch.randint(-8, -5, (pages, hkv), generator=self.g, device=DEV)
        return codes, torch.ldexp(torch.ones((), device=DEV), e)


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def prepare(case, seed):
    c, r = case, _Draws(seed, case["dtype"])
    s = {"case": c}
    if c["op"] == "w4":
        shape = (c["n_out"], c["n_in"])
        groups = (c["n_out"], c["n_in"] // c["group"])
        s["x"] = r.normal((c["tokens"], c["n_in"]))
        s["zeros"] = torch.randint(5, 12, groups, generator=r.g, device=DEV).to(torch.uint8) if c["zeros"] else None
        middle = s["zeros"].float().repeat_interleave(c["group"], 1) if c["zeros"] else 8.0
        q = (torch.randn(shape, generator=r.g, device=DEV) * 2.7 + middle).round().clamp(0, 15).to(torch.uint8)
        s["codes"] = q[:, 0::2] | (q[:, 1::2] << 4)
        s["scales"] = ((torch.rand(groups, generator=r.g, device=DEV) + 0.5) * (0.02 / 2.7)).to(r.dt)
        s["bias"] = r.normal((c["n_out"],), 0.1) if c["bias"] else None
        s["y"] = torch.zeros((c["tokens"], c["n_out"]), dtype=torch.float32 if c["y32"] else r.dt, device=DEV)
    else:
        cached, new = _lengths(c)
        p, hq, hkv, dh = c["page"], c["hq"], c["hkv"], c["dh"]
        held = [-(-(a + b) // p) for a, b in zip(cached, new)]
        pages, wide = sum(held) + 3, max(held)
        perm = torch.randperm(pages, generator=r.g, device=DEV).to(torch.int32)
        seq_of = torch.repeat_interleave(torch.arange(len(held)), torch.tensor(held))
        at = torch.arange(sum(held)) - torch.repeat_interleave(torch.tensor([sum(held[:i]) for i in range(len(held))]), torch.tensor(held))
        s["table"] = torch.full((len(held), wide), -1, dtype=torch.int32, device=DEV)
        s["table"][seq_of.to(DEV), at.to(DEV)] = perm[:sum(held)]
        s["lens"], s["first"] = _i32(cached), _i32([sum(new[:i]) for i in range(len(new) + 1)])
        s["rows"], s["most"] = sum(new), max(new)
        n = s["rows"] + c["pad"]
        s["q"] = r.normal((n, hq, dh), 1.3)
        s["k_pages"], s["k_scales"] = r.pool(pages, hkv, p, dh)
        s["v_pages"], s["v_scales"] = r.pool(pages, hkv, p, dh)
    if c["op"] == "append":
        s["k"], s["v"] = r.normal((n, hkv, dh), 1.3), r.normal((n, hkv, dh), 1.3)
        s["shift"] = _i32([c["ahead"]] * c["seqs"]) if c["ahead"] else None
        s["q_out"] = torch.zeros_like(s["q"]) if c["rope"] else None
        # sequences whose first new token lands in a page that holds earlier ones
        s["joined"] = torch.tensor([i for i in range(c["seqs"]) if cached[i] % p], dtype=torch.int64, device=DEV)
    elif c["op"] == "attend":
        if c["gone"]:
            s["table"][torch.rand(s["table"].shape, generator=r.g, device=DEV) < c["gone"]] = -1
        s["prior"], s["prior_lse"] = None, None
        if c["prior"]:
            s["prior"] = r.normal((n, hq, dh), 0.1)
            s["prior_lse"] = torch.randn((n, hq), generator=r.g, device=DEV) + 8.0
        s["out"] = torch.zeros((n, hq, dh), dtype=r.dt, device=DEV)
        s["lse"] = torch.zeros((n, hq), dtype=torch.float32, device=DEV)
    s["handle"] = _handle(s) if own else None
    return s


def _handle(s):
    """The descriptor and the scratch that a program keeps with its cache."""
    from paper_2505_19342_amd import binding as B
    c = s["case"]
    if c["op"] == "w4":
        return B, B.w4_desc(c["dtype"], c["n_in"], c["n_out"], c["group"], "f32" if c["y32"] else c["dtype"]), None
    desc = B.cache_desc(c["dtype"], c["hq"], c["hkv"], c["dh"], c["page"], s["k_pages"].shape[0], s["table"].shape[0], s["table"].shape[1], s["q"].shape[0],
                        rope_base=c["rope"])
    if c["op"] == "append":
        return B, desc, None
    return B, desc, torch.empty(max(B.astra_cache_attention_workspace_bytes(desc), 256), dtype=torch.uint8, device=DEV)


# ---- one pass ------------------------------------------------------------------------------------------------------
def run(s):
    return {"append": _run_append, "attend": _run_attend, "w4": _run_w4}[s["case"]["op"]](s)


def _run_append(s):
    if own:
        B, desc, _ = s["handle"]
        B.astra_cache_append(desc, s["table"], s["lens"], s["first"], s["shift"], s["q"] if s["q_out"] is not None else None, s["k"], s["v"], s["q_out"],
                             s["k_pages"], s["v_pages"], s["k_scales"], s["v_scales"])
    else:
        p, n = s["case"]["page"], s["rows"]
        row = torch.arange(n, device=DEV)
        seq = torch.bucketize(row, s["first"][1:].long(), right=True)
        token = s["lens"].long()[seq] + row - s["first"].long()[seq]
        page, off = s["table"].long()[seq, token // p], token % p
        k, v = s["k"][:n].float(), s["v"][:n].float()
        if s["q_out"] is not None:
            place = token if s["shift"] is None else token + s["shift"].long()[seq]
            dh = k.shape[-1]
            step = torch.pow(torch.tensor(s["case"]["rope"], dtype=torch.float64, device=DEV), torch.arange(0, dh, 2, device=DEV, dtype=torch.float64) / -dh)
            angle = place.double()[:, None, None] * step
            cos, sin = angle.cos().float(), angle.sin().float()
            k = _turned(k, cos, sin)
            s["q_out"][:n] = _turned(s["q"][:n].float(), cos, sin).to(s["q"].dtype)
        old = s["table"].long()[s["joined"], s["lens"].long()[s["joined"]] // p]
        held = s["lens"].long()[s["joined"]] % p
        _store(s["k_pages"], s["k_scales"], k, page, off, old, held)
        _store(s["v_pages"], s["v_scales"], v, page, off, old, held)
    out = {n: s[n + "_pages"].view(torch.float8_e4m3fn) for n in ("k", "v")}
    out.update({n: s[n] for n in ("k_scales", "v_scales")})
    if s["q_out"] is not None:
        out["q"] = s["q_out"]
    return out


def _turned(x, cos, sin):
    a, b = x[..., 0::2], x[..., 1::2]
    return torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)


def _store(pages, scales, x, page, off, old, held):
    """Rows x [n, heads, dh] to (page, off); the pages `old` hold `held` earlier tokens each."""
    finite = torch.isfinite(x)
    most = torch.where(finite, x.abs(), 0.0).amax(-1)
    need = torch.zeros_like(scales).scatter_reduce_(0, page[:, None].expand_as(most), most, "amax")
    touched = torch.zeros((scales.shape[0], 1), dtype=torch.bool, device=x.device).index_fill_(0, page, True)
    keeps = torch.zeros((scales.shape[0], 1), dtype=torch.bool, device=x.device).index_fill_(0, old, True)
    mantissa, e = torch.frexp(need)
    e = torch.where(need > 0, e - 9 + (mantissa > 0.875), -100).clamp(-100, 110)
    scale = torch.ldexp(torch.ones((), device=x.device), e)
    scale = torch.where(touched, torch.where(keeps, torch.maximum(scales, scale), scale), scales)
    kept = pages[old]
    again = (kept.view(torch.float8_e4m3fn).float() * (scales[old] / scale[old])[..., None, None]).to(torch.float8_e4m3fn).view(torch.uint8)
    earlier = torch.arange(pages.shape[2], device=x.device) < held[:, None]
    pages[old] = torch.where(earlier[:, None, :, None], again, kept)
    scaled = (x / scale[page][..., None]).clamp(-448.0, 448.0)
    pages[page, :, off] = torch.where(finite, scaled, math.nan).to(torch.float8_e4m3fn).view(torch.uint8)
    scales.copy_(scale)


def _run_attend(s):
    if own:
        B, desc, scratch = s["handle"]
        B.astra_cache_attention(desc, s["table"], s["lens"], s["first"], s["q"], s["k_pages"], s["v_pages"], s["k_scales"], s["v_scales"], s["prior"],
                                s["prior_lse"], s["out"], s["lse"], scratch)
        return {"out": s["out"], "lse": s["lse"]}
    c = s["case"]
    table, n_pages, p = s["table"].long(), s["k_pages"].shape[0], c["page"]
    there = (table >= 0) & (table < n_pages)
    at = torch.where(there, table, 0)
    seqs, wide = table.shape
    keys = wide * p
    t = torch.arange(keys, device=DEV)
    total = (s["lens"] + s["first"][1:] - s["first"][:-1]).long()
    real = there.repeat_interleave(p, 1) & (t < total[:, None])                                         # [seqs, keys]

    def rows(pages, scales):
        x = pages[at].view(torch.float8_e4m3fn).float() * scales[at][..., None, None]
        x = x.permute(0, 2, 1, 3, 4).reshape(seqs, c["hkv"], keys, c["dh"])
        return torch.where(real[:, None, :, None], x, 0.0)

    share, most = c["hq"] // c["hkv"], s["most"]
    i = torch.arange(most, device=DEV)
    row = (s["first"][:-1, None] + i).long().clamp(max=s["q"].shape[0] - 1)                            # [seqs, most]
    q = s["q"][row].float().view(seqs, most, c["hkv"], share, c["dh"]).permute(0, 2, 1, 3, 4).reshape(seqs, c["hkv"], most * share, c["dh"])
    score = torch.matmul(q, rows(s["k_pages"], s["k_scales"]).transpose(-1, -2).contiguous()) / math.sqrt(c["dh"])
    sees = real[:, None, :] & (t <= (s["lens"].long()[:, None] + i)[..., None])                         # [seqs, most, keys]
    score = score.masked_fill(~sees.repeat_interleave(share, 1)[:, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    weight = torch.exp(score - top)
    del score
    whole = weight.sum(-1, keepdim=True)
    o = torch.matmul(weight, rows(s["v_pages"], s["v_scales"])) / torch.where(whole > 0, whole, 1.0)
    lse = (top + torch.log(whole))[..., 0]

    def by_row(x):                                                                                       # [seqs, hkv, most * share, ...] -> [seqs, most, hq, ...]
        x = x.view(seqs, c["hkv"], most, share, *x.shape[3:])
        return x.transpose(1, 2).flatten(2, 3)

    o, lse = by_row(o), by_row(lse)
    if s["prior"] is not None:
        o, lse = _joined(o, lse, s["prior"][row].float(), s["prior_lse"][row])
    # a sequence's rows beyond its own new tokens go to a row behind the last, which is cut off
    n = s["q"].shape[0]
    row = torch.where(i < (s["first"][1:] - s["first"][:-1])[:, None], row, n)
    out = torch.zeros((n + 1, c["hq"], c["dh"]), dtype=s["q"].dtype, device=DEV)
    out[row] = o.to(out.dtype)
    all_lse = torch.zeros((n + 1, c["hq"]), dtype=torch.float32, device=DEV)
    all_lse[row] = lse
    # rows behind the last sequence stay as they were
    inside = torch.arange(n, device=DEV) < s["first"][-1]
    return {"out": torch.where(inside[:, None, None], out[:n], 0.0), "lse": torch.where(inside[:, None], all_lse[:n], 0.0)}


def _joined(o, lse, prior, prior_lse):
    top = torch.maximum(lse, prior_lse)
    top = torch.where(top == -math.inf, 0.0, top)
    a, b = torch.exp(lse - top), torch.exp(prior_lse - top)
    whole = a + b
    o = (a[..., None] * o + b[..., None] * prior) / torch.where(whole > 0, whole, 1.0)[..., None]
    return o, top + torch.log(whole)


def _run_w4(s):
    c = s["case"]
    if own:
        B, desc, _ = s["handle"]
        B.astra_w4_linear(desc, s["x"], c["tokens"], s["codes"], s["scales"], s["zeros"], s["bias"], s["y"])
        return s["y"]
    w = torch.stack((s["codes"] & 15, s["codes"] >> 4), -1).flatten(1).float()
    zero = 8.0 if s["zeros"] is None else s["zeros"].float().repeat_interleave(c["group"], 1)
    w = (w - zero) * s["scales"].float().repeat_interleave(c["group"], 1)
    y = torch.matmul(s["x"].float(), w.t())
    if s["bias"] is not None:
        y = y + s["bias"].float()
    return y.to(s["y"].dtype)


# ---- what a pass cannot do without ---------------------------------------------------------------------------------
def work(case):
    c = case
    eb = 2 if c["dtype"] == "bf16" else 4
    if c["op"] == "w4":
        t, k, n = c["tokens"], c["n_in"], c["n_out"]
        groups = n * (k // c["group"])
        n_bytes = n * k // 2 + groups * (eb + c["zeros"]) + t * k * eb + t * n * (4 if c["y32"] else eb) + c["bias"] * n * eb
        return {"bytes": n_bytes, "flops": 2.0 * t * k * n}
    cached, new = _lengths(c)
    n, hq, hkv, dh, p = sum(new), c["hq"], c["hkv"], c["dh"], c["page"]
    if c["op"] == "append":
        blocks = sum(-(-(a + b) // p) - a // p for a, b in zip(cached, new)) * hkv
        turned = 2 * n * hq * dh * eb if c["rope"] else 0
        return {"bytes": turned + 2 * n * hkv * dh * (eb + 1) + 2 * 4 * blocks, "flops": 3.0 * n * (hq + hkv) * dh if c["rope"] else 0.0}
    keys = sum(a + b for a, b in zip(cached, new))
    pairs = sum(b * a + b * (b + 1) // 2 for a, b in zip(cached, new))
    return {"bytes": 2 * keys * hkv * dh + 2 * 4 * hkv * (keys // p) + (2 + c["prior"]) * n * hq * dh * eb + 4 * n * hq, "flops": 4.0 * pairs * hq * dh}


# ---- the definitions in 64 bits ------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    return {"append": _exact_append, "attend": _exact_attend, "w4": _exact_w4}[case["op"]](s)


def _e4m3(x):
    """The nearest value of 4 exponent and 3 mantissa bits, ties to even, of values up to 448."""
    _, e = torch.frexp(x)
    step = torch.ldexp(torch.ones((), dtype=torch.float64, device=x.device), torch.clamp(e - 1, min=-6) - 3)
    return torch.round(x / step) * step


def _exact_append(s):
    c = s["case"]
    cached, new = _lengths(c)
    p, dh = c["page"], c["dh"]
    rotate = c["rope"] > 0
    turns = torch.arange(dh // 2, dtype=torch.float64, device=DEV)
    theta = torch.exp(turns * (-2.0 / dh) * math.log(c["rope"])) if rotate else None
    q_out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    got = {n: s[n + "_pages"].view(torch.float8_e4m3fn).double() for n in ("k", "v")}
    scales = {n: s[n + "_scales"].double() for n in ("k", "v")}
    table = s["table"].tolist()

    def placed(x, first, m):
        z = torch.view_as_complex(x.double().reshape(*x.shape[:-1], dh // 2, 2).contiguous())
        pos = torch.arange(first, first + m, dtype=torch.float64, device=DEV)
        return torch.view_as_real(z * torch.polar(torch.ones((), dtype=torch.float64, device=DEV), pos[:, None] * theta)[:, None]).flatten(-2)

    row = 0
    for i in range(c["seqs"]):
        a, m = cached[i], new[i]
        part = {n: s[n][row:row + m].double() for n in ("k", "v")}
        if rotate:
            part["k"] = placed(s["k"][row:row + m], a + c["ahead"], m)
            q_out[row:row + m] = placed(s["q"][row:row + m], a + c["ahead"], m)
        done = 0
        while done < m:
            at, off = table[i][(a + done) // p], (a + done) % p
            take = min(p - off, m - done)
            for n in ("k", "v"):
                x = part[n][done:done + take].transpose(0, 1)                        # [heads, take, dh]
                most = x.abs().amax((1, 2))
                e = torch.ceil(torch.log2(most / 448.0)).clamp(-100, 110)
                scale = torch.exp2(e)
                if off:
                    scale = torch.maximum(scale, scales[n][at])
                    got[n][at, :, :off] = _e4m3(got[n][at, :, :off] * (scales[n][at] / scale)[:, None, None])
                got[n][at, :, off:off + take] = _e4m3(x / scale[:, None, None])
                scales[n][at] = scale
            done += take
        row += m
    out = {"k": got["k"], "v": got["v"], "k_scales": scales["k"], "v_scales": scales["v"]}
    if rotate:
        out["q"] = q_out
    return out


def _exact_attend(s):
    c = s["case"]
    cached, new = _lengths(c)
    share, p = c["hq"] // c["hkv"], c["page"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.zeros(s["lse"].shape, dtype=torch.float64, device=DEV)
    row = 0
    for i in range(c["seqs"]):
        total, m = cached[i] + new[i], new[i]
        ids = s["table"][i, :-(-total // p)].long()
        known = ids >= 0
        token = torch.arange(ids.numel() * p, device=DEV).view(-1, p)[known].flatten()
        inside = token < total
        token = token[inside]
        k, v = (s[n + "_pages"][ids[known]].view(torch.float8_e4m3fn).double() * s[n + "_scales"][ids[known]].double()[..., None, None] for n in ("k", "v"))
        k, v = (x.transpose(1, 2).reshape(-1, c["hkv"], c["dh"])[inside] for x in (k, v))
        hidden = token[None, :] > (cached[i] + torch.arange(m, device=DEV))[:, None]
        for h in range(c["hq"]):
            z = (s["q"][row:row + m, h].double() @ k[:, h // share].t()) * c["dh"] ** -0.5
            z = z.masked_fill(hidden, -math.inf)
            if c["prior"]:
                z = torch.cat((z, s["prior_lse"][row:row + m, h].double()[:, None]), 1)
            at = torch.logsumexp(z, 1) if z.shape[1] else torch.full((m,), -math.inf, dtype=torch.float64, device=DEV)
            w = torch.exp(z - torch.where(at == -math.inf, 0.0, at)[:, None])
            if c["prior"]:
                out[row:row + m, h] = w[:, :-1] @ v[:, h // share] + w[:, -1:] * s["prior"][row:row + m, h].double()
            else:
                out[row:row + m, h] = w @ v[:, h // share]
            lse[row:row + m, h] = at
        row += m
    return {"out": out, "lse": lse}


def _exact_w4(s):
    c = s["case"]
    x = s["x"].double().view(c["tokens"], -1, c["group"]).transpose(0, 1).contiguous()                  # [groups, tokens, group]
    y = torch.zeros((c["tokens"], c["n_out"]), dtype=torch.float64, device=DEV)
    for at in range(0, c["n_out"], 4096):                                                                # some rows of the weights at a time
        codes = s["codes"][at:at + 4096]
        n = codes.shape[0]
        digit = torch.zeros((n, c["n_in"]), dtype=torch.float64, device=DEV)
        digit[:, 0::2], digit[:, 1::2] = (codes % 16).double(), (codes // 16).double()
        digit = digit.view(n, -1, c["group"])
        digit = digit - (8.0 if s["zeros"] is None else s["zeros"][at:at + n].double()[..., None])
        part = torch.matmul(x, digit.permute(1, 2, 0).contiguous())                                      # [groups, tokens, n]
        y[:, at:at + n] = (part * s["scales"][at:at + n].double().t()[:, None]).sum(0)
    return y if s["bias"] is None else y + s["bias"].double()
