"""Operators of the layers that stand beside the SSD core in a hybrid stack, as users have them run.

A Mamba-2 block normalises the residual stream in front of its projections and the core's output, gated, behind it; a
hybrid stack has an attention layer every few blocks, whose keys and values live in a paged cache.  A case's "kind"
names the operator:

* ``gated``     ``ssd_norm_gated``: the norm between the SSD core and the output projection, with its gate
* ``residual``  ``ssd_norm_residual``: a block's output joins the residual stream, which is normalised for the next block
* ``append``    ``ssd_attn_append``: queries and keys are rotated, keys and values go to the paged cache
* ``step``      ``ssd_attn_step``: attention of one new token of each sequence over its pages
* ``prompt``    ``ssd_attn_prefill``: causal attention of the new tokens of a packed batch over their pages

With ``own`` false ``run`` computes them from elementary torch operations in fp32, rounded once at the end.
"""
import math
import random

import torch

own = False

EPS = 1e-5
ROPE_THETA = 10000.0
LOGIT_SCALE = 2.0      # standard deviation of the attention logits: a few tokens of a context stand out, as they do in use


def listed():
    return [
        # generation for one user: the gate behind the core of a 2.7B-shaped block (80 heads of 64); latency of a call
        dict(name="gated_token", kind="gated", io="bf16", rows=1, width=5120, groups=1, norm_first=False),
        # the same block over a long prompt; the gate is a slice of the input projection's output
        dict(name="gated_prompt", kind="gated", io="bf16", rows=16384, width=5120, groups=1, norm_first=False),
        # generation for a batch of users, residual stream in fp32
        dict(name="residual_b16", kind="residual", io="bf16", rows=16, width=2560, stream="f32", scale=1.0),
        # a prompt on a 130M-shaped stack in fp32, of no round length, with a residual scale
        dict(name="residual_prompt_f32", kind="residual", io="f32", rows=16383, width=768, stream="f32", scale=0.22),
        # one new token for each of 64 users
        dict(name="append_b64", kind="append", io="bf16", seqs=64, new=1, prior=6000, even=False, lens_seed=3, heads=32, kv_heads=8,
             headdim=128, page=16, rotary=128, interleaved=False),
        # a ragged batch of prompts, most of them later pieces
        dict(name="append_prompts", kind="append", io="bf16", seqs=12, new=5119, prior=3000, even=False, lens_seed=5, heads=40, kv_heads=8,
             headdim=64, page=64, rotary=32, interleaved=True),
        # generation for one user after a short prompt: latency of a call
        dict(name="step_short", kind="step", io="bf16", seqs=1, prior=517, even=True, lens_seed=0, heads=32, kv_heads=8, headdim=128,
             page=16, window=0),
        # a server's batch: contexts of very different lengths
        dict(name="step_b64", kind="step", io="bf16", seqs=64, prior=32767, even=False, lens_seed=7, heads=32, kv_heads=8, headdim=128,
             page=16, window=0),
        # few users with long contexts in fp32, as numerics are checked; an odd number of heads per key head
        dict(name="step_long_f32", kind="step", io="f32", seqs=2, prior=100003, even=True, lens_seed=0, heads=10, kv_heads=2, headdim=64,
             page=64, window=0),
        # a prompt on a small model in fp32
        dict(name="prompt_small_f32", kind="prompt", io="f32", seqs=1, new=1023, prior=0, even=True, lens_seed=0, heads=12, kv_heads=4,
             headdim=64, page=16, window=0),
        # one long prompt
        dict(name="prompt_long", kind="prompt", io="bf16", seqs=1, new=16384, prior=0, even=True, lens_seed=0, heads=32, kv_heads=8,
             headdim=128, page=64, window=0),
        # pieces of prompts against what is cached already, with a window; some have no new token
        dict(name="prompt_pieces", kind="prompt", io="bf16", seqs=10, new=512, prior=20000, even=False, lens_seed=2, heads=20, kv_heads=4,
             headdim=128, page=16, window=4096),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _heads(rng):
    kv = rng.choice([1, 2, 4, 5, 8])
    group = rng.choice([1, 2, 4, 5, 7, 8, 16])
    return dict(heads=kv * group, kv_heads=kv, headdim=rng.choice([64, 64, 80, 112, 128, 128, 128, 256]), page=rng.choice([16, 16, 32, 64, 128]))


def draw(rng):
    kind = rng.choice(["gated", "residual", "append", "append", "step", "step", "step", "prompt", "prompt", "prompt"])
    io = rng.choice(["bf16", "bf16", "f32"])
    if kind == "gated":
        groups = rng.choice([1, 1, 1, 2, 8])
        width = groups * _log_int(rng, 48, 8192 // groups)
        rows = _log_int(rng, 1, max(1, min(32768, 16384 * 5120 // width // (1 if io == "bf16" else 2))))
        return dict(kind=kind, io=io, rows=rows, width=width, groups=groups, norm_first=rng.random() < 0.5)
    if kind == "residual":
        width = _log_int(rng, 48, 8192)
        rows = _log_int(rng, 1, max(1, min(32768, 8192 * 2560 // width)))
        return dict(kind=kind, io=io, rows=rows, width=width, stream="f32" if io == "f32" else rng.choice(["f32", "f32", "bf16"]),
                    scale=rng.choice([1.0, 0.22]))
    h = _heads(rng)
    even, lens_seed = rng.random() < 0.3, rng.randrange(1 << 30)
    if kind == "append":
        n = _log_int(rng, 1, 64)
        # (the whole cache is an output here: its size bounds a drawn case)
        most = max(2, min(8192, (1 << 26) // (n * h["kv_heads"] * h["headdim"])))
        new = 1 if rng.random() < 0.5 else _log_int(rng, 1, max(1, min(most // 2, (1 << 26) // (n * h["heads"] * h["headdim"]))))
        return dict(kind=kind, io=io, seqs=n, new=new, prior=_log_int(rng, 1, most) - 1, even=even, lens_seed=lens_seed,
                    rotary=rng.choice([h["headdim"], h["headdim"], h["headdim"] // 2, 32]), interleaved=rng.random() < 0.3, **h)
    window = rng.choice([0, 0, 0, _log_int(rng, 64, 8192)])
    if kind == "step":
        n = _log_int(rng, 1, 128)
        # keys and values of the longest sequence times the batch: what the plain form holds, in fp32
        longest = max(16, min(131072, (1 << (29 if io == "bf16" else 27)) // (n * h["kv_heads"] * h["headdim"])))
        return dict(kind=kind, io=io, seqs=n, prior=_log_int(rng, 16, longest) - 1, even=even, lens_seed=lens_seed, window=window, **h)
    n = _log_int(rng, 1, 8)
    whole = rng.random() < 0.5       # whole prompts, or pieces behind what is cached
    prior = 0 if whole else _log_int(rng, 1, 32768)
    # 4 x headdim x heads operations for each pair of a new token and a token that it sees
    pairs = (2.0e12 if io == "bf16" else 1.0e11) / n / (4.0 * h["headdim"] * h["heads"])
    limit = int(math.sqrt(prior * prior + 2.0 * pairs) - prior)
    new = _log_int(rng, 1, max(1, min(16384 if whole else 2048, limit)))
    return dict(kind=kind, io=io, seqs=n, new=new, prior=prior, even=even, lens_seed=lens_seed, window=window, **h)


def _lengths(case):
    """New and cached tokens of each sequence: all the most that the case names, or the first sequence the most, the
    others spread below it, and every eighth without a new token (unless all have one)."""
    n, most, prior = case["seqs"], case.get("new", 1), case["prior"]
    if case["even"]:
        return [most] * n, [prior] * n
    rng = random.Random(case["lens_seed"])
    new = [most] + [_log_int(rng, 1, most) if i % 8 != 3 or most == 1 else 0 for i in range(1, n)]
    return new, [prior] + [_log_int(rng, 1, prior + 1) - 1 for _ in range(1, n)]


# ---- inputs ----

def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed((int(seed) * 1000003 + 4721) & 0x7FFFFFFFFFFFFFFF)
    return g


def _type(name):
    return torch.float32 if name == "f32" else torch.bfloat16


def _pages(lengths, page, g):
    """A page table (sequences, most pages) of pages in no order, unused entries -1, and the number of pages."""
    need = [-(-n // page) for n in lengths]
    total = max(1, sum(need))
    order = torch.randperm(total, generator=g, device="cuda").to(torch.int32)
    table = torch.full((len(lengths), max(1, max(need))), -1, dtype=torch.int32, device="cuda")
    at = 0
    for i, n in enumerate(need):
        table[i, :n] = order[at:at + n]
        at += n
    return table, total


def _inputs(case, seed):
    g = _generator(seed)

    def normal(*shape, scale=1.0, dtype=None):
        return torch.randn(shape, generator=g, device="cuda").mul_(scale).to(dtype or _type(case["io"]))

    kind = case["kind"]
    if kind == "gated":
        rows, width = case["rows"], case["width"]
        # the input projection's output: the gate is its first columns
        proj = normal(rows, width + 64)
        return dict(y=normal(rows, width), z=proj[:, :width], weight=1.0 + normal(width, scale=0.1, dtype=torch.float32))
    if kind == "residual":
        rows, width = case["rows"], case["width"]
        return dict(x=normal(rows, width), residual=normal(rows, width, scale=3.0, dtype=_type(case["stream"])),
                    weight=1.0 + normal(width, scale=0.1, dtype=torch.float32))
    H, Hk, D, page = case["heads"], case["kv_heads"], case["headdim"], case["page"]
    new, prior = _lengths(case)
    lengths = [a + b for a, b in zip(new, prior)]
    table, total = _pages(lengths, page, g)
    s = dict(table=table, lens=torch.tensor(lengths, dtype=torch.int32, device="cuda"))
    cu = [0]
    for n in new:
        cu.append(cu[-1] + n)
    if kind == "prompt" or any(n != 1 for n in new):
        s["cu"] = torch.tensor(cu, dtype=torch.int32, device="cuda")
    tokens = cu[-1]
    s["k_cache"] = normal(total, Hk, page, D)
    s["v_cache"] = normal(total, Hk, page, D)
    if kind == "append":
        # one projection gives queries, keys and values: the three are slices of its output
        qkv = normal(tokens, (H + 2 * Hk) * D)
        s["q"] = qkv[:, :H * D].view(tokens, H, D)
        s["k"] = qkv[:, H * D:(H + Hk) * D].view(tokens, Hk, D)
        s["v"] = qkv[:, (H + Hk) * D:].view(tokens, Hk, D)
        half = case["rotary"] // 2
        at = torch.arange(table.shape[1] * page, dtype=torch.float64, device="cuda")
        freq = ROPE_THETA ** (-torch.arange(half, dtype=torch.float64, device="cuda") / half)
        angle = at[:, None] * freq[None, :]
        s["cos"], s["sin"] = angle.cos().float(), angle.sin().float()
    else:
        s["q"] = normal(tokens, H, D, scale=LOGIT_SCALE)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    io = _type(case["io"])
    if case["kind"] in ("gated", "residual"):
        key = "y" if case["kind"] == "gated" else "x"
        s["out"] = torch.empty_like(s[key])
        if case["kind"] == "residual":
            s["residual_out"] = torch.empty_like(s["residual"])
    else:
        s["out"] = torch.empty(s["q"].shape, dtype=io, device="cuda")
        s["new"], prior = _lengths(case)
        s["lengths"] = [a + b for a, b in zip(s["new"], prior)]
    if own and case["kind"] in ("step", "prompt"):
        from paper_2603_09555_amd import ssd
        shape = ssd.make_attn_shape(len(s["lengths"]), s["q"].shape[0], case["heads"], s["k_cache"], s["table"], case["window"])
        need = ssd.attn_step_workspace_bytes(shape) if case["kind"] == "step" else ssd.attn_prefill_workspace_bytes(shape)
        s["workspace"] = torch.empty((max(need, 256),), dtype=torch.uint8, device="cuda")
    return s


# ---- one pass ----

def run(state):
    case = state["case"]
    return (_run_own if own else _run_plain)(case, state)


def _run_own(case, s):
    from paper_2603_09555_amd import ssd
    kind = case["kind"]
    if kind == "gated":
        return ssd.ssd_norm_gated(s["y"], s["z"], s["weight"], eps=EPS, groups=case["groups"], norm_first=case["norm_first"], out=s["out"])
    if kind == "residual":
        return ssd.ssd_norm_residual(s["residual"], s["x"], s["weight"], scale=case["scale"], eps=EPS, out=s["out"],
                                     residual_out=s["residual_out"])
    if kind == "append":
        q = ssd.ssd_attn_append(s["q"], s["k"], s["v"], s["k_cache"], s["v_cache"], s["table"], s["lens"], cu_seqlens=s.get("cu"),
                                rope=(s["cos"], s["sin"]), interleaved=case["interleaved"], q_out=s["out"])
        return q, s["k_cache"], s["v_cache"]
    if kind == "step":
        return ssd.ssd_attn_step(s["q"], s["k_cache"], s["v_cache"], s["table"], s["lens"], window=case["window"], y=s["out"],
                                 workspace=s["workspace"])
    return ssd.ssd_attn_prefill(s["q"], s["k_cache"], s["v_cache"], s["table"], s["lens"], s["cu"], window=case["window"], y=s["out"],
                                workspace=s["workspace"])


def _run_plain(case, s):
    return dict(gated=_plain_gated, residual=_plain_residual, append=_plain_append, step=_plain_step, prompt=_plain_prompt)[case["kind"]](case, s)


def _plain_gated(case, s):
    y, z = s["y"].float(), s["z"].float()
    gate = z / (1.0 + torch.exp(-z))
    v = y if case["norm_first"] else y * gate
    v = v.view(case["rows"], case["groups"], -1)
    v = v / torch.sqrt((v * v).mean(dim=2, keepdim=True) + EPS)
    v = v.view(case["rows"], -1) * s["weight"]
    if case["norm_first"]:
        v = v * gate
    return v.to(s["y"].dtype)


def _plain_residual(case, s):
    r = s["residual"].float() + case["scale"] * s["x"].float()
    out = r / torch.sqrt((r * r).mean(dim=1, keepdim=True) + EPS) * s["weight"]
    return out.to(s["x"].dtype), r.to(s["residual"].dtype)


def _token_positions(s):
    """Sequence and position of every new token."""
    new = torch.tensor(s["new"], device="cuda")
    seq = torch.repeat_interleave(torch.arange(len(s["new"]), device="cuda"), new)
    first = torch.cumsum(new, 0) - new
    at = torch.arange(seq.numel(), device="cuda") - first[seq]
    return seq, s["lens"].long()[seq] - new[seq] + at


def _rotate(t, cos, sin, interleaved):
    half = cos.shape[2]
    t = t.float()
    a, b = (t[..., 0:2 * half:2], t[..., 1:2 * half:2]) if interleaved else (t[..., :half], t[..., half:2 * half])
    ra, rb = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack((ra, rb), dim=-1).flatten(-2) if interleaved else torch.cat((ra, rb), dim=-1)
    return torch.cat((turned, t[..., 2 * half:]), dim=-1)


def _plain_append(case, s):
    seq, pos = _token_positions(s)
    cos, sin = s["cos"][pos][:, None], s["sin"][pos][:, None]
    io = s["q"].dtype
    page = s["table"].long()[seq, pos // case["page"]]
    s["k_cache"][page, :, pos % case["page"]] = _rotate(s["k"], cos, sin, case["interleaved"]).to(io)
    s["v_cache"][page, :, pos % case["page"]] = s["v"]
    return _rotate(s["q"], cos, sin, case["interleaved"]).to(io), s["k_cache"], s["v_cache"]


def _softmax(scores):
    e = torch.exp(scores - scores.amax(dim=-1, keepdim=True))
    return e / e.sum(dim=-1, keepdim=True)


def _plain_step(case, s):
    B, H, Hk, D, page = len(s["lengths"]), case["heads"], case["kv_heads"], case["headdim"], case["page"]
    table = s["table"].long().clamp(min=0)
    k = s["k_cache"][table].float().permute(0, 2, 1, 3, 4).reshape(B, Hk, -1, D)
    q = s["q"].float().view(B, Hk, H // Hk, D)
    scores = torch.matmul(q, k.transpose(2, 3)) * (D ** -0.5)
    del k
    at = torch.arange(table.shape[1] * page, device="cuda")
    lens = s["lens"].long()[:, None]
    seen = at[None, :] < lens
    if case["window"] > 0:
        seen &= at[None, :] >= lens - case["window"]
    p = _softmax(torch.where(seen[:, None, None, :], scores, float("-inf")))
    v = s["v_cache"][table].float().permute(0, 2, 1, 3, 4).reshape(B, Hk, -1, D)
    return torch.matmul(p, v).view(B, H, D).to(s["q"].dtype)


def _plain_prompt(case, s):
    H, Hk, D, page = case["heads"], case["kv_heads"], case["headdim"], case["page"]
    G = H // Hk
    out = s["out"]
    first = 0
    for i, (n, length) in enumerate(zip(s["new"], s["lengths"])):
        if n == 0:
            continue
        pages = s["table"][i, :-(-length // page)].long()
        k = s["k_cache"][pages].permute(1, 0, 2, 3).reshape(Hk, -1, D)[:, :length].float()
        v = s["v_cache"][pages].permute(1, 0, 2, 3).reshape(Hk, -1, D)[:, :length].float()
        block = max(1, min(n, (1 << 28) // (H * length)))
        for a in range(0, n, block):
            b = min(n, a + block)
            q = s["q"][first + a:first + b].float().view(b - a, Hk, G, D).permute(1, 2, 0, 3).reshape(Hk, G * (b - a), D)
            scores = torch.matmul(q, k.transpose(1, 2)).view(Hk, G, b - a, length) * (D ** -0.5)
            pos = (length - n + torch.arange(a, b, device="cuda"))[:, None]
            at = torch.arange(length, device="cuda")[None, :]
            seen = at <= pos
            if case["window"] > 0:
                seen &= at > pos - case["window"]
            p = _softmax(torch.where(seen, scores, float("-inf"))).view(Hk, G * (b - a), length)
            y = torch.matmul(p, v).view(Hk, G, b - a, D).permute(2, 0, 1, 3)
            out[first + a:first + b] = y.reshape(b - a, H, D).to(out.dtype)
        first += n
    return out


# ---- what a pass cannot do without ----

def work(case):
    size = 4 if case["io"] == "f32" else 2
    kind = case["kind"]
    if kind == "gated":
        n = case["rows"] * case["width"]
        return dict(bytes=3 * n * size + 4 * case["width"], flops=8 * n)
    if kind == "residual":
        n = case["rows"] * case["width"]
        return dict(bytes=2 * n * size + 2 * n * (4 if case["stream"] == "f32" else 2) + 4 * case["width"], flops=6 * n)
    H, Hk, D = case["heads"], case["kv_heads"], case["headdim"]
    new, prior = _lengths(case)
    if kind == "append":
        t = sum(new)
        return dict(bytes=2 * t * (H + 2 * Hk) * D * size + 4 * t * case["rotary"], flops=3 * t * (H + Hk) * case["rotary"])
    window = case["window"]
    if kind == "step":
        seen = sum(min(n + 1, window) if window > 0 else n + 1 for n in prior)
        return dict(bytes=2 * seen * Hk * D * size + 2 * len(prior) * H * D * size, flops=4 * seen * H * D)
    pairs = kv = 0
    for n, p in zip(new, prior):
        if n == 0:
            continue
        if window > 0:
            full = max(0, min(n, n + p - window))          # tokens that see a whole window
            rest = n - full                                # the others see all that is in front of them
            pairs += full * window + rest * p + rest * (rest + 1) // 2
            kv += min(n + p, n + window - 1)
        else:
            pairs += n * p + n * (n + 1) // 2
            kv += n + p
    return dict(bytes=2 * kv * Hk * D * size + 2 * sum(new) * H * D * size, flops=4 * pairs * H * D)


# ---- the definitions, in 64 bits ----

def exact(case, seed):
    s = _inputs(case, seed)
    kind = case["kind"]
    if kind == "gated":
        y, z, w = s["y"].double(), s["z"].double(), s["weight"].double()
        gate = z * torch.sigmoid(z)
        cols = case["width"] // case["groups"]
        out = torch.empty_like(y)
        for a in range(0, case["width"], cols):
            part = slice(a, a + cols)
            u = y[:, part] if case["norm_first"] else y[:, part] * gate[:, part]
            u = u * torch.rsqrt(u.pow(2).sum(1, keepdim=True) / cols + EPS) * w[part]
            out[:, part] = u * gate[:, part] if case["norm_first"] else u
        return out
    if kind == "residual":
        r = torch.add(s["residual"].double(), s["x"].double(), alpha=case["scale"])
        return r * torch.rsqrt(r.square().sum(1, keepdim=True) / case["width"] + EPS) * s["weight"].double(), r
    D, page, Hk = case["headdim"], case["page"], case["kv_heads"]
    new, prior = _lengths(case)
    lengths = [a + b for a, b in zip(new, prior)]
    if kind == "append":
        k_cache, v_cache = s["k_cache"].double(), s["v_cache"].double()
        half = case["rotary"] // 2
        q_out = s["q"].double()
        k = s["k"].double()
        v = s["v"].double()
        if case["interleaved"]:
            even, odd = slice(0, 2 * half, 2), slice(1, 2 * half, 2)
        else:
            even, odd = slice(0, half), slice(half, 2 * half)
        first = 0
        for i, (n, length) in enumerate(zip(new, lengths)):
            at = slice(first, first + n)
            c, d = s["cos"][length - n:length].double()[:, None], s["sin"][length - n:length].double()[:, None]
            for t in (q_out, k):
                turn = torch.complex(t[at, :, even], t[at, :, odd]) * torch.complex(c, d)
                t[at, :, even], t[at, :, odd] = turn.real, turn.imag
            done = 0
            while done < n:                                 # a page at a time
                p, o = divmod(length - n + done, page)
                m = min(page - o, n - done)
                where = int(s["table"][i, p])
                k_cache[where, :, o:o + m] = k[first + done:first + done + m].transpose(0, 1)
                v_cache[where, :, o:o + m] = v[first + done:first + done + m].transpose(0, 1)
                done += m
            first += n
        return q_out, k_cache, v_cache
    G = case["heads"] // Hk
    out = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
    first = 0
    for i, (n, length) in enumerate(zip(new, lengths)):
        if n == 0:
            continue
        lo = 0 if case["window"] <= 0 else max(0, length - n + 1 - case["window"])      # what the first of them sees first
        at = torch.arange(lo, length, device="cuda")
        where, slot = s["table"][i].long()[at // page], at % page
        for h in range(Hk):
            k, v = s["k_cache"][where, h, slot].double(), s["v_cache"][where, h, slot].double()
            rows = max(1, (1 << 28) // (G * at.numel()))
            for a in range(0, n, rows):
                b = min(n, a + rows)
                q = s["q"][first + a:first + b, h * G:(h + 1) * G].double()
                scores = torch.tensordot(q, k, dims=([2], [1])).div_(math.sqrt(D))
                pos = torch.arange(length - n + a, length - n + b, device="cuda").view(-1, 1, 1)
                hide = at > pos
                if case["window"] > 0:
                    hide |= pos - at >= case["window"]
                p = torch.softmax(scores.masked_fill_(hide, -math.inf), dim=2)
                out[first + a:first + b, h * G:(h + 1) * G] = torch.tensordot(p, v, dims=([2], [0]))
        first += n
    return out

