"""A small hybrid stack on this library: Mamba-2 or Mamba-1 blocks with an attention block among them, as a server runs it -- a
packed, ragged batch of prompts (or later pieces of them), then one token for every sequence at a time.

Every block normalises the residual stream (``ssd_norm_residual``, which also takes up the block before).  A Mamba-2 block is
projection, convolution (``ssd_conv1d_varlen`` or ``ssd_conv1d_step``), SSD core, gated norm (``ssd_norm_gated``), projection; a
Mamba-1 block is projection, convolution, projection to step sizes, B and C, selective scan with its gate
(``ssd_selective_prefill`` or ``ssd_selective_step``), projection; an attention block is projection, append to the paged cache
with rotation (``ssd_attn_append``, or ``ssd_attn_append_norm`` where heads are normalised), attention over it
(``ssd_attn_prefill`` or ``ssd_attn_step``), projection.
Projections are plain matrix products.  Weights are random: this shows the calls, and ``python -m paper_2603_09555_amd.hybrid``
checks that prompts continued token by token give what longer prompts give.
"""
from __future__ import annotations

import math
from dataclasses import dataclass, field

import torch

from . import ssd


@dataclass(frozen=True)
class HybridConfig:
    width: int = 256
    blocks: str = "MMAM"        # M: Mamba-2, S: Mamba-1 (selective scan), A: attention
    nheads: int = 8             # of the SSD core
    headdim: int = 64
    dstate: int = 128
    ngroups: int = 1
    conv_taps: int = 4
    chunk: int = 256
    attn_heads: int = 8
    attn_kv_heads: int = 2
    attn_headdim: int = 64
    rotary: int = 64
    window: int = 0             # of the attention blocks, 0: all tokens
    page_size: int = 16
    residual_scale: float = 1.0
    eps: float = 1e-5
    selective_states: int = 16  # of a channel of a Mamba-1 block, which has nheads * headdim of them
    head_norm: bool = False     # queries and keys of the attention blocks are normalised, head by head


@dataclass
class HybridCache:
    """What a batch of sequences leaves between calls.  ``lens`` counts the tokens of each sequence, ``held`` on the host."""
    lens: torch.Tensor                     # (batch) int32
    page_table: torch.Tensor               # (batch, max_pages) int32
    conv: dict = field(default_factory=dict)    # block -> (batch, channels, taps - 1)
    state: dict = field(default_factory=dict)   # block -> (batch, nheads, headdim, dstate), (batch, channels, states) fp32
    keys: dict = field(default_factory=dict)    # block -> (npages, kv_heads, page_size, headdim)
    values: dict = field(default_factory=dict)
    workspace: torch.Tensor | None = None       # of the single-token attention, kept from step to step
    held: list | None = None                    # lens on the host (None: not read yet)


class HybridStack:
    def __init__(self, config: HybridConfig, dtype=torch.bfloat16, seed: int = 0, device="cuda"):
        self.config, self.dtype, self.device = config, dtype, device
        g = torch.Generator(device="cpu").manual_seed(seed)
        c = config

        def weight(rows, cols):
            return (torch.randn((rows, cols), generator=g) / math.sqrt(rows)).to(dtype).to(device)

        def vector(n, mean, spread):
            return (mean + spread * torch.randn((n,), generator=g)).to(device)

        self.inner = c.nheads * c.headdim
        self.conv_split = (self.inner, c.ngroups * c.dstate, c.ngroups * c.dstate)
        self.rank = -(-c.width // 16)       # of a Mamba-1 block's step sizes
        self.blocks = []
        for kind in c.blocks:
            b = {"kind": kind, "norm": vector(c.width, 1.0, 0.1)}
            if kind == "M":
                channels = sum(self.conv_split)
                b["in"] = weight(c.width, self.inner + channels + c.nheads)      # gate | convolution's channels | step sizes
                b["conv_w"] = torch.randn((channels, c.conv_taps), generator=g).to(device) / c.conv_taps
                b["conv_b"] = vector(channels, 0.0, 0.1)
                b["A"] = -(torch.rand((c.nheads,), generator=g) * 8 + 0.5).to(device)
                b["D"] = vector(c.nheads, 0.0, 1.0)
                b["dt_bias"] = vector(c.nheads, math.log(math.expm1(1e-2)), 0.1)
                b["gate_norm"] = vector(self.inner, 1.0, 0.1)
                b["out"] = weight(self.inner, c.width)
            elif kind == "S":
                N = c.selective_states
                b["in"] = weight(c.width, 2 * self.inner)                         # the convolution's channels | gate
                b["conv_w"] = torch.randn((self.inner, c.conv_taps), generator=g).to(device) / c.conv_taps
                b["conv_b"] = vector(self.inner, 0.0, 0.1)
                b["mix"] = weight(self.inner, self.rank + 2 * N)                  # step sizes' low-rank form | B | C
                b["dt"] = weight(self.rank, self.inner)
                b["dt_bias"] = vector(self.inner, math.log(math.expm1(1e-2)), 0.5)
                b["A"] = -(torch.arange(1, N + 1) * (0.3 * torch.randn((self.inner, N), generator=g)).exp()).to(device)
                b["D"] = vector(self.inner, 0.0, 1.0)
                b["out"] = weight(self.inner, c.width)
            else:
                heads = c.attn_heads + 2 * c.attn_kv_heads
                b["in"] = weight(c.width, heads * c.attn_headdim)
                b["out"] = weight(c.attn_heads * c.attn_headdim, c.width)
                if c.head_norm:
                    b["q_norm"], b["k_norm"] = (vector(c.attn_headdim, 1.0, 0.1) for _ in range(2))
            self.blocks.append(b)
        self.final_norm = vector(c.width, 1.0, 0.1)
        self.rope = None

    def new_cache(self, batch: int, max_tokens: int, seed: int = 0) -> HybridCache:
        """Empty sequences with pages for ``max_tokens`` each (a server would take pages from its pool as sequences grow)."""
        c = self.config
        pages = -(-max_tokens // c.page_size)
        order = torch.randperm(batch * pages, generator=torch.Generator().manual_seed(seed))
        cache = HybridCache(torch.zeros((batch,), dtype=torch.int32, device=self.device),
                            order.to(torch.int32).view(batch, pages).to(self.device), held=[0] * batch)
        for i, b in enumerate(self.blocks):
            if b["kind"] == "M":
                cache.conv[i] = torch.zeros((batch, sum(self.conv_split), c.conv_taps - 1), dtype=self.dtype, device=self.device)
                cache.state[i] = torch.zeros((batch, c.nheads, c.headdim, c.dstate), device=self.device)
            elif b["kind"] == "S":
                cache.conv[i] = torch.zeros((batch, self.inner, c.conv_taps - 1), dtype=self.dtype, device=self.device)
                cache.state[i] = torch.zeros((batch, self.inner, c.selective_states), device=self.device)
            else:
                shape = (batch * pages, c.attn_kv_heads, c.page_size, c.attn_headdim)
                cache.keys[i] = torch.empty(shape, dtype=self.dtype, device=self.device)
                cache.values[i] = torch.empty(shape, dtype=self.dtype, device=self.device)
        capacity = pages * c.page_size
        if self.rope is None or self.rope[0].shape[0] < capacity:   # a row for every position a page table row can hold
            half = c.rotary // 2
            angle = torch.arange(capacity, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(half, dtype=torch.float64) / half)
            self.rope = (angle.cos().float().to(self.device), angle.sin().float().to(self.device))
        return cache

    def _grow(self, cache, new):
        """Sequences get ``new`` tokens each, for which there must be pages."""
        if cache.held is None:
            cache.held = cache.lens.tolist()
        held = [h + n for h, n in zip(cache.held, new, strict=True)]
        if max(held) > cache.page_table.shape[1] * self.config.page_size:
            raise ValueError("a sequence has outgrown its pages")
        cache.held = held

    def _mamba(self, i, b, h, cache, cu):
        """``cu``: boundaries of the sequences' new tokens, or None for one each."""
        c = self.config
        G, N = c.ngroups, c.dstate
        proj = h @ b["in"]
        z = proj[:, :self.inner]
        u = proj[:, self.inner:self.inner + sum(self.conv_split)]
        dt = proj[:, -c.nheads:].float().contiguous()
        heads = (c.nheads, c.headdim)
        if cu is None:
            x, B, C = ssd.ssd_conv1d_step(cache.conv[i], u.contiguous(), b["conv_w"], b["conv_b"], split=self.conv_split)
            y = ssd.ssd_decode_step_layers(cache.state[i][None], x.view(1, -1, *heads), dt[None], b["A"][None], B.view(1, -1, G, N),
                                           C.view(1, -1, G, N), b["D"][None], dt_bias=b["dt_bias"][None], dt_softplus=True)[0]
        else:
            (x, B, C), _ = ssd.ssd_conv1d_varlen(u, b["conv_w"], b["conv_b"], cu, cache.conv[i], split=self.conv_split,
                                                 conv_state_out=cache.conv[i])
            y, _ = ssd.ssd_prefill_varlen(x.view(-1, *heads), dt, b["A"], B.view(-1, G, N), C.view(-1, G, N), b["D"], cu, c.chunk,
                                          h0=cache.state[i], final_state=cache.state[i], dt_bias=b["dt_bias"], dt_softplus=True)
        y = ssd.ssd_norm_gated(y.reshape(-1, self.inner), z, b["gate_norm"], eps=c.eps)
        return y @ b["out"]

    def _selective(self, i, b, h, cache, cu):
        proj = h @ b["in"]
        u, z = proj[:, :self.inner], proj[:, self.inner:]
        if cu is None:
            x, = ssd.ssd_conv1d_step(cache.conv[i], u.contiguous(), b["conv_w"], b["conv_b"])
        else:
            (x,), _ = ssd.ssd_conv1d_varlen(u, b["conv_w"], b["conv_b"], cu, cache.conv[i], conv_state_out=cache.conv[i])
        low, B, C = (x @ b["mix"]).split((self.rank, self.config.selective_states, self.config.selective_states), dim=1)
        args = (x, low @ b["dt"], b["A"], B, C, b["D"])
        step = dict(z=z, dt_bias=b["dt_bias"], dt_softplus=True)
        if cu is None:
            y = ssd.ssd_selective_step(cache.state[i], *args, **step)
        else:
            y, _ = ssd.ssd_selective_prefill(*args, cu, h0=cache.state[i], final_state=cache.state[i], **step)
        return y @ b["out"]

    def _attention(self, i, b, h, cache, cu):
        c = self.config
        H, Hk, D = c.attn_heads, c.attn_kv_heads, c.attn_headdim
        q, k, v = (h @ b["in"]).view(-1, H + 2 * Hk, D).split((H, Hk, Hk), dim=1)     # slices of one projection's output
        to = (cache.keys[i], cache.values[i], cache.page_table, cache.lens, cu)
        if c.head_norm:
            q = ssd.ssd_attn_append_norm(q, k, v, b["q_norm"], b["k_norm"], *to, rope=self.rope, eps=c.eps)
        else:
            q = ssd.ssd_attn_append(q, k, v, *to, rope=self.rope)
        if cu is None:
            if cache.workspace is None:
                shape = ssd.make_attn_shape(q.shape[0], q.shape[0], H, cache.keys[i], cache.page_table, c.window)
                cache.workspace = torch.empty((max(256, ssd.attn_step_workspace_bytes(shape)),), dtype=torch.uint8, device=self.device)
            y = ssd.ssd_attn_step(q, cache.keys[i], cache.values[i], cache.page_table, cache.lens, window=c.window, workspace=cache.workspace)
        else:
            y = ssd.ssd_attn_prefill(q, cache.keys[i], cache.values[i], cache.page_table, cache.lens, cu, window=c.window)
        return y.view(-1, H * D) @ b["out"]

    def _run(self, x, cache, cu):
        c = self.config
        mixer = {"M": self._mamba, "S": self._selective, "A": self._attention}
        out, residual, scale = x, None, 1.0
        for i, b in enumerate(self.blocks):
            h, residual = ssd.ssd_norm_residual(residual, out, b["norm"], scale=scale, eps=c.eps, residual_out=residual)
            out = mixer[b["kind"]](i, b, h, cache, cu)
            scale = c.residual_scale
        return ssd.ssd_norm_residual(residual, out, self.final_norm, scale=scale, eps=c.eps, residual_out=residual)[0]

    def prefill(self, x, lengths, cache: HybridCache):
        """``x (tokens,width)``: ``lengths[b]`` new tokens of every sequence, packed.  Returns the normalised stream of every token."""
        if x.shape[0] != sum(lengths):
            raise ValueError("x must hold the sequences' new tokens")
        self._grow(cache, lengths)
        new = torch.tensor(lengths, dtype=torch.int32)
        cu = torch.cat((torch.zeros(1, dtype=torch.int32), new.cumsum(0).to(torch.int32))).to(self.device)
        cache.lens += new.to(self.device)
        return self._run(x, cache, cu)

    def step(self, x, cache: HybridCache):
        """``x (batch,width)``: one new token of every sequence."""
        self._grow(cache, [1] * len(cache.lens))
        cache.lens += 1
        return self._run(x, cache, None)


def check(dtype=torch.bfloat16, lengths=(70, 1, 333), steps=5, config=HybridConfig(), seed=0) -> float:
    """Prompts continued token by token against prompts that hold these tokens: the largest difference over the largest value."""
    stack = HybridStack(config, dtype, seed)
    g = torch.Generator().manual_seed(seed + 1)
    embed = [torch.randn((n + steps, config.width), generator=g).to(dtype).cuda() for n in lengths]
    whole = stack.new_cache(len(lengths), max(lengths) + steps)
    ref = stack.prefill(torch.cat(embed), [n + steps for n in lengths], whole)
    ends = torch.tensor(lengths).cumsum(0) + steps * torch.arange(1, len(lengths) + 1)
    grown = stack.new_cache(len(lengths), max(lengths) + steps, seed=1)
    # (prompts come in two pieces each)
    halves = [n // 2 for n in lengths]
    if sum(halves):
        stack.prefill(torch.cat([e[:k] for e, k in zip(embed, halves)]), halves, grown)
    stack.prefill(torch.cat([e[k:n] for e, k, n in zip(embed, halves, lengths)]), [n - k for n, k in zip(lengths, halves)], grown)
    worst = 0.0
    for t in range(steps):
        y = stack.step(torch.stack([e[n + t] for e, n in zip(embed, lengths)]), grown)
        at = (ends - steps + t).to(ref.device)
        worst = max(worst, float((y.float() - ref[at].float()).abs().max() / ref[at].float().abs().max()))
    return worst


def main():
    for config in (HybridConfig(), HybridConfig(blocks="SSAS", head_norm=True)):
        for dtype in (torch.float32, torch.bfloat16):
            print("%s: prompts continued by tokens against longer prompts, %s: largest difference %.2e of the largest value"
                  % (config.blocks, dtype, check(dtype, config=config)))


if __name__ == "__main__":
    main()
