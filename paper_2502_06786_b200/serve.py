"""A small decoder served from its nested weights: prompts, chunks of prompts, drafted and single tokens.

    python -m paper_2502_06786_b200.serve

Shows the serving calls as they are used together.  A layer keeps its matrices once as 8-bit codes and serves a nested precision r of them: up to
``FEW`` tokens go through the decode GEMV on the packed plane (``gemv_grouped``), more through the 8-bit tensor-core product on the unpacked
slice (``quantize_tokens`` once per input, ``gemm_a8`` per matrix).  New keys and values are rotated and appended to a paged cache
(``kv_append``), and the new tokens attend to it (``attn_paged``).  Norms, activations and residual sums are plain torch.
"""
from __future__ import annotations

from dataclasses import dataclass

import torch

from . import binding as mq

FEW = 8


@dataclass
class Config:
    hidden: int = 512
    ffn: int = 1024
    q_heads: int = 8
    kv_heads: int = 2
    head_dim: int = 64
    layers: int = 2
    r: int = 4                  # nested precision that is served
    window: int = 0
    softcap: float = 0.0
    page_size: int = 16
    max_pos: int = 4096
    theta: float = 10000.0


class Linear:
    """One matrix, quantised to 8-bit codes and sliced to r bits: a packed plane for few tokens, the unpacked slice for many."""

    def __init__(self, W: torch.Tensor, r: int):
        self.N, self.K = W.shape
        self.r = r
        q, self.alpha, self.zero = mq.quantize(W)
        out = mq.slice_pack(q, r, want_unpacked=True)
        self.packed, self.sliced = out["packed"], out["sliced"]


def apply(linears, x):
    """The products of one input [T, K] (bf16) with several matrices: bf16 [T, N] each."""
    T = x.shape[0]
    if T <= FEW:
        ys = [torch.empty((T, l.N), dtype=torch.float32, device=x.device) for l in linears]
        mq.gemv_grouped([dict(packed=l.packed, K=l.K, r=l.r, alpha=l.alpha, zero=l.zero, x=x if T > 1 else x[0], y=y if T > 1 else y[0])
                         for l, y in zip(linears, ys)])
        return [y.to(torch.bfloat16) for y in ys]
    xq, scale, rowsum = mq.quantize_tokens(x)
    return [mq.gemm_a8(xq, scale, rowsum, l.sliced, l.alpha, l.zero, out_dtype=torch.bfloat16, flags=mq.GEMV_PDL) for l in linears]


class PagedCache:
    """Keys and values of all layers in pages, and which pages belong to which sequence.  The page numbers are the same in every layer."""

    def __init__(self, cfg: Config, n_pages: int, device="cuda"):
        shape = (n_pages, cfg.kv_heads, cfg.page_size, cfg.head_dim)
        self.k = [torch.empty(shape, dtype=torch.bfloat16, device=device) for _ in range(cfg.layers)]
        self.v = [torch.empty(shape, dtype=torch.bfloat16, device=device) for _ in range(cfg.layers)]
        self.page_size, self.free = cfg.page_size, list(range(n_pages - 1, -1, -1))
        self.pages, self.length = {}, {}

    def extend(self, seq, n: int) -> None:
        """Makes room for n more tokens of a sequence."""
        self.extend_all([(seq, n)])

    def extend_all(self, steps) -> None:
        """Makes room for (sequence, number of new tokens) pairs: for all of them, or, if the pages do not suffice, for none."""
        length = {seq: self.length.get(seq, 0) + n for seq, n in steps}
        if len(length) != len(steps):
            raise ValueError("a sequence occurs twice")
        need = {seq: -(-t // self.page_size) - len(self.pages.get(seq, ())) for seq, t in length.items()}
        if sum(need.values()) > len(self.free):
            raise RuntimeError("the cache is full")
        for seq, t in length.items():
            self.pages.setdefault(seq, []).extend(self.free.pop() for _ in range(need[seq]))
            self.length[seq] = t

    def release(self, seq) -> None:
        self.free.extend(reversed(self.pages.pop(seq)))
        del self.length[seq]


class Batch:
    """The device arrays that one step's calls share: (sequence, number of new tokens) pairs, their pages and lengths."""

    def __init__(self, cache: PagedCache, steps, device="cuda"):
        cache.extend_all(steps)
        width = max(len(cache.pages[s]) for s, _ in steps)
        table = [cache.pages[s] + [-1] * (width - len(cache.pages[s])) for s, _ in steps]
        cu = [0]
        for _, n in steps:
            cu.append(cu[-1] + n)
        lens = [cache.length[s] for s, _ in steps]
        self.page_table = torch.tensor(table, dtype=torch.int32, device=device)
        self.cu_q = torch.tensor(cu, dtype=torch.int32, device=device)
        self.kv_len = torch.tensor(lens, dtype=torch.int32, device=device)
        self.max_q, self.max_kv = max(n for _, n in steps), max(lens)


def rms_norm(x):
    f = x.float()
    return (f * torch.rsqrt(f.square().mean(-1, keepdim=True) + 1e-6)).to(torch.bfloat16)


class Decoder:
    """A decoder with random weights (std 0.02) quantised to 8 bits."""

    def __init__(self, cfg: Config, seed: int = 0, device="cuda"):
        self.cfg = cfg
        g = torch.Generator(device=device).manual_seed(seed)

        def linear(n, k):
            return Linear((torch.randn(n, k, generator=g, device=device) * 0.02).to(torch.bfloat16), cfg.r)
        d, f, D = cfg.hidden, cfg.ffn, cfg.head_dim
        self.layers = [dict(q=linear(cfg.q_heads * D, d), k=linear(cfg.kv_heads * D, d), v=linear(cfg.kv_heads * D, d), o=linear(d, cfg.q_heads * D),
                            gate=linear(f, d), up=linear(f, d), down=linear(d, f)) for _ in range(cfg.layers)]
        half = D // 2
        freq = cfg.theta ** (-torch.arange(half, dtype=torch.float64, device=device) / half)
        angle = torch.arange(cfg.max_pos, dtype=torch.float64, device=device)[:, None] * freq
        self.cos_sin = torch.cat([angle.cos(), angle.sin()], 1).float().contiguous()

    def forward(self, x: torch.Tensor, cache: PagedCache, batch: Batch, dev_status=None) -> torch.Tensor:
        """x: bf16 [T, hidden], the new tokens of the batch's sequences one after another.  Returns bf16 [T, hidden]."""
        cfg, T = self.cfg, x.shape[0]
        if batch.max_kv > cfg.max_pos:
            raise ValueError(f"a sequence of {batch.max_kv} tokens passes the {cfg.max_pos} positions of the rotation table")
        paged = (batch.page_table, batch.cu_q, batch.kv_len)
        for i, l in enumerate(self.layers):
            q, k, v = apply([l["q"], l["k"], l["v"]], rms_norm(x))
            q, k, v = (t.view(T, -1, cfg.head_dim) for t in (q, k, v))
            mq.kv_append(cache.k[i], cache.v[i], *paged, k, v, cos_sin=self.cos_sin, q=q, q_out=q, dev_status=dev_status)
            a = mq.attn_paged(q, cache.k[i], cache.v[i], *paged, batch.max_q, batch.max_kv, softcap=cfg.softcap, window=cfg.window, dev_status=dev_status)
            x = x + apply([l["o"]], a.view(T, -1))[0]
            gate, up = apply([l["gate"], l["up"]], rms_norm(x))
            x = x + apply([l["down"]], torch.nn.functional.silu(gate) * up)[0]
        return x


def main() -> None:
    cfg = Config()
    model, cache = Decoder(cfg), PagedCache(cfg, 64)
    g = torch.Generator(device="cuda").manual_seed(1)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    prompt = (torch.randn(100 + 37, cfg.hidden, generator=g, device="cuda")).to(torch.bfloat16)
    out = model.forward(prompt, cache, Batch(cache, [("a", 100), ("b", 37)]), status)            # two prompts in one step
    for _ in range(4):                                                                          # then a token each at a time
        out = model.forward(out[-2:], cache, Batch(cache, [("a", 1), ("b", 1)]), status)
    torch.cuda.synchronize()
    if int(status.item()) != mq.OK or not bool(torch.isfinite(out.float()).all()):
        raise SystemExit(f"serve: {mq.status_string(int(status.item()))}")
    print("ok", {s: cache.length[s] for s in cache.pages})


if __name__ == "__main__":
    main()
