"""An equivariant encoder of images and video on the library's layers.

    stem     rotation-equivariant 3 x 3 convolutions (``gconv``) with group norm and activation between (``norm``)
    tokens   the features of p x p pixels averaged, a frame in raster order, frames after one another, after a few
             register tokens
    blocks   ``EQViTBlock`` with rotary positions (time, height, width) and windowed attention (``attention``)

Every part commutes with the group action on the T axis.  Without a limit to the right every token sees as far ahead as
back; with ``right = 0`` a video can also be encoded frame by frame over caches (``EQEncoder.stream``), whose tokens are
those of the whole clip.

``python -m paper_2607_21271_amd.encoder`` trains a small encoder on synthetic clips for a few steps and streams one.
"""
from __future__ import annotations

import torch
import torch.nn.functional as F

from . import attention, rotary
from .blocks import EQViTBlock
from .gconv import GroupConv2d
from .norm import GroupNormAct


class EQWindowBlock(EQViTBlock):
    """``EQViTBlock`` whose attention has rotary positions and a window: x [B, L, C, T], positions [L, axes]."""

    def __init__(self, T: int, C: int, heads: int, sections, left: int = -1, right: int = -1, sinks: int = 0,
                 mlp_ratio: int = 4, device=None, dtype=None):
        super().__init__(T, C, heads, mlp_ratio, device=device, dtype=dtype)
        self.sections, self.left, self.right, self.sinks = tuple(sections), left, right, sinks
        self.register_buffer("freqs", rotary.axis_frequencies(self.sections, device=device), persistent=False)

    def _apply(self, fn, recurse=True):
        # the frequencies follow the weights to another device, not to another type: rounded to 16 bits they would turn a
        # token at position 2,048 wrong by tenths of a radian (fp16) or by radians (bf16)
        freqs = self.freqs
        super()._apply(fn, recurse)
        device = self.freqs.device
        self.freqs = rotary.axis_frequencies(self.sections, device=device) if freqs.is_meta else freqs.to(device)
        return self

    def heads_of(self, h):
        B, L = h.shape[:2]
        return h.view(B, L, 3 * self.heads, self.C // self.heads * self.T)

    def forward(self, x, positions=None, lengths=None):
        B, L = x.shape[:2]
        qkv = self.heads_of(self.qkv(self.norm1(x)))
        o = attention.packed_window_attention(qkv, self.heads, positions, self.freqs, self.sections, self.T,
                                              lengths=lengths, left=self.left, right=self.right, sinks=self.sinks)
        x = x + self.proj(o.view(B, L, self.C, self.T))
        return x + self.fc2(F.gelu(self.fc1(self.norm2(x))))

    @torch.no_grad()
    def extend(self, x, positions, cache, filled: int, lengths, starts):
        """``forward`` of the n newest tokens x [B, n, C, T], which take places filled .. filled + n of the cache (keys,
        values [B, capacity, heads, D]); lengths and starts are filled + n and filled for every sequence, int32 [B]."""
        B, n = x.shape[:2]
        H = self.heads
        if filled < 0 or any(filled + n > c.shape[1] for c in cache):
            raise ValueError("%d tokens from place %d on do not fit a cache of %d" % (n, filled, cache[0].shape[1]))
        qkv = self.heads_of(self.qkv(self.norm1(x)))
        rotary.rotary_axes_(qkv[:, :, :2 * H], positions, self.freqs, self.sections, self.T)
        for c, new in zip(cache, (qkv[:, :, H:2 * H], qkv[:, :, 2 * H:])):
            c[:, filled:filled + n] = new
        o = attention.window_attention(qkv[:, :, :H], *cache, left=self.left, right=self.right, sinks=self.sinks,
                                       lengths=lengths, starts=starts)
        x = x + self.proj(o.view(B, n, self.C, self.T))
        return x + self.fc2(F.gelu(self.fc1(self.norm2(x))))


class EQEncoder(torch.nn.Module):
    """Clips [B, frames, H, W, Cin, T] -> tokens [B, registers + frames * H/p * W/p, C, T]."""

    def __init__(self, T: int, Cin: int, C: int, heads: int, depth: int, sections, patch: int = 4, registers: int = 4,
                 left: int = -1, right: int = -1, stem: int = 2, groups: int = 4, activation: str = "silu", device=None,
                 dtype=None):
        super().__init__()
        kw = {"device": device, "dtype": dtype}
        self.T, self.C, self.patch = T, C, patch
        self.stem = torch.nn.ModuleList(torch.nn.ModuleList((GroupConv2d(T, Cin if i == 0 else C, C, **kw),
                                                             GroupNormAct(C, groups, activation, **kw)))
                                        for i in range(stem))
        # one value per channel, the same for every group element
        self.registers = torch.nn.Parameter(torch.randn(registers, C, 1, **kw) * 0.02)
        self.blocks = torch.nn.ModuleList(EQWindowBlock(T, C, heads, sections, left, right, registers, **kw)
                                          for _ in range(depth))

    def positions(self, frames, H, W, device, first: int = 0):
        """Of the tokens of frames first .. first + frames - 1, after the registers where first is 0."""
        p = rotary.grid_positions((frames, H // self.patch, W // self.patch), 0 if first else len(self.registers),
                                  device)
        if first:
            p[:, 0] += first
        return p

    def tokens(self, clip):
        """The stem's tokens [B, frames * H/p * W/p, C, T]."""
        B, N, H, W = clip.shape[:4]
        p = self.patch
        if clip.dim() != 6 or H % p or W % p:
            raise ValueError("clips are [B, frames, H, W, Cin, T] with H, W multiples of %d, got %s" % (p, tuple(clip.shape)))
        f = clip.reshape(B * N, H, W, *clip.shape[4:])
        for conv, norm in self.stem:
            f = norm(conv(f))
        f = f.view(B * N, H // p, p, W // p, p, self.C, self.T).mean((2, 4))
        return f.reshape(B, -1, self.C, self.T)

    def _with_registers(self, x):
        return torch.cat((self.registers.expand(x.shape[0], -1, self.C, self.T), x), 1)

    def forward(self, clip):
        x = self._with_registers(self.tokens(clip))
        pos = self.positions(*clip.shape[1:4], clip.device)
        for block in self.blocks:
            x = block(x, pos)
        return x

    @torch.no_grad()
    def stream(self, clip):
        """The same tokens, frame by frame: every frame's tokens attend over the caches of the frames before."""
        if any(b.right != 0 for b in self.blocks):
            raise ValueError("streaming needs right = 0: a token may not see later ones")
        B, N, H, W = clip.shape[:4]
        n = H // self.patch * (W // self.patch)
        capacity = len(self.registers) + N * n
        D = self.C // self.blocks[0].heads * self.T
        caches = [tuple(torch.empty(B, capacity, b.heads, D, dtype=clip.dtype, device=clip.device) for _ in range(2))
                  for b in self.blocks]
        out, filled = [], 0
        for t in range(N):
            x = self.tokens(clip[:, t:t + 1])
            if t == 0:
                x = self._with_registers(x)
            pos = self.positions(1, H, W, clip.device, first=t)
            spans = torch.full((2, B), filled, dtype=torch.int32, device=clip.device)
            spans[0] += x.shape[1]
            for block, cache in zip(self.blocks, caches):
                x = block.extend(x, pos, cache, filled, spans[0], spans[1])
            filled += x.shape[1]
            out.append(x)
        return torch.cat(out, 1)


def main(steps: int = 20, device: str = "cuda") -> None:
    """Trains a small encoder to tell the direction in which a pattern drifts, then streams a clip."""
    torch.manual_seed(0)
    T, frames, size = 4, 4, 32
    enc = EQEncoder(T, 4, 32, heads=4, depth=2, sections=(2, 1, 1), left=200, right=0, device=device)
    head = torch.nn.Linear(32, 2, device=device)
    opt = torch.optim.AdamW([*enc.parameters(), *head.parameters()], lr=3e-4)

    def clips(n):
        label = torch.randint(0, 2, (n,), device=device)
        base = torch.randn(n, size, size, 4, T, device=device)
        moved = [torch.stack([b.roll((2 * int(s) - 1) * 3 * t, 0) for b, s in zip(base, label)]) for t in range(frames)]
        return torch.stack(moved, 1), label

    for step in range(steps):
        x, label = clips(8)
        loss = F.cross_entropy(head(enc(x)[:, 1:].mean((1, 3))), label)
        opt.zero_grad(set_to_none=True)
        loss.backward()
        opt.step()
        print("step %d loss %.4f" % (step, loss.item()), flush=True)
    x, _ = clips(2)
    with torch.no_grad():
        whole, streamed = enc(x), enc.stream(x)
    print("streamed against whole clip: largest difference %.2e of %.2f" % (
        (whole - streamed).abs().max().item(), whole.abs().max().item()), flush=True)


if __name__ == "__main__":
    main()
