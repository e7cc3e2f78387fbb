"""An equivariant encoder of images and video on the library's layers.

    stem     rotation-equivariant 3 x 3 convolutions (``gconv``) with group norm and activation between (``norm``)
    tokens   the features of p x p pixels averaged, a frame in raster order, frames after one another, after a few
             register tokens
    blocks   ``EQViTBlock`` with rotary positions (time, height, width) and windowed attention (``attention``), or
             recurrent ones: a short causal convolution and a selective scan (``scan``) between fused norms

Every part commutes with the group action on the T axis.  Without a limit to the right every token sees as far ahead as
back; with ``right = 0`` a video can also be encoded frame by frame over caches (``EQEncoder.stream``), whose tokens are
those of the whole clip; recurrent blocks see earlier tokens only and stream with a state of fixed size.

``python -m paper_2607_21271_amd.encoder [attention|scan]`` trains a small encoder on synthetic clips for a few steps and
streams one.
"""
from __future__ import annotations

import sys

import torch
import torch.nn.functional as F

from . import attention, rotary, scan
from .blocks import EQViTBlock, GroupLayerNorm
from .gconv import GroupConv2d
from .norm import GroupNormAct, residual_norm
from .ops import EQLinear


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


class EQScanBlock(torch.nn.Module):
    """A recurrent block on tokens x [B, L, C, T], each of which sees itself and the tokens before:

        x = x + scale1 * gate * mix(norm1(x)),  x = x + scale2 * gate * fc2(gelu(fc1(norm2(x))))

    ``mix`` projects to 2 x ``expand`` x C channels, half of them the gate, runs a causal convolution of ``width`` tokens and a
    selective scan of ``states`` states a channel, and projects back.  The steps come from an equivariant layer of rank
    ``rank``, Bt and Ct from the mean over the group, so the block commutes with the group action.  ``layer_scale``: first value
    of scale1 and scale2 (None: without); ``post_norm``: both branches are normalised before they are added."""

    def __init__(self, T: int, C: int, expand: int = 2, states: int = 16, width: int = 4, groups: int = 1,
                 rank: int | None = None, mlp_ratio: int = 4, kind: str = "layer", layer_scale: float | None = None,
                 post_norm: bool = False, device=None, dtype=None):
        super().__init__()
        kw = {"device": device, "dtype": dtype}
        wide = {"device": device, "dtype": torch.float32}
        E = expand * C
        rank = max(1, -(-C // 16)) if rank is None else rank
        self.T, self.C, self.E, self.states, self.width, self.groups, self.kind = T, C, E, states, width, groups, kind
        self.norm1, self.norm2 = GroupLayerNorm(C, **kw), GroupLayerNorm(C, **kw)
        self.post1, self.post2 = (GroupLayerNorm(C, **kw) if post_norm else None for _ in range(2))
        for name in ("scale1", "scale2"):
            self.register_parameter(name, None if layer_scale is None else
                                    torch.nn.Parameter(torch.full((C,), float(layer_scale), **kw)))
        self.in_proj = EQLinear(T, C, 2 * E, **kw)
        self.conv_weight = torch.nn.Parameter(torch.rand(E, width, **kw).mul_(2).sub_(1).mul_(width ** -0.5))
        self.conv_bias = torch.nn.Parameter(torch.zeros(E, **kw))
        self.bc = torch.nn.Linear(E, 2 * groups * states, bias=False, **kw)
        self.delta_down, self.delta_up = EQLinear(T, E, rank, bias=False, **kw), EQLinear(T, rank, E, bias=False, **kw)
        # decays of 1, 2, .. states a unit of step, steps between 0.001 and 0.1 at first; held in float32 whatever the
        # block's type: what a state keeps over thousands of tokens goes by their last digits
        self.A_log = torch.nn.Parameter(torch.arange(1, states + 1, **wide).log().repeat(E, 1))
        self.D = torch.nn.Parameter(torch.ones(E, **wide))
        step = torch.exp(torch.rand(E, **wide) * 4.605 - 6.908)
        self.delta_bias = torch.nn.Parameter(torch.log(torch.expm1(step)))
        self.out_proj = EQLinear(T, E, C, **kw)
        self.fc1, self.fc2 = EQLinear(T, C, mlp_ratio * C, **kw), EQLinear(T, mlp_ratio * C, C, **kw)

    def _apply(self, fn, recurse=True):
        wide = [t for p in (self.A_log, self.D, self.delta_bias) for t in (p, p.grad) if t is not None]

        def keep(t):
            out = fn(t)
            return t.to(out.device) if out.dtype != t.dtype and any(t is w for w in wide) else out

        return super()._apply(keep, recurse)

    def new_cache(self, B: int):
        """What ``extend`` carries from call to call: the last tokens of the convolution and the states, zeros at first."""
        w = self.conv_weight
        return (w.new_zeros((B, self.width - 1, self.E, self.T)),
                self.A_log.new_zeros((B, self.E, self.T, self.states)))

    def mix(self, h, lengths=None, cache=None):
        B, L = h.shape[:2]
        x, z = self.in_proj(h).chunk(2, 2)
        last, state = cache or (None, None)
        x = scan.causal_conv(x, self.conv_weight, self.conv_bias, "silu", lengths, last, state_out=last)
        x = x if cache is None else x[0]
        with torch.autocast(x.device.type, enabled=False):  # (a dense layer: it would give Bt and Ct a type that x has not)
            bc = self.bc(x.mean(3)).view(B, L, 2 * self.groups, self.states)
        y = scan.selective_scan(x, self.delta_up(self.delta_down(x)), -torch.exp(self.A_log), bc[:, :, :self.groups],
                                bc[:, :, self.groups:], self.D, z, self.delta_bias, lengths=lengths, state=state,
                                state_out=state)
        return self.out_proj(y if cache is None else y[0])

    def forward(self, x, lengths=None, gate=None, cache=None):
        """``gate`` [B, C]: of both branches, 0 where a sequence drops them."""
        post = lambda n: {} if n is None else {"post_weight": n.weight, "post_bias": n.bias}
        kw = {"kind": self.kind, "eps": self.norm1.eps}
        _, h = residual_norm(x, weight=self.norm1.weight, bias=self.norm1.bias, **kw)
        x, h = residual_norm(x, self.mix(h, lengths, cache), self.norm2.weight, self.norm2.bias, scale=self.scale1, gate=gate,
                             **post(self.post1), **kw)
        return residual_norm(x, self.fc2(F.gelu(self.fc1(h))), scale=self.scale2, gate=gate, **post(self.post2), **kw)[0]

    @torch.no_grad()
    def extend(self, x, cache):
        """``forward`` of the next tokens x [B, n, C, T], which carries on from the cache (``new_cache``) and updates it."""
        return self.forward(x, cache=cache)


class EQEncoder(torch.nn.Module):
    """Clips [B, frames, H, W, Cin, T] -> tokens [B, registers + frames * H/p * W/p, C, T]."""

    def __init__(self, T: int, Cin: int, C: int, heads: int, depth: int, sections, patch: int = 4, registers: int = 4,
                 left: int = -1, right: int = -1, stem: int = 2, groups: int = 4, activation: str = "silu", device=None,
                 dtype=None, mixer: str = "attention"):
        super().__init__()
        if mixer not in ("attention", "scan"):
            raise ValueError("mixer must be attention or scan, got %r" % (mixer,))
        kw = {"device": device, "dtype": dtype}
        self.T, self.C, self.patch, self.mixer = T, C, patch, mixer
        self.stem = torch.nn.ModuleList(torch.nn.ModuleList((GroupConv2d(T, Cin if i == 0 else C, C, **kw),
                                                             GroupNormAct(C, groups, activation, **kw)))
                                        for i in range(stem))
        # one value per channel, the same for every group element
        self.registers = torch.nn.Parameter(torch.randn(registers, C, 1, **kw) * 0.02)
        self.blocks = torch.nn.ModuleList(EQWindowBlock(T, C, heads, sections, left, right, registers, **kw)
                                          if mixer == "attention" else EQScanBlock(T, C, **kw) for _ in range(depth))

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
        if self.mixer == "scan":
            for block in self.blocks:
                x = block(x)
            return x
        pos = self.positions(*clip.shape[1:4], clip.device)
        for block in self.blocks:
            x = block(x, pos)
        return x

    @torch.no_grad()
    def stream(self, clip):
        """The same tokens, frame by frame: every frame's tokens attend over the caches of the frames before, or carry on
        from the states behind them."""
        if self.mixer == "scan":
            caches = [b.new_cache(clip.shape[0]) for b in self.blocks]
            out = []
            for t in range(clip.shape[1]):
                x = self.tokens(clip[:, t:t + 1])
                if t == 0:
                    x = self._with_registers(x)
                for block, cache in zip(self.blocks, caches):
                    x = block.extend(x, cache)
                out.append(x)
            return torch.cat(out, 1)
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


def main(steps: int = 20, device: str = "cuda", mixer: str = "attention") -> None:
    """Trains a small encoder to tell the direction in which a pattern drifts, then streams a clip."""
    torch.manual_seed(0)
    T, frames, size = 4, 4, 32
    enc = EQEncoder(T, 4, 32, heads=4, depth=2, sections=(2, 1, 1), left=200, right=0, device=device, mixer=mixer)
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
    main(mixer=sys.argv[1] if len(sys.argv) > 1 else "attention")
