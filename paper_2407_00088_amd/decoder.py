"""The attention half of a decoder layer with low-bit projections: q, k, v and o through runner.LinearLUT, positions by rotation
(plain torch), attention over prompts, a cache that keeps the heaviest keys, and decode steps of a batch that may share a prefix.

  python -m paper_2407_00088_amd.decoder      # prompts, then a few decode steps, of a small random layer
"""
from __future__ import annotations

import torch

from . import binding as B
from .attention import KVCache, attn_prompt, attn_weights


def rotated(x, positions, base: float = 10000.0):
    """x [T, H, D] turned by its tokens' positions [T]: elements i and i + D / 2 by positions * base^(-2 i / D)."""
    half = x.shape[-1] // 2
    angle = positions[:, None].float() * base ** (-torch.arange(half, device=x.device) / half)
    c, s = torch.cos(angle)[:, None], torch.sin(angle)[:, None]
    a, b = x[..., :half].float(), x[..., half:].float()
    return torch.cat([a * c - b * s, a * s + b * c], dim=-1).to(x.dtype)


class DecoderAttention:
    """q, k, v, o: LinearLUT holders of [Hq D, M], [Hkv D, M], [Hkv D, M] and [M, Hq D] weights, with room (max_N) for the tokens of a
    call.  `capacity` slots for each sequence and key head, of which the `recent` last tokens' are kept in any case."""

    def __init__(self, q, k, v, o, Hq: int, Hkv: int, batch: int, capacity: int, recent: int):
        self.q, self.k, self.v, self.o, self.Hq, self.Hkv = q, k, v, o, Hq, Hkv
        self.D = q.M // Hq
        self.cache = KVCache(batch, Hkv, self.D, capacity, recent=recent, Hq=Hq)
        self.prefix = None            # (keys, values) that all sequences share
        self.prefix_length = 0
        self.position = torch.zeros(batch, dtype=torch.int64, device=self.cache.k.device)

    def project(self, x, positions):
        """Hidden states [T, M] (fp16) as rotated queries and keys and plain values, [T, H, D]."""
        rows = [lin.forward_one_call(x, out_t=B.TMAC_OUT_F16).view(x.shape[0], -1, self.D) for lin in (self.q, self.k, self.v)]
        return rotated(rows[0], positions), rotated(rows[1], positions), rows[2]

    def share(self, x) -> None:
        """A prefix [P, M] for all sequences, which comes before their own tokens: those, if there are any, end here."""
        _, k, v = self.project(x, torch.arange(x.shape[0], device=x.device))
        self.prefix, self.prefix_length = (k, v), x.shape[0]
        self.cache.lens.zero_(), self.cache.seen.zero_()
        self.position.fill_(self.prefix_length)

    def prompt(self, x, cu):
        """The sequences' own prompts, packed: x [T, M], cu int32 [batch + 1] on the GPU and the tokens' positions by it.  Returns [T, M]; the cache
        keeps what it has room for, and nothing of earlier prompts and steps."""
        n = (cu[1:] - cu[:-1]).long()
        at = torch.arange(x.shape[0], device=x.device)
        positions = at - torch.repeat_interleave(cu[:-1].long(), n) + self.prefix_length
        q, k, v = self.project(x, positions)
        if self.prefix is None:
            keys, values, cu_k = k, v, cu
        else:
            # every sequence's keys after the shared ones
            P, T = self.prefix_length, x.shape[0]
            cu_k = cu + P * torch.arange(cu.numel(), dtype=torch.int32, device=x.device)
            rows = at + P * (torch.repeat_interleave(torch.arange(n.numel(), device=x.device), n) + 1)
            shared = (cu_k[:-1, None].long() + torch.arange(P, device=x.device)).reshape(-1)
            keys, values = (t.new_empty((T + P * n.numel(), *t.shape[1:])) for t in (k, v))
            for t, own, first in ((keys, k, self.prefix[0]), (values, v, self.prefix[1])):
                t[rows] = own
                t[shared] = first.repeat(n.numel(), 1, 1)
        out, lse = attn_prompt(q, keys, values, cu, cu_k)
        weight = attn_weights(q, keys, lse, cu, cu_k)
        if self.prefix is not None:
            weight = weight[:, rows]
        self.cache.fill(k, v, weight, cu)
        torch.add(n, self.prefix_length, out=self.position)
        return self.o.forward_one_call(out.view(x.shape[0], -1), out_t=B.TMAC_OUT_F16)

    def step(self, x):
        """One token of every sequence: x [batch, M].  Returns [batch, M]."""
        q, k, v = self.project(x, self.position)
        self.cache.append(k, v)
        out, _ = self.cache.attend(q, *(self.prefix or (None, None)))
        self.position += 1
        return self.o.forward_one_call(out.view(x.shape[0], -1), out_t=B.TMAC_OUT_F16)


def random_layer(M: int, Hq: int, Hkv: int, D: int, batch: int, capacity: int, recent: int, max_N: int, bits: int = 4, group: int = 64,
                 seed: int = 0) -> DecoderAttention:
    """A layer of random weights, scaled so that unit inputs give projections of about one."""
    import numpy as np

    from .runner import LinearLUT
    rng = np.random.default_rng(seed)

    def linear(rows: int, cols: int):
        q = rng.integers(0, 1 << bits, size=(rows, cols), dtype=np.uint8)
        s = np.full((rows, cols // group), 1.0 / (cols ** 0.5 * ((1 << bits) / 12 ** 0.5)), dtype=np.float16)
        return LinearLUT(rows, cols, bits, group, q, s, max_N=max_N, layout=B.TMAC_LAYOUT_R64K32)

    return DecoderAttention(linear(Hq * D, M), linear(Hkv * D, M), linear(Hkv * D, M), linear(M, Hq * D), Hq, Hkv, batch, capacity, recent)


def main(steps: int = 8) -> None:
    torch.manual_seed(0)
    batch, M = 3, 512
    layer = random_layer(M, Hq=8, Hkv=2, D=64, batch=batch, capacity=48, recent=16, max_N=512)
    x = lambda n: torch.randn((n, M), device="cuda").half()  # noqa: E731
    layer.share(x(100))
    lengths = [70, 9, 33]
    cu = torch.tensor([0, 70, 79, 112], dtype=torch.int32, device="cuda")
    y = layer.prompt(x(sum(lengths)), cu)
    print(f"prompts of {lengths} tokens after a shared prefix of 100: {tuple(y.shape)}, rms {float(y.float().square().mean().sqrt()):.3f}, "
          f"slots in use {layer.cache.lens[:, 0].tolist()}")
    for t in range(steps):
        y = layer.step(x(batch))
        print(f"step {t}: rms {float(y.float().square().mean().sqrt()):.3f}, slots in use {layer.cache.lens[:, 0].tolist()}, "
              f"tokens seen {layer.cache.seen[:, 0].tolist()}")


if __name__ == "__main__":
    main()
