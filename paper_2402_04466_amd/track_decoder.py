"""A track decoder layer on the library's operators: one token per tool and frame.

    python -m paper_2402_04466_amd.track_decoder [--streams 16] [--frames 600]

Each track's tokens carry a state from frame to frame (``hs_retention``, behind ``hs_norm_rotate``), then look at the
cells of their frame's feature map (``hs_cross_attention``).  The projections are torch products; weights are seeded, not
trained.  A recording goes through in one call, live streams frame by frame from a captured HIP graph, with the same state.
"""
from __future__ import annotations

import argparse
import time

import torch

from . import api
from .harness import heads_of

DTYPES = {torch.float16: api.HS_F16, torch.bfloat16: api.HS_BF16}


class TrackDecoder:
    """One layer: x += W_o retention(norm, rotation of x W_qkv);  x += W_o2 attention(norm of x W_q2, map W_kv).

    x is [streams, frames, tools, channels], maps are [streams, frames, cells, channels]; either one stream and any
    number of frames (a clip) or one frame of any number of streams.  All streams count their frames together, and every
    tool has a token in every frame."""

    def __init__(self, ctx: int, *, streams: int, tools: int = 8, heads: int = 8, head_dim: int = 64,
                 dtype: torch.dtype = torch.float16, seed: int = 0, device: str = "cuda:0"):
        self.ctx, self.streams, self.tools = ctx, streams, tools
        self.heads, self.head_dim, self.dtype, self.device = heads, head_dim, dtype, device
        self.channels = c = heads * head_dim
        g = torch.Generator().manual_seed(seed)

        def weight(rows, cols):
            return (torch.randn(rows, cols, generator=g) * rows ** -0.5).to(device=device, dtype=dtype)
        self.w_qkv, self.w_o = weight(c, 3 * c), weight(c, c)
        self.w_q2, self.w_kv, self.w_o2 = weight(c, c), weight(c, 2 * c), weight(c, c)
        self.w_norm = (1 + 0.1 * torch.randn(3, head_dim, generator=g)).to(device)      # q, k; q of the attention
        self.frequencies = 10000.0 ** (-torch.arange(0, head_dim, 2, dtype=torch.float64, device=device) / head_dim)
        # half-lives from 22 frames on
        self.decay = [1.0 - 2.0 ** (-5.0 - 7.0 * h / max(1, heads - 1)) for h in range(heads)]
        self.state = torch.zeros(streams * tools, heads, head_dim, head_dim, device=device)
        self.frame = torch.zeros(1, dtype=torch.int64, device=device)

    def reset(self) -> None:
        """All tracks begin again: no state, frame 0.  In place, since captured graphs work on this memory."""
        self.state.zero_()
        self.frame.zero_()

    def _norm_rotate(self, stream, q, k, w_q, w_k, positions):
        side = dict(q=heads_of(q), q_out=heads_of(q), q_heads=q.shape[2], d_q_weight=w_q.data_ptr(), k_heads=0)
        if k is not None:
            side.update(k=heads_of(k), k_out=heads_of(k), k_heads=k.shape[2], d_k_weight=w_k.data_ptr())
        if positions is not None:
            side.update(rotary_dim=self.head_dim, d_frequencies=self.frequencies.data_ptr(), d_positions=positions.data_ptr())
        api.hs_norm_rotate(self.ctx, api.make_norm_rotate_desc(
            dtype=DTYPES[self.dtype], batch=q.shape[0], tokens=q.shape[1], head_dim=self.head_dim, **side), stream)

    def _workspace(self, desc, need):
        work = torch.empty(need, dtype=torch.uint8, device=self.device)
        desc.d_workspace, desc.workspace_bytes = (work.data_ptr() if need else None), need
        return work

    def forward(self, x: torch.Tensor, maps: torch.Tensor, mask: torch.Tensor | None = None) -> torch.Tensor:
        """The next frames of every track.  mask: [streams, frames, cells] uint8 or bool, 0 where a cell is hidden."""
        def must_be(name, t, shape, *dtypes):
            if t.shape != shape or t.dtype not in dtypes or t.device != self.state.device:
                raise ValueError(f"{name} must be {list(shape)}, {' or '.join(map(str, dtypes))} on {self.state.device}, "
                                 f"got {list(t.shape)}, {t.dtype} on {t.device}")
        s, t, c = self.streams, self.tools, self.channels
        f = x.shape[1] if x.dim() == 4 else 0
        must_be("x", x, (s, f, t, c), self.dtype)
        if s > 1 and f > 1:
            raise ValueError("need one stream, or one frame of every stream")
        cells = maps.shape[2] if maps.dim() == 4 else 0
        must_be("maps", maps, (s, f, cells, c), self.dtype)
        if mask is not None:
            must_be("mask", mask, (s, f, cells), torch.uint8, torch.bool)
            mask = mask.contiguous()
        h, d, stream = self.heads, self.head_dim, torch.cuda.current_stream().cuda_stream

        positions = self.frame + torch.arange(f, device=self.device)
        qkv = self._tracks((x @ self.w_qkv).view(s, f, t, 3, h, d))
        q, k, v = qkv[:, :, 0], qkv[:, :, 1], qkv[:, :, 2]
        self._norm_rotate(stream, q, k, self.w_norm[0], self.w_norm[1], positions)
        mixed = torch.empty(s, f, t, h, d, dtype=self.dtype, device=self.device)
        work = self._mix(stream, x, qkv, self._tracks(mixed))
        x = x + mixed.flatten(-2) @ self.w_o

        q = (x @ self.w_q2).view(s * f, t, h, d)
        self._norm_rotate(stream, q, None, self.w_norm[2], None, None)
        kv = (maps @ self.w_kv).view(s * f, cells, 2, h, d)
        looked = torch.empty(s * f, t, h, d, dtype=self.dtype, device=self.device)
        work2 = self._look(stream, q, kv, looked, mask)
        self.frame += f
        del work, work2                             # (torch reuses them on this stream only)
        return self._end(stream, x + looked.view(s, f, t, c) @ self.w_o2)

    def _tracks(self, y):
        """[streams, frames, tools, ...] as [streams * tools, frames, ...], without a copy."""
        return y.flatten(0, 1).transpose(0, 1) if self.streams == 1 else y.transpose(1, 2).flatten(0, 1)

    def _mix(self, stream, x, qkv, out):
        """The tracks' tokens (x: what they were projected from), behind norm and rotation, into `out`."""
        h, d = self.heads, self.head_dim
        q, k, v = qkv[:, :, 0], qkv[:, :, 1], qkv[:, :, 2]
        desc = api.make_retention_desc(
            dtype=DTYPES[self.dtype], batch=q.shape[0], tokens=q.shape[1], q_heads=h, kv_heads=h, key_dim=d, value_dim=d,
            scale=d ** -0.5, decay=self.decay, q=heads_of(q), k=heads_of(k), v=heads_of(v), out=heads_of(out),
            d_state_in=self.state.data_ptr(), d_state_out=self.state.data_ptr())
        work = self._workspace(desc, api.hs_query_retention_workspace(desc))
        api.hs_retention(self.ctx, desc, stream)
        return work

    def _look(self, stream, q, kv, out, mask):
        """Queries on keys and values of the cells, into `out`."""
        n, t, h, d = q.shape
        cells = kv.shape[1]
        desc = api.make_cross_attention_desc(
            dtype=DTYPES[self.dtype], batch=n, q_tokens=t, k_tokens=cells, q_heads=h, kv_heads=h, head_dim=d,
            scale=d ** -0.5, q=heads_of(q), k=heads_of(kv[:, :, 0]), v=heads_of(kv[:, :, 1]), out=heads_of(out),
            d_mask=0 if mask is None else mask.data_ptr(), mask_batch_stride=cells)
        work = self._workspace(desc, api.hs_query_cross_attention_workspace(desc))
        api.hs_cross_attention(self.ctx, desc, stream)
        return work

    def _end(self, stream, x):
        return x

    def live(self, cells: int) -> "LiveTracks":
        return LiveTracks(self, cells)


class LiveTracks:
    """One frame of every stream at a time, replayed from a HIP graph: fill ``x`` and ``maps``, ``step()``, read ``out``."""

    def __init__(self, decoder: TrackDecoder, cells: int):
        dec, kw = decoder, dict(dtype=decoder.dtype, device=decoder.device)
        self.x = torch.zeros(dec.streams, 1, dec.tools, dec.channels, **kw)
        self.maps = torch.zeros(dec.streams, 1, cells, dec.channels, **kw)
        state, frame = dec.state.clone(), dec.frame.clone()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            dec.forward(self.x, self.maps)          # libraries set themselves up outside of the capture
        torch.cuda.current_stream().wait_stream(side)
        self.graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(self.graph):
            self.out = dec.forward(self.x, self.maps)
        dec.state.copy_(state)
        dec.frame.copy_(frame)
        self._decoder = decoder                     # the graph works on its state

    def step(self) -> torch.Tensor:
        self.graph.replay()
        return self.out


def run_example(decoder, doc: str) -> None:
    ap = argparse.ArgumentParser(description=doc.splitlines()[0])
    ap.add_argument("--streams", type=int, default=16)
    ap.add_argument("--frames", type=int, default=600)
    ap.add_argument("--cells", type=int, default=405)
    args = ap.parse_args()
    ctx = api.hs_init(0)

    def timed(what, per, call):
        call()
        torch.cuda.synchronize()
        t0 = time.perf_counter()
        call()
        torch.cuda.synchronize()
        print(f"{what}: {(time.perf_counter() - t0) / per * 1e6:.1f} us per frame")
    clip = decoder(ctx, streams=1)
    x = torch.randn(1, args.frames, clip.tools, clip.channels, dtype=clip.dtype, device=clip.device)
    maps = torch.randn(1, args.frames, args.cells, clip.channels, dtype=clip.dtype, device=clip.device)
    timed(f"a clip of {args.frames} frames in one call", args.frames, lambda: clip.forward(x, maps))
    live = decoder(ctx, streams=args.streams).live(args.cells)
    live.x.normal_()
    live.maps.normal_()
    timed(f"{args.streams} live streams", args.frames, lambda: [live.step() for _ in range(args.frames)])
    torch.cuda.synchronize()
    api.hs_shutdown(ctx)


def main() -> None:
    run_example(TrackDecoder, __doc__)


if __name__ == "__main__":
    main()
