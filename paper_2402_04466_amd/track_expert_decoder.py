"""A track decoder layer whose tracks forget by key, compare two looks at the map and pass through experts.

    python -m paper_2402_04466_amd.track_expert_decoder [--streams 16] [--frames 600]

The counterpart of ``track_decoder`` on ``hs_delta_rule`` (in place of ``hs_retention``), ``hs_differential_attention`` (in
place of ``hs_cross_attention``) and ``hs_expert_layer``.  The projections are torch products; weights are seeded, not
trained.  A recording goes through in one call, live streams frame by frame from a captured HIP graph, with the same state.
"""
from __future__ import annotations

import torch

from . import api
from .harness import gates_of, heads_of
from .track_decoder import DTYPES, TrackDecoder, run_example


class ExpertTrackDecoder(TrackDecoder):
    """One layer:  x += W_o rule(norm and rotation of x W_qkv, gates of x W_g);
    x += W_o2 difference(norm of x W_q2, map W_kv2);  x += experts(norm of x).

    Shapes, streams and frames as TrackDecoder.  Keys have length 1; head h of the comparison is heads 2h and 2h + 1 of
    x W_q2 and of the map's keys, with values twice as wide."""

    def __init__(self, ctx: int, *, streams: int, tools: int = 8, heads: int = 8, head_dim: int = 64, experts: int = 16, top: int = 2,
                 hidden: int = 1024, dtype: torch.dtype = torch.float16, seed: int = 0, device: str = "cuda:0"):
        if heads % 2:
            raise ValueError("heads must be even: two of them are compared")
        for name, value, step, most in (("head_dim", head_dim, 16, 64), ("heads * head_dim", heads * head_dim, 16, api.HS_MAX_CHANNELS),
                                        ("hidden", hidden, 8, api.HS_MAX_CHANNELS), ("experts", experts, 1, api.HS_MAX_EXPERTS),
                                        ("top", top, 1, min(api.HS_MAX_TOP, experts))):
            if not step <= value <= most or value % step:          # (values are twice as wide as head_dim, and 128 the most)
                raise ValueError(f"{name} must be a multiple of {step} in {step}..{most}, got {value}")
        super().__init__(ctx, streams=streams, tools=tools, heads=heads, head_dim=head_dim, dtype=dtype, seed=seed, device=device)
        c, self.top, self.hidden = self.channels, top, hidden
        g = torch.Generator().manual_seed(seed + 1)

        def weight(*shape):
            return (torch.randn(*shape, generator=g) * shape[-1] ** -0.5).to(device=device, dtype=dtype)
        self.w_gates = weight(2 * heads, c).T.contiguous()
        self.w_norm[1] = head_dim ** -0.5                # keys of length 1
        self.lam = torch.rand(heads // 2, generator=g).to(device) * 0.6 + 0.2
        self.w_looked = 0.2 * (1 + 0.1 * torch.randn(2 * head_dim, generator=g)).to(device)
        self.router, self.w_in, self.w_out = weight(experts, c), weight(experts, 2 * hidden, c), weight(experts, c, hidden)

    def _mix(self, stream, x, qkv, out):
        """The tracks' tokens, behind norm and rotation, into `out`."""
        s, f, t, h, d = self.streams, x.shape[1], self.tools, self.heads, self.head_dim
        gates = (x @ self.w_gates).float()
        log_decay = -torch.nn.functional.softplus(gates[..., :h]) * 2.0 ** -5
        both = self._tracks(torch.cat((log_decay, torch.sigmoid(gates[..., h:])), -1))
        desc = api.make_delta_rule_desc(
            dtype=DTYPES[self.dtype], batch=s * t, tokens=f, heads=h, qk_heads=h, key_dim=d, value_dim=d, scale=d ** -0.5,
            q=heads_of(qkv[:, :, 0]), k=heads_of(qkv[:, :, 1]), v=heads_of(qkv[:, :, 2]), out=heads_of(out),
            log_decay=gates_of(both[..., :h]), beta=gates_of(both[..., h:]), d_state_in=self.state.data_ptr(), d_state_out=self.state.data_ptr())
        work = self._workspace(desc, api.hs_query_delta_rule_workspace(desc))
        api.hs_delta_rule(self.ctx, desc, stream)
        return work, both

    def _look(self, stream, q, kv, out, mask):
        """Queries on keys and values of the cells, into `out`."""
        n, t, h, d = q.shape
        cells = kv.shape[1]
        out = out.view(n, t, h // 2, 2 * d)
        values = kv[:, :, 1].flatten(-2).view(n, cells, h // 2, 2 * d)
        desc = api.make_differential_attention_desc(
            dtype=DTYPES[self.dtype], batch=n, q_tokens=t, k_tokens=cells, q_heads=h // 2, kv_heads=h // 2, head_dim=d, value_dim=2 * d,
            scale=d ** -0.5, q=heads_of(q), k=heads_of(kv[:, :, 0]), v=heads_of(values), out=heads_of(out), d_lambda=self.lam.data_ptr(),
            norm=True, eps=1e-5, d_norm_weight=self.w_looked.data_ptr(), d_mask=0 if mask is None else mask.data_ptr(), mask_batch_stride=cells)
        work = self._workspace(desc, api.hs_query_differential_attention_workspace(desc))
        api.hs_differential_attention(self.ctx, desc, stream)
        return work

    def _end(self, stream, x):
        """Each token through the experts that it picks, 1024 tokens at a time."""
        c = self.channels
        y = x.reshape(-1, 1, self.heads, self.head_dim).clone()
        self._norm_rotate(stream, y, None, self.w_norm[2], None, None)
        y, out = y.view(-1, c), torch.empty(x.numel() // c, c, dtype=self.dtype, device=self.device)
        keep = []
        for at in range(0, len(y), api.HS_MAX_EXPERT_TOKENS):
            part = y[at:at + api.HS_MAX_EXPERT_TOKENS]
            desc = api.make_expert_layer_desc(
                dtype=DTYPES[self.dtype], tokens=len(part), channels=c, hidden=self.hidden, experts=self.router.shape[0], top=self.top,
                d_x=part.data_ptr(), x_stride=c, d_out=out[at:].data_ptr(), out_stride=c, d_router=self.router.data_ptr(),
                d_w_in=self.w_in.data_ptr(), d_w_out=self.w_out.data_ptr())
            keep.append(self._workspace(desc, api.hs_query_expert_layer_workspace(desc)))
            api.hs_expert_layer(self.ctx, desc, stream)
        return x + out.view(x.shape)


if __name__ == "__main__":
    run_example(ExpertTrackDecoder, __doc__)
