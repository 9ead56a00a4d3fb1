"""What the GPU tests of the track decoder's further operators share."""
import math

import torch

DEV = "cuda:0"
TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}
F32 = 2.0 ** -24                     # half a step of fp32, relative


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def normal(g, *shape, dtype=torch.float32):
    return torch.randn(*shape, generator=g, device=DEV).to(dtype)


def stream():
    return torch.cuda.current_stream().cuda_stream


def ptr(t):
    return 0 if t is None else t.data_ptr()


def type_of(hs, t):
    return hs.HS_F16 if t.dtype == torch.float16 else hs.HS_BF16


def close(got, want, bound, what):
    got = got.double()
    assert torch.isfinite(got).all(), what
    off = (got - want).abs() - bound
    worst = off.max().item() if off.numel() else 0.0
    assert worst <= 0, f"{what}: {worst:.3e} beyond the bound, at {torch.nonzero(off == off.max())[0].tolist()}"


def smallest(dtype):
    """Half of the smallest step that the type has: what lies below its normal numbers is rounded to that at best."""
    return math.ldexp(1.0, -25) if dtype == torch.float16 else 0.0


def give_workspace(desc, need):
    """A workspace full of ones, as nothing may be expected of it."""
    work = torch.empty(need, dtype=torch.uint8, device=DEV).fill_(0xff)
    desc.d_workspace, desc.workspace_bytes = (work.data_ptr() if need else None), need
    return work


def delta_call(hs, ctx, q, k, v, out, log_decay, beta, state_in, state_out, scale, lengths=None, at=None):
    from paper_2402_04466_amd.harness import gates_of, heads_of
    d = hs.make_delta_rule_desc(
        dtype=type_of(hs, q), batch=q.shape[0], tokens=q.shape[1], heads=v.shape[2], qk_heads=q.shape[2],
        key_dim=q.shape[3], value_dim=v.shape[3], scale=scale, q=heads_of(q), k=heads_of(k), v=heads_of(v),
        out=heads_of(out), log_decay=None if log_decay is None else gates_of(log_decay),
        beta=None if beta is None else gates_of(beta), d_lengths=ptr(lengths), d_state_in=ptr(state_in),
        d_state_out=ptr(state_out))
    work = give_workspace(d, hs.hs_query_delta_rule_workspace(d))
    hs.hs_delta_rule(ctx, d, stream() if at is None else at)
    return work


def differential_call(hs, ctx, q, k, v, out, lam, scale, *, norm=True, eps=1e-5, weight=None, lengths=None, mask=None, at=None):
    from paper_2402_04466_amd.harness import heads_of
    d = hs.make_differential_attention_desc(
        dtype=type_of(hs, q), batch=q.shape[0], q_tokens=q.shape[1], k_tokens=k.shape[1], q_heads=q.shape[2] // 2,
        kv_heads=v.shape[2], head_dim=q.shape[3], value_dim=v.shape[3], scale=scale, q=heads_of(q), k=heads_of(k),
        v=heads_of(v), out=heads_of(out), d_lambda=ptr(lam), norm=norm, eps=eps, d_norm_weight=ptr(weight),
        d_lengths=ptr(lengths), d_mask=ptr(mask), mask_batch_stride=0 if mask is None else mask.stride(0))
    work = give_workspace(d, hs.hs_query_differential_attention_workspace(d))
    hs.hs_differential_attention(ctx, d, stream() if at is None else at)
    return work


def expert_call(hs, ctx, x, router, w_in, w_out, out, top, *, renormalise=True, mask=None, chosen=None, weights=None, at=None):
    d = hs.make_expert_layer_desc(
        dtype=type_of(hs, x), tokens=x.shape[0], channels=x.shape[1], hidden=w_out.shape[2], experts=router.shape[0],
        top=top, renormalise=renormalise, d_x=ptr(x), x_stride=x.stride(0), d_out=ptr(out), out_stride=out.stride(0),
        d_router=ptr(router), d_w_in=ptr(w_in), d_w_out=ptr(w_out), d_mask=ptr(mask), d_chosen=ptr(chosen),
        d_weights=ptr(weights))
    work = give_workspace(d, hs.hs_query_expert_layer_workspace(d))
    hs.hs_expert_layer(ctx, d, stream() if at is None else at)
    return work
