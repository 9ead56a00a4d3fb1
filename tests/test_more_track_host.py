"""CPU-only tests of the delta rule, the differential attention and the expert layer at the boundary: the binding's
descriptions have the header's sizes, and everything a call must refuse is refused before any GPU work (no context
exists here, and a description that passes every check ends at the missing context)."""
import ctypes
import os
import subprocess

import pytest

import paper_2402_04466_amd as hs
from paper_2402_04466_amd import api

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 1 << 20     # a well aligned address that nothing reads


def heads(d=P, batch=8 * 64 * 16, token=8 * 64, head=64):
    return hs.hs_heads(d, batch, token, head)


def gates(d=P, batch=8 * 16, token=8, head=1):
    return hs.hs_gates(d, batch, token, head)


def delta(**change):
    kw = dict(dtype=hs.HS_F16, batch=2, tokens=16, heads=8, qk_heads=8, key_dim=64, value_dim=64, scale=0.125, q=heads(),
              k=heads(2 * P), v=heads(3 * P), out=heads(4 * P), log_decay=gates(), beta=gates(2 * P), d_state_in=P, d_state_out=P,
              d_workspace=P, workspace_bytes=1 << 40)
    kw.update(change)
    return hs.make_delta_rule_desc(**kw)


def differential(**change):
    kw = dict(dtype=hs.HS_F16, batch=2, q_tokens=16, k_tokens=16, q_heads=8, kv_heads=8, head_dim=32, value_dim=64, scale=0.125,
              q=heads(), k=heads(2 * P), v=heads(3 * P), out=heads(4 * P), d_lambda=P, d_norm_weight=P, d_workspace=P,
              workspace_bytes=1 << 40)
    kw.update(change)
    return hs.make_differential_attention_desc(**kw)


def experts(**change):
    kw = dict(dtype=hs.HS_F16, tokens=16, channels=64, hidden=128, experts=8, top=2, d_x=P, x_stride=64, d_out=2 * P, out_stride=64,
              d_router=3 * P, d_w_in=4 * P, d_w_out=5 * P, d_workspace=P, workspace_bytes=1 << 40)
    kw.update(change)
    return hs.make_expert_layer_desc(**kw)


CALLS = {"hs_delta_rule": (hs.hs_delta_rule, delta, hs.hs_query_delta_rule_workspace),
         "hs_differential_attention": (hs.hs_differential_attention, differential, hs.hs_query_differential_attention_workspace),
         "hs_expert_layer": (hs.hs_expert_layer, experts, hs.hs_query_expert_layer_workspace)}
ATTENTION = ["hs_delta_rule", "hs_differential_attention"]


def refused(name, desc, words, status=hs.HS_E_INVAL):
    with pytest.raises(hs.HsError) as e:
        CALLS[name][0](0, desc)
    assert e.value.status == status and name in str(e.value) and words in str(e.value), str(e.value)


def test_binding_sizes_of_the_descriptions_match_the_header(tmp_path):
    names = ["hs_gates", "hs_delta_rule_desc", "hs_differential_attention_desc", "hs_expert_layer_desc"]
    limits = ["HS_MAX_EXPERT_TOKENS", "HS_MAX_CHANNELS", "HS_MAX_EXPERTS", "HS_MAX_TOP"]
    last = {"hs_delta_rule_desc": "workspace_bytes", "hs_differential_attention_desc": "mask_batch_stride", "hs_expert_layer_desc": "d_mask"}
    src = tmp_path / "sz.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "hs.h"\nint main(void){'
                   + "".join(f'printf("%zu\\n", sizeof({n}));' for n in names)
                   + "".join(f'printf("%zu\\n", offsetof({n}, {f}));' for n, f in last.items())
                   + "".join(f'printf("%d\\n", {n});' for n in limits) + 'return 0;}\n')
    exe = tmp_path / "sz"
    subprocess.check_call(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)])
    out = [int(v) for v in subprocess.check_output([str(exe)]).split()]
    assert out == ([ctypes.sizeof(getattr(hs, n)) for n in names] + [getattr(getattr(hs, n), f).offset for n, f in last.items()]
                   + [getattr(hs, n) for n in limits])


@pytest.mark.parametrize("name", sorted(CALLS))
def test_a_sound_description_is_only_short_of_a_context(name):
    refused(name, CALLS[name][1](), "NULL context")
    assert getattr(api.load(), name)(None, None, None) == hs.HS_E_INVAL
    assert "NULL description" in hs.hs_last_error()


@pytest.mark.parametrize("name", sorted(CALLS))
@pytest.mark.parametrize("dtype", [0, 3, -1])
def test_types(name, dtype):
    refused(name, CALLS[name][1](dtype=dtype), "dtype")


@pytest.mark.parametrize("name", ATTENTION)
@pytest.mark.parametrize("change, words", [
    (dict(batch=-1), "negative"), (dict(q=heads(0)), "q must be"), (dict(q=heads(P + 8)), "q must be"),
    (dict(q=heads(token=8 * 64 + 4)), "strides of q"), (dict(k=heads(0)), "k must be"), (dict(k=heads(head=68)), "strides of k"),
    (dict(v=heads(0)), "v must be"), (dict(v=heads(batch=4)), "strides of v"), (dict(out=heads(0)), "out must be"),
    (dict(scale=float("nan")), "scale"), (dict(scale=float("-inf")), "scale"), (dict(d_lengths=P + 2), "d_lengths"),
    (dict(value_dim=4), "value_dim"), (dict(value_dim=132), "value_dim"), (dict(value_dim=136), "value_dim")])
def test_refusals_common_to_attention(name, change, words):
    refused(name, CALLS[name][1](**change), words)


@pytest.mark.parametrize("name", ATTENTION)
@pytest.mark.parametrize("strides", [dict(head=32), dict(head=0), dict(token=0), dict(batch=0), dict(batch=8 * 64),
                                     dict(token=-8 * 32), dict(batch=-(1 << 63))])
def test_outputs_whose_rows_overlap_are_refused(name, strides):
    refused(name, CALLS[name][1](out=heads(5 * P, **strides)), "out")


@pytest.mark.parametrize("change, words", [
    (dict(heads=0), "multiple of qk_heads"), (dict(qk_heads=3), "multiple of qk_heads"), (dict(qk_heads=0), "multiple of qk_heads"),
    (dict(heads=8, qk_heads=16), "multiple of qk_heads"), (dict(key_dim=12), "key_dim"), (dict(key_dim=136), "key_dim"),
    (dict(tokens=-1), "negative"), (dict(log_decay=gates(P + 2)), "log_decay"), (dict(beta=gates(P + 1)), "beta"),
    (dict(d_state_out=0), "d_state_out"), (dict(d_state_out=P + 8), "d_state_out"), (dict(d_state_in=P + 4), "d_state_in")])
def test_refusals_of_the_delta_rule(change, words):
    refused("hs_delta_rule", delta(**change), words)


@pytest.mark.parametrize("change, words", [
    (dict(kv_heads=3), "multiple of kv_heads"), (dict(q_heads=0), "multiple of kv_heads"), (dict(head_dim=12), "head_dim"),
    (dict(head_dim=0), "head_dim"), (dict(q_tokens=-1), "negative"), (dict(k_tokens=-1), "negative"), (dict(d_lambda=0), "d_lambda"),
    (dict(d_lambda=P + 2), "d_lambda"), (dict(eps=-1.0), "eps"), (dict(eps=float("nan")), "eps"), (dict(d_norm_weight=P + 1), "d_norm_weight")])
def test_refusals_of_the_differential_attention(change, words):
    refused("hs_differential_attention", differential(**change), words)


@pytest.mark.parametrize("change, words", [
    (dict(tokens=-1), "tokens"), (dict(tokens=1025), "tokens"), (dict(channels=60), "channels"), (dict(channels=0), "channels"),
    (dict(channels=16392), "channels"), (dict(hidden=12), "hidden"), (dict(hidden=16392), "hidden"), (dict(experts=0), "experts"),
    (dict(experts=257), "experts"), (dict(top=0), "top"), (dict(top=9, experts=16), "top"), (dict(top=3, experts=2), "top"),
    (dict(d_x=0), "d_x"), (dict(d_x=P + 8), "d_x"), (dict(x_stride=60), "d_x"), (dict(d_out=0), "d_out"), (dict(out_stride=68), "d_out"),
    (dict(out_stride=56), "overlap"), (dict(out_stride=0), "overlap"), (dict(out_stride=-56), "overlap"), (dict(d_router=0), "d_router"),
    (dict(d_w_in=0), "d_w_in"), (dict(d_w_out=P + 4), "d_w_out"), (dict(d_chosen=P + 2), "d_chosen"), (dict(d_weights=P + 2), "d_weights")])
def test_refusals_of_the_expert_layer(change, words):
    refused("hs_expert_layer", experts(**change), words)


def test_what_is_allowed_is_taken():
    for change in (dict(log_decay=None), dict(beta=None), dict(log_decay=gates(P + 4, 0, -3, 7)), dict(d_state_in=0), dict(qk_heads=2),
                   dict(batch=0, q=None, k=None, v=None, out=None, d_state_out=0), dict(tokens=0, q=None, k=None, v=None, out=None),
                   dict(heads=96, qk_heads=32, out=heads(batch=96 * 64 * 16, token=96 * 64))):
        refused("hs_delta_rule", delta(**change), "NULL context")
    for change in (dict(norm=False, eps=-1.0, d_norm_weight=1), dict(d_norm_weight=0), dict(k_tokens=0, k=None, v=None),
                   dict(q_tokens=0, q=None, k=None, v=None, out=None, d_lambda=0), dict(batch=0, q=None, out=None), dict(kv_heads=2)):
        refused("hs_differential_attention", differential(**change), "NULL context")
    for change in (dict(tokens=0, d_x=0, d_out=0, d_router=0, d_w_in=0, d_w_out=0), dict(x_stride=0), dict(x_stride=-64), dict(out_stride=-64),
                   dict(tokens=1, out_stride=0), dict(d_mask=P + 1), dict(tokens=1024), dict(top=8), dict(experts=256)):
        refused("hs_expert_layer", experts(**change), "NULL context")


@pytest.mark.parametrize("name", sorted(CALLS))
def test_workspaces(name):
    call, make, query = CALLS[name]
    none = dict(d_workspace=0, workspace_bytes=0)
    none.update(dict(d_x=0, d_out=0, d_router=0, d_w_in=0, d_w_out=0) if name == "hs_expert_layer" else dict(q=None, k=None, v=None, out=None))
    assert query(make(**none)) >= 0
    with pytest.raises(hs.HsError) as e:
        query(make(dtype=7, **none))
    assert e.value.status == hs.HS_E_INVAL
    n = ctypes.c_size_t()
    raw = getattr(api.load(), query.__name__)
    assert raw(None, ctypes.byref(n)) == hs.HS_E_INVAL and raw(ctypes.byref(make()), None) == hs.HS_E_INVAL
    sizes = {"hs_delta_rule": dict(batch=8, tokens=600, out=heads(batch=1 << 30)), "hs_differential_attention": dict(batch=1, q_tokens=8, k_tokens=100000),
             "hs_expert_layer": dict()}[name]
    need = query(make(**sizes))
    if need:
        refused(name, make(**sizes, workspace_bytes=need - 1), "workspace too small", hs.HS_E_NOMEM)
        refused(name, make(**sizes, d_workspace=0), "workspace too small", hs.HS_E_NOMEM)
        refused(name, make(**sizes, d_workspace=P + 128), "256-byte aligned")
    refused(name, make(**sizes, workspace_bytes=need), "NULL context")


def test_counts_beyond_one_call_are_refused():
    far = heads(batch=1 << 40, token=1 << 20, head=64)
    refused("hs_delta_rule", delta(tokens=(1 << 31) - 1023, out=far), "too many tokens")
    refused("hs_delta_rule", delta(batch=1 << 20, heads=1 << 14, qk_heads=1, out=far), "too many heads")
    refused("hs_differential_attention", differential(batch=1 << 20, q_heads=1 << 13, kv_heads=1, out=far), "too many heads")
    refused("hs_differential_attention", differential(q_tokens=1 << 30, kv_heads=4, out=far), "too many tokens")


def test_gates_are_views_of_float32_tensors():
    import torch
    from paper_2402_04466_amd.harness import gates_of
    t = torch.zeros(2, 3, 4)
    g = gates_of(t[:, :, 1:])
    assert (g.d, g.batch, g.token, g.head) == (t.data_ptr() + 4, 12, 4, 1)
    for bad in (t.half(), t[0]):
        with pytest.raises(ValueError):
            gates_of(bad)


def test_the_expert_decoders_keys_have_length_one_and_its_state_is_the_track_decoders():
    import torch
    from paper_2402_04466_amd.track_expert_decoder import ExpertTrackDecoder
    dec = ExpertTrackDecoder(0, streams=2, heads=2, experts=3, hidden=8, device="cpu")
    assert torch.equal(dec.w_norm[1], torch.full((64,), 0.125)) and dec.state.shape == (16, 2, 64, 64)
    with pytest.raises(ValueError, match="even"):
        ExpertTrackDecoder(0, streams=1, heads=3, device="cpu")
    with pytest.raises(ValueError, match="one stream"):
        dec.forward(torch.zeros(2, 2, 8, 128, dtype=torch.float16), torch.zeros(2, 2, 5, 128, dtype=torch.float16))


@pytest.mark.parametrize("bad, name", [
    (dict(head_dim=128), "head_dim"), (dict(head_dim=72), "head_dim"), (dict(head_dim=24), "head_dim"), (dict(head_dim=0), "head_dim"),
    (dict(heads=258), "heads"), (dict(heads=0), "heads"), (dict(hidden=12), "hidden"), (dict(hidden=0), "hidden"),
    (dict(hidden=16392), "hidden"), (dict(experts=257), "experts"), (dict(experts=0), "experts"), (dict(top=0), "top"),
    (dict(top=9), "top"), (dict(experts=2, top=3), "top")])
def test_the_expert_decoder_refuses_what_its_operators_do(bad, name):
    """When it is made, not at the first frame."""
    from paper_2402_04466_amd.track_expert_decoder import ExpertTrackDecoder
    with pytest.raises(ValueError, match=name):
        ExpertTrackDecoder(0, **{**dict(streams=1, heads=2, device="cpu"), **bad})


@pytest.mark.parametrize("head_dim", [16, 64])
def test_the_expert_decoders_widest_and_narrowest_heads(head_dim):
    from paper_2402_04466_amd.track_expert_decoder import ExpertTrackDecoder
    assert ExpertTrackDecoder(0, streams=1, heads=2, head_dim=head_dim, experts=8, top=8, hidden=8, device="cpu").channels == 2 * head_dim
