"""CPU-only tests of the track decoder's operators at the boundary: the binding's descriptions have the header's
sizes, and everything a call must refuse is refused before any GPU work (no context exists here, and a
description that passes every check ends at the missing context)."""
import ctypes
import os
import subprocess

import pytest

import paper_2402_04466_amd as hs
from paper_2402_04466_amd import api

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 1 << 20     # a well aligned address that nothing reads


def test_binding_sizes_of_the_descriptions_match_the_header(tmp_path):
    names = ["hs_heads", "hs_norm_rotate_desc", "hs_retention_desc", "hs_cross_attention_desc"]
    src = tmp_path / "sz.c"
    src.write_text('#include <stdio.h>\n#include "hs.h"\nint main(void){'
                   + "".join(f'printf("%zu\\n", sizeof({n}));' for n in names)
                   + 'printf("%d %d %d\\n", HS_F16, HS_BF16, HS_MAX_HEADS);return 0;}\n')
    exe = tmp_path / "sz"
    subprocess.check_call(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)])
    out = subprocess.check_output([str(exe)]).split()
    assert [int(v) for v in out] == [ctypes.sizeof(getattr(hs, n)) for n in names] + [
        hs.HS_F16, hs.HS_BF16, hs.HS_MAX_HEADS]


def heads(d=P, batch=8 * 64 * 16, token=8 * 64, head=64):
    return hs.hs_heads(d, batch, token, head)


def norm_rotate(**change):
    kw = dict(dtype=hs.HS_F16, batch=2, tokens=16, q_heads=8, k_heads=8, head_dim=64, q=heads(), k=heads(2 * P),
              q_out=heads(3 * P), k_out=heads(4 * P), rotary_dim=64, d_frequencies=P)
    kw.update(change)
    return hs.make_norm_rotate_desc(**kw)


def retention(**change):
    kw = dict(dtype=hs.HS_F16, batch=2, tokens=16, q_heads=8, kv_heads=8, key_dim=64, value_dim=64, scale=0.125,
              decay=[0.9] * 8, q=heads(), k=heads(2 * P), v=heads(3 * P), out=heads(4 * P), d_state_in=P,
              d_state_out=P, d_workspace=P, workspace_bytes=1 << 40)
    kw.update(change)
    if "q_heads" in change and "decay" not in change:
        kw["decay"] = [0.9] * max(0, change["q_heads"])
    return hs.make_retention_desc(**kw)


def cross(**change):
    kw = dict(dtype=hs.HS_F16, batch=2, q_tokens=16, k_tokens=16, q_heads=8, kv_heads=8, head_dim=64, scale=0.125,
              q=heads(), k=heads(2 * P), v=heads(3 * P), out=heads(4 * P), d_workspace=P, workspace_bytes=1 << 40)
    kw.update(change)
    return hs.make_cross_attention_desc(**kw)


CALLS = {"hs_norm_rotate": (hs.hs_norm_rotate, norm_rotate), "hs_retention": (hs.hs_retention, retention),
         "hs_cross_attention": (hs.hs_cross_attention, cross)}


def refused(name, desc, words, status=hs.HS_E_INVAL):
    with pytest.raises(hs.HsError) as e:
        CALLS[name][0](0, desc)
    assert e.value.status == status and name in str(e.value) and words in str(e.value), str(e.value)


@pytest.mark.parametrize("name", sorted(CALLS))
def test_a_sound_description_is_only_short_of_a_context(name):
    refused(name, CALLS[name][1](), "NULL context")
    assert getattr(api.load(), name)(None, None, None) == hs.HS_E_INVAL
    assert "NULL description" in hs.hs_last_error()


BOTH = ["hs_retention", "hs_cross_attention"]
OUT = {"hs_norm_rotate": "q_out", "hs_retention": "out", "hs_cross_attention": "out"}


@pytest.mark.parametrize("name", sorted(CALLS))
@pytest.mark.parametrize("change, words", [
    (dict(dtype=0), "dtype"), (dict(dtype=3), "dtype"), (dict(batch=-1), "negative"),
    (dict(q=heads(0)), "q must be"), (dict(q=heads(P + 8)), "q must be"), (dict(q=heads(token=8 * 64 + 4)), "strides of q"),
    (dict(k=heads(0)), "k must be"), (dict(k=heads(head=68)), "strides of k"), (dict(k=heads(batch=4)), "strides of k")])
def test_refusals_common_to_all(name, change, words):
    refused(name, CALLS[name][1](**change), words)


@pytest.mark.parametrize("name", sorted(CALLS))
@pytest.mark.parametrize("strides", [dict(head=32), dict(head=0), dict(token=0), dict(batch=0), dict(batch=8 * 64),
                                     dict(token=-8 * 32), dict(batch=-(1 << 63))])
def test_outputs_whose_rows_overlap_are_refused(name, strides):
    refused(name, CALLS[name][1](**{OUT[name]: heads(5 * P, **strides)}), OUT[name])


@pytest.mark.parametrize("name", sorted(CALLS))
@pytest.mark.parametrize("strides", [dict(batch=64, token=2 * 8 * 64, head=128), dict(token=-8 * 64), dict(batch=1 << 40),
                                     dict(batch=64 * 16, token=64, head=2 * 64 * 16)])
def test_outputs_in_any_order_are_taken(name, strides):
    refused(name, CALLS[name][1](**{OUT[name]: heads(5 * P, **strides)}), "NULL context")


@pytest.mark.parametrize("name", BOTH)
@pytest.mark.parametrize("change, words", [
    (dict(kv_heads=3), "multiple of kv_heads"), (dict(kv_heads=0), "multiple of kv_heads"),
    (dict(q_heads=0), "multiple of kv_heads"), (dict(scale=float("nan")), "scale"), (dict(scale=float("inf")), "scale"),
    (dict(v=heads(0)), "v must be"), (dict(out=heads(0)), "out must be"), (dict(d_lengths=P + 2), "d_lengths")])
def test_refusals_common_to_attention(name, change, words):
    refused(name, CALLS[name][1](**change), words)


@pytest.mark.parametrize("change, words", [
    (dict(head_dim=60), "head_dim"), (dict(head_dim=136), "head_dim"), (dict(head_dim=0), "head_dim"),
    (dict(tokens=-1), "negative"), (dict(q_heads=-1), "heads"), (dict(rotary_dim=24), "rotary_dim"),
    (dict(rotary_dim=80), "rotary_dim"), (dict(rotary_dim=-16), "rotary_dim"), (dict(eps=-1e-6), "eps"),
    (dict(eps=float("nan")), "eps"), (dict(d_frequencies=0), "d_frequencies"), (dict(d_frequencies=P + 4), "d_frequencies"),
    (dict(d_positions=P + 4), "d_positions"), (dict(d_q_weight=P + 2), "weight"),
    (dict(q_out=heads(token=2 * 8 * 64, batch=2 * 8 * 64 * 16)), "other strides")])
def test_refusals_of_norm_rotate(change, words):
    refused("hs_norm_rotate", norm_rotate(**change), words)


def test_norm_rotate_takes_one_side_alone_and_outputs_in_place():
    for change in (dict(k_heads=0, k=None, k_out=None), dict(q_heads=0, q=None, q_out=None), dict(q_out=heads()),
                   dict(rotary_dim=0, d_frequencies=0), dict(norm=False, eps=-1.0), dict(tokens=0, q=None, k=None)):
        refused("hs_norm_rotate", norm_rotate(**change), "NULL context")


@pytest.mark.parametrize("change, words", [
    (dict(key_dim=4), "key_dim"), (dict(value_dim=132), "value_dim"), (dict(tokens=-1), "negative"),
    (dict(q_heads=72, kv_heads=8), "at most 64"), (dict(decay=[0.9] * 7 + [1.5]), "decay of head 7"),
    (dict(decay=[-0.1] + [0.9] * 7), "decay of head 0"), (dict(decay=[float("nan")] * 8), "decay of head 0"),
    (dict(d_state_out=0), "d_state_out"), (dict(d_state_out=P + 8), "d_state_out"), (dict(d_state_in=P + 4), "d_state_in")])
def test_refusals_of_retention(change, words):
    refused("hs_retention", retention(**change), words)


def test_retention_without_decay_is_refused():
    d = retention()
    d.decay = None
    refused("hs_retention", d, "NULL decay")


@pytest.mark.parametrize("change, words", [
    (dict(head_dim=12), "head_dim"), (dict(q_tokens=-1), "negative"), (dict(k_tokens=-1), "negative"),
    (dict(d_lse=P + 2), "d_lse")])
def test_refusals_of_cross_attention(change, words):
    refused("hs_cross_attention", cross(**change), words)


def test_calls_over_nothing_look_at_no_pointer():
    refused("hs_cross_attention", cross(k_tokens=0, k=None, v=None), "NULL context")
    refused("hs_cross_attention", cross(q_tokens=0, q=None, k=None, v=None, out=None), "NULL context")
    refused("hs_retention", retention(tokens=0, q=None, k=None, v=None, out=None), "NULL context")
    refused("hs_retention", retention(batch=0, q=None, k=None, v=None, out=None, d_state_out=0), "NULL context")


def test_workspace_queries_need_no_pointers_and_refuse_what_the_calls_refuse():
    for make, query in ((retention, hs.hs_query_retention_workspace), (cross, hs.hs_query_cross_attention_workspace)):
        none = dict(q=None, k=None, v=None, out=None, d_workspace=0, workspace_bytes=0)
        assert query(make(**none)) >= 0
        with pytest.raises(hs.HsError) as e:
            query(make(dtype=7, **none))
        assert e.value.status == hs.HS_E_INVAL
    n = ctypes.c_size_t()
    for name in ("hs_query_retention_workspace", "hs_query_cross_attention_workspace"):
        assert getattr(api.load(), name)(None, ctypes.byref(n)) == hs.HS_E_INVAL
    assert api.load().hs_query_retention_workspace(ctypes.byref(retention()), None) == hs.HS_E_INVAL
    assert api.load().hs_query_cross_attention_workspace(ctypes.byref(cross()), None) == hs.HS_E_INVAL


def test_binding_refuses_a_decay_of_another_length():
    with pytest.raises(ValueError):
        retention(decay=[0.9] * 7)


def test_counts_beyond_one_call_are_refused():
    """Products of two counts that would not fit the kernels' numbers."""
    far = heads(batch=1 << 40, token=1 << 20, head=64)
    refused("hs_norm_rotate", norm_rotate(batch=1 << 16, tokens=1 << 16, q=far, k=far, q_out=far, k_out=far), "too many tokens")
    refused("hs_cross_attention", cross(batch=1 << 20, q_heads=1 << 14, kv_heads=1), "too many heads")


def test_a_decoders_reset_keeps_the_memory_that_graphs_work_on():
    import torch
    from paper_2402_04466_amd.track_decoder import TrackDecoder
    dec = TrackDecoder(0, streams=2, heads=1, device="cpu")
    state, frame = dec.state, dec.frame
    state.fill_(3.0)
    frame.fill_(5)
    dec.reset()
    assert dec.state is state and dec.frame is frame
    assert not state.any() and not frame.any()
    assert state.dtype == torch.float32 and frame.dtype == torch.int64


def test_a_decoder_refuses_inputs_that_do_not_fit_before_any_work():
    import torch
    from paper_2402_04466_amd.track_decoder import TrackDecoder
    dec = TrackDecoder(0, streams=1, heads=1, device="cpu")
    half = dict(dtype=torch.float16)
    x, maps, mask = torch.zeros(1, 3, 8, 64, **half), torch.zeros(1, 3, 405, 64, **half), torch.ones(1, 3, 405, dtype=torch.uint8)
    for bad in (x[0], x[:, :, :7], x.float(), x.to("meta"), torch.zeros(2, 3, 8, 64, **half), torch.zeros(1, 3, 8, 32, **half)):
        with pytest.raises(ValueError, match="x must be"):
            dec.forward(bad, maps, mask)
    for bad in (maps[0], maps[:, :1], torch.zeros(1, 1, 405 * 3, 64, **half), torch.zeros(1, 3, 405, 32, **half), maps.to(torch.bfloat16),
                maps.to("meta")):
        with pytest.raises(ValueError, match="maps must be"):
            dec.forward(x, bad, mask)
    for bad in (mask[0], mask[:, :1], mask[:, :, :404], mask.long(), mask.to(torch.float16), mask.to("meta")):
        with pytest.raises(ValueError, match="mask must be"):
            dec.forward(x, maps, bad)
    several = TrackDecoder(0, streams=2, heads=1, device="cpu")
    with pytest.raises(ValueError, match="one stream"):
        several.forward(torch.zeros(2, 2, 8, 64, **half), torch.zeros(2, 2, 5, 64, **half))
    assert not dec.frame.any() and not several.frame.any()
