"""hs_delta_rule through the C ABI against the recurrence in 64 bits.

Bounds.  With keys of length at most 1, beta in [0, 1] and g <= 1 a token's map of the state, g (1 - beta k k^T), lengthens
no column, so the errors of the tokens add up at most.  One token's own error in a column of the state, as a
length, is at most 20 * 2^-24 of (length of the column + |u|): a sum of at most 128 products in fp32 (8 in a row, then a
tree of 4 levels), the decay (2), its product, the difference, the product by beta, and the update (2).  A chunk of 32
tokens, formed by matrix products, has 32 such shares, and takes fewer steps: sums of at most 128 + 32 products in a row of
24-bit parts and a solved system of 32 rows whose solution no element of exceeds the values that the recurrence forms.
An output is rounded once and has the state's error times the query's length, and, where the state and the values go through
the matrix pipe in two parts, 2^-16 of the sum of magnitudes."""
import pytest
import torch

from operator_common import DEV, F32, TYPES, close, delta_call, half_step, normal, smallest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx(hs):
    c = hs.hs_init(0)
    yield c
    hs.hs_shutdown(c)


@pytest.fixture
def gen():
    return torch.Generator(device=DEV).manual_seed(11)


def inputs(g, b, n, h, hk, dk, dv, t):
    q, k = normal(g, b, n, hk, dk), normal(g, b, n, hk, dk)
    q, k = (x / x.norm(dim=-1, keepdim=True) * 0.99 for x in (q, k))       # at most 1 after rounding
    log_decay = -torch.rand(b, n, h, generator=g, device=DEV) ** 4
    beta = torch.rand(b, n, h, generator=g, device=DEV)
    return q.to(t), k.to(t), normal(g, b, n, h, dv, dtype=t), log_decay, beta, normal(g, b, h, dk, dv)


def reference(q, k, v, log_decay, beta, state, scale, lengths=None):
    """Outputs, final state and bounds of both, token by token."""
    b, n, h, dv = v.shape
    dk = q.shape[3]
    group = h // q.shape[2]
    q, k = (x.double().repeat_interleave(group, 2) for x in (q, k))
    v = v.double()
    s = torch.zeros(b, h, dk, dv, dtype=torch.float64, device=DEV) if state is None else state.double().clone()
    g = torch.ones(b, n, h, dtype=torch.float64, device=DEV) if log_decay is None else log_decay.double().exp()
    beta = torch.ones(b, n, h, dtype=torch.float64, device=DEV) if beta is None else beta.double()
    out, size = torch.zeros(2, b, n, h, dv, dtype=torch.float64, device=DEV)
    err = torch.zeros(b, h, dv, dtype=torch.float64, device=DEV)
    for t in range(n):
        on = torch.ones(b, dtype=torch.bool, device=DEV) if lengths is None else t < lengths
        kt, qt = (torch.where(on[:, None, None], x[:, t], 0.0) for x in (k, q))
        vt, gt, bt = (torch.where(on.view(-1, *[1] * (x.dim() - 2)), x[:, t], fill) for x, fill in ((v, 0.0), (g, 1.0), (beta, 0.0)))
        u = bt[..., None] * (vt - gt[..., None] * (kt[..., None, :] @ s).squeeze(-2))
        step = 20 * F32 * (s.norm(dim=-2) + bt[..., None] * (vt.abs() + s.norm(dim=-2)) + u.abs())
        err = err + torch.where(on[:, None, None], step, 0.0)
        s = gt[..., None, None] * s + kt[..., None] * u[..., None, :]
        out[:, t] = (qt[..., None, :] @ s).squeeze(-2) * scale
        # magnitudes of what is summed: the state's columns and the values since
        size[:, t] = abs(scale) * (err + 2.0 ** -16 * (s.norm(dim=-2) + 8 * u.abs() + s.abs().amax(-2)))
    return out, s, size, err


def check(got, end, ref, dtype, what):
    out, s, size, err = ref
    u = half_step(dtype)
    close(got, out, u * out.abs() + (1 + u) * size + smallest(dtype), f"{what}: outputs")
    close(end, s, err[:, :, None, :].expand_as(s), f"{what}: state")


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("b, n, h, hk, dk, dv", [
    (1, 1, 1, 1, 8, 8), (8, 1, 8, 8, 64, 64), (3, 1, 6, 2, 128, 128), (2, 2, 4, 4, 72, 56), (2, 8, 4, 2, 64, 64),
    (2, 9, 4, 2, 64, 64), (1, 16, 2, 2, 16, 24), (2, 31, 3, 1, 96, 80), (1, 32, 2, 1, 128, 128), (1, 33, 2, 2, 40, 104),
    (5, 63, 2, 2, 64, 64), (2, 64, 2, 1, 128, 64), (1, 65, 8, 8, 64, 128), (2, 130, 6, 3, 104, 72), (1, 257, 2, 2, 96, 80),
    (3, 100, 2, 2, 8, 8), (2, 70, 2, 1, 120, 8), (2, 70, 2, 1, 8, 120)])
def test_matches_the_recurrence(hs, ctx, gen, dtype, b, n, h, hk, dk, dv):
    t = TYPES[dtype]
    q, k, v, log_decay, beta, state = inputs(gen, b, n, h, hk, dk, dv, t)
    out, end = torch.full((b, n, h, dv), 7.0, dtype=t, device=DEV), torch.full_like(state, 7.0)
    delta_call(hs, ctx, q, k, v, out, log_decay, beta, state, end, dk ** -0.5)
    check(out, end, reference(q, k, v, log_decay, beta, state, dk ** -0.5), t, "whole")
    # in place, and the same bits again
    again, same = torch.empty_like(out), state.clone()
    delta_call(hs, ctx, q, k, v, again, log_decay, beta, same, same, dk ** -0.5)
    assert torch.equal(again, out) and torch.equal(same, end)


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("n, lengths", [(1, [0, 1, -3, 5]), (5, [0, 1, 5, 4]), (70, [0, 1, 70, 33, 32, 31, 64, 900, -1]), (300, [257, 8, 9, 300])])
def test_ragged_lengths(hs, ctx, gen, dtype, n, lengths):
    """Lengths of nothing, beyond the ends, and within chunks; what lies behind them is not used whatever it holds."""
    t, b, h, dk, dv = TYPES[dtype], len(lengths), 3, 64, 72
    q, k, v, log_decay, beta, state = inputs(gen, b, n, h, h, dk, dv, t)
    lens = torch.tensor(lengths, dtype=torch.int32, device=DEV)
    inside = lens.clamp(0, n)
    ref = reference(q, k, v, log_decay, beta, state, 0.125, inside)
    behind = torch.arange(n, device=DEV) >= inside[:, None]
    for x, poison in ((q, float("nan")), (k, float("inf")), (v, float("nan")), (log_decay, float("nan")), (beta, float("inf"))):
        x[behind] = poison
    out, end = torch.full((b, n, h, dv), 7.0, dtype=t, device=DEV), torch.full_like(state, 7.0)
    delta_call(hs, ctx, q, k, v, out, log_decay, beta, state, end, 0.125, lens)
    assert not out[behind].any()
    check(out, end, ref, t, "ragged")


def test_no_tokens_copies_the_state_and_no_state_is_zeros(hs, ctx, gen):
    t = torch.float16
    q, k, v, log_decay, beta, state = inputs(gen, 2, 40, 2, 2, 64, 64, t)
    out, end = torch.empty(2, 40, 2, 64, dtype=t, device=DEV), torch.full_like(state, 7.0)
    delta_call(hs, ctx, q[:, :0], k[:, :0], v[:, :0], out[:, :0], log_decay[:, :0], beta[:, :0], state, end, 1.0)
    assert torch.equal(end, state)
    delta_call(hs, ctx, q[:0], k[:0], v[:0], out[:0], log_decay[:0], beta[:0], state[:0], end[:0], 1.0)
    for n in (1, 8, 40):
        o = torch.empty(2, n, 2, 64, dtype=t, device=DEV)
        delta_call(hs, ctx, q[:, :n], k[:, :n], v[:, :n], o, log_decay[:, :n], beta[:, :n], None, end, 1.0)
        check(o, end, reference(q[:, :n], k[:, :n], v[:, :n], log_decay[:, :n], beta[:, :n], None, 1.0), t, f"{n} tokens, no state")


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("n", [1, 5, 70])
def test_gates_left_out_and_at_their_ends(hs, ctx, gen, dtype, n):
    """No decay, no beta, either; a decay of nothing (log of zero) in the middle of it, and betas of 0 and 1."""
    t = TYPES[dtype]
    q, k, v, log_decay, beta, state = inputs(gen, 2, n, 2, 2, 64, 64, t)
    log_decay[:, n // 2, 0] = -float("inf")
    log_decay[:, n // 3, 1] = -3000.0
    log_decay[:, n // 3 + 1:, 1] = -1e-3
    beta[:, n // 2] = 1.0
    beta[:, n // 4] = 0.0
    for a, e in ((log_decay, beta), (None, beta), (log_decay, None), (None, None)):
        out, end = torch.empty_like(v), torch.empty_like(state)
        delta_call(hs, ctx, q, k, v, out, a, e, state, end, 0.125)
        check(out, end, reference(q, k, v, a, e, state, 0.125), t, f"{a is None}, {e is None}")


@pytest.mark.parametrize("n", [70, 200])
def test_the_same_key_again_and_again(hs, ctx, gen, n):
    """One key for all tokens, beta 1: the state holds the newest value only; the chunks' system is as full as it gets."""
    t = torch.bfloat16
    q, k, v, log_decay, beta, state = inputs(gen, 2, n, 2, 2, 64, 64, t)
    k = torch.zeros_like(k)
    k[..., 5] = 1.0
    log_decay.zero_()
    beta.fill_(1.0)
    out, end = torch.empty_like(v), torch.empty_like(state)
    delta_call(hs, ctx, k, k, v, out, log_decay, beta, state, end, 1.0)
    check(out, end, reference(k, k, v, log_decay, beta, state, 1.0), t, "one key")
    assert (out.float() - v.float()).abs().max() <= 2 * half_step(t) * v.float().abs().max()


@pytest.mark.parametrize("dtype", sorted(TYPES))
def test_a_clip_cut_into_calls_is_the_clip(hs, ctx, gen, dtype):
    t = TYPES[dtype]
    q, k, v, log_decay, beta, state = inputs(gen, 3, 150, 4, 2, 64, 64, t)
    ref = reference(q, k, v, log_decay, beta, state, 0.125)
    for cuts in ([0, 150], [0, 1, 2, 70, 150], [0, 32, 64, 150], list(range(151))):
        out, s = torch.empty_like(v), state.clone()
        for a, e in zip(cuts, cuts[1:]):
            delta_call(hs, ctx, q[:, a:e], k[:, a:e], v[:, a:e], out[:, a:e], log_decay[:, a:e], beta[:, a:e], s, s, 0.125)
        check(out, s, ref, t, f"{len(cuts) - 1} calls")


@pytest.mark.parametrize("n", [1, 3, 100])
def test_strides_of_every_kind(hs, ctx, gen, n):
    """Token-major tensors, one projection for several, reversed order, one sequence's keys for all, gates side by side."""
    b, h, d, t = 4, 2, 64, torch.bfloat16
    _, _, _, log_decay, beta, state = inputs(gen, b, n, h, h, d, d, t)
    x = normal(gen, n, b, 3 * h, d + 8)
    x = (x / x[..., :d].norm(dim=-1, keepdim=True) * 0.99).to(t)
    q, k, v = (x[:, :, i * h:(i + 1) * h, :d].transpose(0, 1) for i in range(3))
    k = k[:1].expand(b, n, h, d)
    both = torch.stack((log_decay.transpose(0, 1), beta.transpose(0, 1)), -1)          # [n, b, h, 2]
    log_decay, beta = (both[..., i].transpose(0, 1) for i in range(2))
    beta = beta[:, :, :1].expand(b, n, h)
    ref = reference(q, k, v, log_decay, beta, state, 0.125)
    wide = torch.full((n, h, b, d + 16), 7.0, dtype=t, device=DEV)
    out = wide[:, :, :, 8:8 + d].permute(2, 0, 1, 3)
    end = torch.empty_like(state)
    delta_call(hs, ctx, q, k, v, out, log_decay, beta, state, end, 0.125)
    check(out, end, ref, t, "strided")
    assert bool((wide[..., :8] == 7).all()) and bool((wide[..., 8 + d:] == 7).all())


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("n", [1, 20, 100])
@pytest.mark.parametrize("size", [2.0 ** -60, 2.0 ** 60])
def test_states_of_every_magnitude(hs, ctx, gen, dtype, n, size):
    """A state's column of another magnitude than the values, and another one than its neighbours, keeps its bits."""
    t = TYPES[dtype]
    q, k, v, log_decay, beta, state = inputs(gen, 2, n, 2, 2, 64, 64, t)
    v[..., ::2] = 0
    state[..., ::2] *= size
    out, end = torch.empty_like(v), torch.empty_like(state)
    delta_call(hs, ctx, q, k, v, out, log_decay, beta, state, end, 0.125)
    want, s, room, err = reference(q, k, v, log_decay, beta, state, 0.125)
    close(end, s, err[:, :, None, :].expand_as(s), "state")
    fits = want.abs() < torch.finfo(t).max / 2
    close(torch.where(fits, out, 0), torch.where(fits, want, 0.0), half_step(t) * (want.abs() + room) + room + smallest(t), "outputs")


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("n, spot", [(1, 0), (5, 3), (70, 1), (70, 66), (200, 63), (200, 64)])
@pytest.mark.parametrize("which", ["q", "k", "v", "log_decay", "beta", "state"])
@pytest.mark.parametrize("value", [float("inf"), float("nan")])
def test_what_is_not_finite_reaches_its_columns_from_its_token_on(hs, ctx, gen, dtype, n, spot, which, value):
    t, b, h, d = TYPES[dtype], 2, 2, 64
    q, k, v, log_decay, beta, state = inputs(gen, b, n, h, h, d, d, t)
    clean, end0 = torch.empty_like(v), torch.empty_like(state)
    delta_call(hs, ctx, q, k, v, clean, log_decay, beta, state, end0, 0.125)
    ref = reference(q, k, v, log_decay, beta, state, 0.125)
    bad_out, bad_end = torch.zeros_like(v, dtype=torch.bool), torch.zeros_like(state, dtype=torch.bool)
    if which == "q":
        q[1, spot, 1, 7] = value
        bad_out[1, spot, 1] = True
    elif which == "v":
        v[1, spot, 1, 7] = value
        bad_out[1, spot:, 1, 7], bad_end[1, 1, :, 7] = True, True
    elif which == "state":
        state[1, 1, 3, 7] = value
        bad_out[1, :, 1, 7], bad_end[1, 1, :, 7] = True, True
    else:
        if which == "k":
            k[1, spot, 1, 7] = value
        else:
            (log_decay if which == "log_decay" else beta)[1, spot, 1] = value
        bad_out[1, spot:, 1], bad_end[1, 1] = True, True
    out, end = torch.empty_like(v), torch.empty_like(state)
    delta_call(hs, ctx, q, k, v, out, log_decay, beta, state, end, 0.125)
    assert torch.equal(~torch.isfinite(out), bad_out) and torch.equal(~torch.isfinite(end), bad_end)
    want, s, size, err = ref
    out, end = torch.where(bad_out, clean, out), torch.where(bad_end, end0, end)
    check(out, end, ref, t, "what stays finite")


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("n", [4, 40])
def test_long_keys_follow_the_formula(hs, ctx, gen, dtype, n):
    """Keys that are not of length one: the state grows token by token, and follows the recurrence relative to its size."""
    t, b, h, d = TYPES[dtype], 2, 2, 32
    q, k, v, log_decay, beta, state = inputs(gen, b, n, h, h, d, d, t)
    k = (k.float() * 1.5).to(t)
    beta.fill_(1.0)                                    # a token's map lengthens by up to |1 - 2.2| = 1.2
    out, end = torch.empty_like(v), torch.empty_like(state)
    delta_call(hs, ctx, q, k, v, out, log_decay, beta, state, end, 0.125)
    want, s, _, err = reference(q, k, v, log_decay, beta, state, 0.125)
    # errors grow with the same factor, and enter with keys and sums 1.5 and 2.3 times as large
    grown = 3 * 1.25 ** n
    close(end, s, grown * err[:, :, None, :].expand_as(s), "state")
    close(out, want, half_step(t) * want.abs() + 0.125 * (grown * err[:, None] + 2.0 ** -12 * s.norm(dim=-2)[:, None]) + 2.0 ** -12 * want.abs().amax()
          + smallest(t), "outputs")


@pytest.mark.parametrize("n", [1, 90])
def test_on_another_stream_and_in_graphs_that_share_a_workspace(hs, ctx, gen, n):
    b, h, d, t = 4, 4, 64, torch.float16
    q, k, v, log_decay, beta, state = inputs(gen, b, n, h, h, d, d, t)
    want, end = torch.empty_like(v), torch.empty_like(state)
    keep = [delta_call(hs, ctx, q, k, v, want, log_decay, beta, state, end, 0.125)]
    other = torch.cuda.Stream()
    torch.cuda.synchronize()
    out, s = torch.empty_like(v), torch.empty_like(state)
    with torch.cuda.stream(other):
        heavy = torch.randn(2048, 2048, device=DEV)
        for _ in range(20):
            heavy = (heavy @ heavy).clamp_(-1, 1)
        late = v * 1.0                                 # written on this stream, behind the products
        keep.append(delta_call(hs, ctx, q, k, late, out, log_decay, beta, state, s, 0.125))
    other.synchronize()
    assert torch.equal(out, want) and torch.equal(s, end)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        keep.append(delta_call(hs, ctx, q, k, v, out, log_decay, beta, state, s, 0.125))
    for i in range(3):
        v.mul_(0.5)
        delta_call(hs, ctx, q, k, v, want, log_decay, beta, state, end, 0.125)
        out.fill_(7.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(s, end), i


def test_offsets_beyond_32_bits(hs, ctx, gen):
    """Sequences and tokens more than 2^32 elements apart."""
    t, n, d = torch.float16, 40, 64
    q, k, v, log_decay, beta, state = inputs(gen, 2, n, 1, 1, d, d, t)
    far = torch.empty(2 ** 32 + 2 ** 20, dtype=t, device=DEV)
    view = far.as_strided((2, n, 1, d), (2 ** 32, 128, d, 1), 64)
    view.copy_(v)
    out = far.as_strided((2, n, 1, d), (2 ** 32, 128, d, 1), 2 ** 19)
    end = torch.empty_like(state)
    delta_call(hs, ctx, q, k, view, out, log_decay, beta, state, end, 0.125)
    check(out, end, reference(q, k, v, log_decay, beta, state, 0.125), t, "far")


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("b, n, h, dk, dv", [(70, 12, 8, 40, 24), (70, 14, 8, 40, 24), (300, 22, 8, 16, 16), (300, 23, 8, 16, 16), (1, 9, 1, 8, 128),
                                             (2, 40, 2, 32, 48), (2, 40, 2, 24, 80)])
def test_both_forms_next_to_the_number_of_tokens_that_parts_them(hs, ctx, gen, dtype, b, n, h, dk, dv):
    t = TYPES[dtype]
    q, k, v, log_decay, beta, state = inputs(gen, b, n, h, h, dk, dv, t)
    lens = torch.randint(0, n + 1, (b,), generator=gen, device=DEV, dtype=torch.int32)
    out, end = torch.full((b, n, h, dv), 7.0, dtype=t, device=DEV), torch.full_like(state, 7.0)
    delta_call(hs, ctx, q, k, v, out, log_decay, beta, state, end, 0.25, lens)
    check(out, end, reference(q, k, v, log_decay, beta, state, 0.25, lens), t, "next to it")


def of_two_parts(dtype):
    """What outputs lose of a product with a state's or token's 24 bits that go through the matrix pipe as two bf16 parts, each rounded: 2^-17 of what
    the parts leave, and 2^-16 for the two second parts' product where the other factor has more than 8 bits too."""
    return 2.0 ** -17 + (2.0 ** -16 if dtype == torch.float16 else 0.0)


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("dk", [8, 64, 128])
@pytest.mark.parametrize("n", [3, 40])
def test_what_a_state_loses_on_its_way_to_outputs(hs, ctx, gen, dtype, dk, n):
    """A state that stays as it is (beta 0, no decay), of values whose last bits all count the same way in products that nearly cancel."""
    t = TYPES[dtype]
    half = dk // 2
    a = 1 + 2.0 ** -7 - 2.0 ** -10 if dtype == "fp16" else 1.0            # cut off after 8 bits it would lose nearly 2^-7 (nothing)
    for s in (1 + 2.0 ** -7 - 2.0 ** -23, 1 + 2.0 ** -8 + 2.0 ** -15 - 2.0 ** -23, None):
        q = torch.full((1, n, 1, dk), -1.0, device=DEV)
        state = torch.empty(1, 1, dk, 8, device=DEV)
        if s is None:
            q[..., :half], state[:, :, :half] = normal(gen, n, 1, half), normal(gen, half, 8)
        else:
            q[..., :half], state[:, :, :half] = a, s
        q = q.to(t)
        state[:, :, half:] = (q[0, 0, 0, :half, None].float() * state[:, :, :half]).to(torch.bfloat16).float()
        k, v = normal(gen, 1, n, 1, dk, dtype=t), normal(gen, 1, n, 1, 8, dtype=t)
        out, end = torch.empty(1, n, 1, 8, dtype=t, device=DEV), torch.empty_like(state)
        delta_call(hs, ctx, q, k, v, out, None, torch.zeros(1, n, 1, device=DEV), state, end, 1.0)
        assert torch.equal(end, state)
        want = (q[0, :, 0].double() @ state[0, 0].double())[None, :, None]
        size = (q[0, :, 0].double().abs() @ state[0, 0].double().abs())[None, :, None]
        bound = half_step(t) * want.abs() * (1 + 2.0 ** -8) + (of_two_parts(t) + (dk + 32) * F32) * size + smallest(t)
        close(out, want, bound, f"state of {s}")


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("n", [4, 32, 50])
def test_what_tokens_lose_on_their_way_to_outputs(hs, ctx, gen, dtype, n):
    """Keys that have nothing in common, so that each token adds beta times its value, 24 bits of it, which later tokens' queries
    weigh; as above.  The weights are in two parts as well: 2^-16 for the two second parts' product, 2^-17 for what each leaves."""
    t, dk = TYPES[dtype], 64
    k = torch.eye(dk, device=DEV)[:n].view(1, n, 1, dk).to(t)
    a = 1 + 2.0 ** -7 - 2.0 ** -10 if dtype == "fp16" else 1.0
    for crafted in (True, False):
        q = torch.full((1, n, 1, dk), -1.0, device=DEV)
        q[..., 0::2] = a if crafted else normal(gen, n, 1, dk // 2)
        q = q.to(t)
        v = torch.ones(1, n, 1, 8, dtype=t, device=DEV)
        beta = torch.empty(1, n, 1, device=DEV)
        beta[:, 0::2] = 1 + 2.0 ** -7 - 2.0 ** -23 if crafted else torch.rand(1, n, 1, generator=gen, device=DEV)[:, 0::2]
        beta[:, 1::2] = (a * beta[:, 0:n // 2 * 2:2]).to(torch.bfloat16).float()
        out, end = torch.empty(1, n, 1, 8, dtype=t, device=DEV), torch.empty(1, 1, dk, 8, device=DEV)
        delta_call(hs, ctx, q, k, v, out, None, beta, None, end, 1.0)
        weights = torch.tril(q[0, :, 0, :n].double())                     # of token j for token i
        u = beta[0].double().expand(n, 8)
        want, size = (weights @ u)[None, :, None], (weights.abs() @ u.abs())[None, :, None]
        bound = half_step(t) * want.abs() * (1 + 2.0 ** -8) + (2.0 ** -15 + (n + 32) * F32) * size + smallest(t)
        close(out, want, bound, f"crafted {crafted}")


@pytest.mark.parametrize("n", [3, 40])
def test_finite_values_beyond_the_largest_of_bf16(hs, ctx, gen, n):
    """fp32 goes a little further than bf16: such values of the state, and of a token's value times beta, stay what they are."""
    t, dk, dv = torch.bfloat16, 16, 24
    far = 3.4e38
    assert torch.isinf(torch.tensor(far).to(t)) and far < torch.finfo(torch.float32).max
    k = torch.zeros(1, n, 1, dk, dtype=t, device=DEV)
    k[0, 1, 0, 3] = 1.0
    q = torch.full_like(k, 2.0 ** -20)
    v = torch.zeros(1, n, 1, dv, dtype=t, device=DEV)
    v[0, 1, 0, 5] = torch.finfo(t).max
    beta = torch.full((1, n, 1), far / torch.finfo(t).max, device=DEV)
    state = torch.zeros(1, 1, dk, dv, device=DEV)
    state[0, 0, 7, 2], state[0, 0, 8, 20] = far, 1.5
    out, end = torch.empty(1, n, 1, dv, dtype=t, device=DEV), torch.empty_like(state)
    delta_call(hs, ctx, q, k, v, out, None, beta, state, end, 1.0)
    want = state.clone()
    want[0, 0, 3, 5] = (v[0, 1, 0, 5].float() * beta[0, 1, 0])
    assert torch.equal(end, want) and torch.isfinite(want).all()
    for i in range(n):
        y = (want if i >= 1 else state)[0, 0].double().sum(0) * 2.0 ** -20
        close(out[0, i, 0], y, (half_step(t) + 16 * F32) * y.abs() + smallest(t), f"token {i}")
