"""hs_expert_layer through the C ABI against the formulas in 64 bits.

The choice has to be that of scores summed in 64 bits.  Bounds of the outputs, value by value: a weight of a chosen expert is off by
at most e = (2 * channels + 64) * 2^-24 * (1 + the sum of |x| |router|) relative, as scores of fp32 sums are good enough for it; a
product's fp32 sum of n terms by n * 2^-24 of the sum of magnitudes; silu's slope is at most 1.1; what the second product takes is
rounded to the type once (u), or below that to 2^-32 of the row's largest; the output is rounded once."""
import pytest
import torch

from operator_common import DEV, F32, TYPES, close, expert_call, half_step, normal, smallest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx(hs):
    c = hs.hs_init(0)
    yield c
    hs.hs_shutdown(c)


@pytest.fixture
def gen():
    return torch.Generator(device=DEV).manual_seed(17)


def inputs(g, n, ch, f, e, t):
    return (normal(g, n, ch, dtype=t), (normal(g, e, ch) * ch ** -0.5).to(t), (normal(g, e, 2 * f, ch) * ch ** -0.5).to(t),
            (normal(g, e, ch, f) * f ** -0.5).to(t))


def reference(x, router, w_in, w_out, top, renormalise, mask):
    u = half_step(x.dtype)
    n, ch = x.shape
    e, f = router.shape[0], w_out.shape[2]
    here = torch.ones(n, dtype=torch.bool, device=DEV) if mask is None else mask != 0
    xx = x.double()
    score = xx @ router.double().T
    ranked = score.sort(dim=-1, descending=True, stable=True)
    chosen = ranked.indices[:, :top]
    p = torch.softmax(ranked.values[:, :top], -1) if renormalise else torch.softmax(score, -1).gather(1, chosen)
    size = (xx.abs() @ router.double().abs().T).amax(-1, keepdim=True)
    p_off = p * (2 * ch + 64) * F32 * (1 + size)
    out, bound = torch.zeros(2, n, ch, dtype=torch.float64, device=DEV)
    for i in range(e):
        hit, slot = torch.nonzero((chosen == i) & here[:, None], as_tuple=True)
        if not len(hit):
            continue
        a, w = xx[hit], w_in[i].double()
        y, m = a @ w.T, a.abs() @ w.abs().T * (ch + 8) * F32
        gate, up = y[:, :f], y[:, f:]
        h = gate * torch.sigmoid(gate) * up
        off = 1.1 * m[:, :f] * up.abs() + (gate * torch.sigmoid(gate)).abs() * m[:, f:] + m[:, :f] * m[:, f:] + 8 * F32 * h.abs()
        off = off * (1 + u) + u * h.abs() + 2.0 ** -32 * h.abs().amax(-1, keepdim=True)
        wo = w_out[i].double()
        part = h @ wo.T
        part_off = off @ wo.abs().T + (h.abs() + off) @ wo.abs().T * (f + 8) * F32
        out[hit] += p[hit, slot, None] * part
        bound[hit] += p[hit, slot, None] * part_off + p_off[hit, slot, None] * (part.abs() + part_off)
    bound = bound * (1 + u + 16 * F32) + (u + 16 * F32) * out.abs() + smallest(x.dtype)
    chosen = torch.where(here[:, None], chosen, -1).to(torch.int32)
    return out, torch.where(here[:, None], bound, 0.0), chosen, torch.where(here[:, None], p, 0.0), p_off + F32


def check(hs, ctx, x, router, w_in, w_out, top, renormalise=True, mask=None, what="", poison=False):
    want, bound, chosen, p, p_off = reference(x, router, w_in, w_out, top, renormalise, mask)
    if poison:
        x = torch.where(mask[:, None] != 0, x, float("nan"))
    n, ch = x.shape
    out = torch.full((n, ch), 7.0, dtype=x.dtype, device=DEV)
    got = torch.full((n, top), 99, dtype=torch.int32, device=DEV)
    weights = torch.full((n, top), 7.0, device=DEV)
    expert_call(hs, ctx, x, router, w_in, w_out, out, top, renormalise=renormalise, mask=mask, chosen=got, weights=weights)
    assert torch.equal(got, chosen), what
    close(weights, p, p_off, f"{what}: weights")
    close(out, want, bound, f"{what}: outputs")
    again = torch.empty_like(out)                        # without the choice, and the same bits again
    expert_call(hs, ctx, x, router, w_in, w_out, again, top, renormalise=renormalise, mask=mask)
    assert torch.equal(again, out)
    return out


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("n, ch, f, e, top, renormalise", [
    (1, 8, 8, 1, 1, True), (1, 512, 1024, 16, 2, True), (8, 512, 1024, 16, 2, True), (2, 64, 72, 3, 3, False),
    (37, 520, 1336, 6, 3, False), (16, 128, 256, 64, 8, True), (17, 136, 40, 5, 1, False), (33, 8, 264, 7, 7, True),
    (64, 256, 136, 2, 1, True), (65, 64, 8, 256, 8, False), (128, 1024, 512, 32, 4, True), (300, 72, 200, 4, 2, True),
    (1024, 64, 64, 3, 2, False), (1000, 264, 328, 70, 5, True), (1024, 16, 24, 1, 1, True), (5, 2056, 24, 4, 2, True),
    (0, 64, 64, 4, 2, True)])
def test_matches_the_formulas(hs, ctx, gen, dtype, n, ch, f, e, top, renormalise):
    check(hs, ctx, *inputs(gen, n, ch, f, e, TYPES[dtype]), top, renormalise)


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("n", [1, 9, 130, 1024])
def test_masked_tokens_pass_through_none(hs, ctx, gen, dtype, n):
    args = inputs(gen, n, 72, 136, 6, TYPES[dtype])
    mask = (torch.rand(n, generator=gen, device=DEV) < 0.6).to(torch.uint8) * 5
    for m in (mask, torch.zeros_like(mask)):
        check(hs, ctx, *args, 3, mask=m, poison=True, what=f"{int((m != 0).sum())} of {n}")


@pytest.mark.parametrize("n", [3, 40, 700])
def test_all_tokens_on_one_expert_and_experts_without_a_token(hs, ctx, gen, n):
    x, router, w_in, w_out = inputs(gen, n, 64, 72, 9, torch.float16)
    x[:, 0] = 8.0
    router[:, 0] = 0
    router[4, 0], router[7, 0] = 4.0, 2.0
    out = check(hs, ctx, x, router, w_in, w_out, 1)
    assert out.any()
    check(hs, ctx, x, router, w_in, w_out, 2, renormalise=False)


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("n", [1, 8, 200])
def test_ties_go_to_the_lower_index_and_neighbours_are_told_apart(hs, ctx, gen, dtype, n):
    """Equal rows of the router give equal scores; rows that differ by one step of one small value differ by less than
    fp32 sums can tell."""
    x, router, w_in, w_out = inputs(gen, n, 256, 24, 12, TYPES[dtype])
    router[5:] = router[2]
    check(hs, ctx, x, router, w_in, w_out, 8)
    router[:] = router[2]
    check(hs, ctx, x, router, w_in, w_out, 3, renormalise=False)
    x[:, 9] = 2.0 ** -8
    router[:, 9] = 2.0 ** -12
    router[6, 9] = 2.0 ** -12 * (1 + 2 * half_step(x.dtype))
    check(hs, ctx, x, router, w_in, w_out, 3, renormalise=False)
    x[:, 9] = -x[:, 9]
    check(hs, ctx, x, router, w_in, w_out, 2)


@pytest.mark.parametrize("n", [1, 40])
@pytest.mark.parametrize("size", [2.0 ** -9, 1.0, 48.0])
def test_hidden_values_of_every_magnitude(hs, ctx, gen, n, size):
    """Hidden values below and beyond fp16's range keep their bits."""
    x, router, w_in, w_out = inputs(gen, n, 64, 136, 4, torch.float16)
    w_in = (w_in.float() * size).to(torch.float16)
    x = (x.float() * (size if size > 1 else 1)).to(torch.float16)
    w_out = (w_out.float() * (2.0 ** -10 if size > 1 else 1)).to(torch.float16)
    check(hs, ctx, x, router, w_in, w_out, 2)


def test_a_token_that_is_not_finite_changes_no_other(hs, ctx, gen):
    for n in (4, 100):
        for bad in (float("nan"), float("inf")):
            x, router, w_in, w_out = inputs(gen, n, 64, 72, 5, torch.bfloat16)
            clean, out = (torch.empty_like(x) for _ in range(2))
            expert_call(hs, ctx, x, router, w_in, w_out, clean, 2)
            x[n // 2, 3] = bad
            chosen = torch.empty(n, 2, dtype=torch.int32, device=DEV)
            expert_call(hs, ctx, x, router, w_in, w_out, out, 2, chosen=chosen)
            others = torch.arange(n, device=DEV) != n // 2
            assert torch.equal(out[others], clean[others]) and not torch.isfinite(out[n // 2]).any()
            assert bool((chosen >= 0).all()) and bool((chosen < 5).all()) and chosen[n // 2, 0] != chosen[n // 2, 1]


@pytest.mark.parametrize("n", [5, 90])
def test_strides(hs, ctx, gen, n):
    """Rows of wider tensors, in and out, backwards, and one row for all."""
    _, router, w_in, w_out = inputs(gen, n, 64, 72, 5, torch.float16)
    wide_x = normal(gen, n, 96, dtype=torch.float16)
    x = wide_x[:, 8:72]
    want, bound, chosen, _, _ = reference(x, router, w_in, w_out, 2, True, None)
    wide = torch.full((n, 88), 7.0, dtype=torch.float16, device=DEV)
    out = wide[:, 16:80]
    expert_call(hs, ctx, x, router, w_in, w_out, out, 2)
    close(out, want, bound, "strided")
    assert bool((wide[:, :16] == 7).all()) and bool((wide[:, 80:] == 7).all())
    same = x[:1].expand(n, 64)
    expert_call(hs, ctx, same, router, w_in, w_out, out, 2)
    want, bound, _, _, _ = reference(same, router, w_in, w_out, 2, True, None)
    close(out, want, bound, "one row")
    d = hs.make_expert_layer_desc(dtype=hs.HS_F16, tokens=n, channels=64, hidden=72, experts=5, top=2, d_x=x[n - 1:].data_ptr(),
                                  x_stride=-96, d_out=out[n - 1:].data_ptr(), out_stride=-88, d_router=router.data_ptr(),
                                  d_w_in=w_in.data_ptr(), d_w_out=w_out.data_ptr())
    from operator_common import give_workspace, stream
    work = give_workspace(d, hs.hs_query_expert_layer_workspace(d))
    hs.hs_expert_layer(ctx, d, stream())
    want, bound, _, _, _ = reference(x, router, w_in, w_out, 2, True, None)
    close(out, want, bound, "backwards")


@pytest.mark.parametrize("n", [8, 200])
def test_on_another_stream_and_in_graphs(hs, ctx, gen, n):
    x, router, w_in, w_out = inputs(gen, n, 128, 136, 8, torch.bfloat16)
    want = torch.empty_like(x)
    keep = [expert_call(hs, ctx, x, router, w_in, w_out, want, 2)]
    other = torch.cuda.Stream()
    torch.cuda.synchronize()
    out = torch.empty_like(x)
    with torch.cuda.stream(other):
        heavy = torch.randn(2048, 2048, device=DEV)
        for _ in range(20):
            heavy = (heavy @ heavy).clamp_(-1, 1)
        late = x * 1.0
        keep.append(expert_call(hs, ctx, late, router, w_in, w_out, out, 2))
    other.synchronize()
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        keep.append(expert_call(hs, ctx, x, router, w_in, w_out, out, 2))
    for i in range(4):
        x.copy_(x.roll(1, 0) * 0.75)
        expert_call(hs, ctx, x, router, w_in, w_out, want, 2)
        out.fill_(7.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want), i


def test_weights_beyond_32_bits(hs, ctx, gen):
    """Experts more than 2^32 elements apart."""
    ch, f, e, n = 4096, 2056, 256, 3
    t = torch.bfloat16
    x, router = normal(gen, n, ch, dtype=t), (normal(gen, e, ch) * ch ** -0.5).to(t)
    w_in, w_out = torch.zeros(e, 2 * f, ch, dtype=t, device=DEV), torch.zeros(e, ch, f, dtype=t, device=DEV)
    used = (x.double() @ router.double().T).topk(2, -1).indices.flatten().unique().tolist()
    assert max(used) > 128
    for i in used:
        w_in[i], w_out[i] = normal(gen, 2 * f, ch, dtype=t) * ch ** -0.5, normal(gen, ch, f, dtype=t) * f ** -0.5
    check(hs, ctx, x, router, w_in, w_out, 2)


@pytest.mark.parametrize("n, e, top", [(200, 64, 1), (300, 40, 4), (70, 3, 2), (1024, 256, 1)])
def test_many_tokens_on_an_expert_that_few_are_expected_on(hs, ctx, gen, n, e, top):
    """All tokens pick the same experts, so that theirs are taken in turn, in every form that the average number asks for."""
    x, router, w_in, w_out = inputs(gen, n, 64, 72, e, torch.bfloat16)
    x[:, 0] = 8.0
    router[:, 0] = 0
    router[1, 0] = 4.0
    check(hs, ctx, x, router, w_in, w_out, top)


def test_two_calls_at_once_with_workspaces_of_their_own(hs, ctx, gen):
    sets = [inputs(gen, n, 128, 136, 8, torch.float16) for n in (12, 200)]
    want = [torch.empty_like(s[0]) for s in sets]
    keep = [expert_call(hs, ctx, *s, out, 2) for s, out in zip(sets, want)]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in sets], [torch.empty_like(s[0]) for s in sets]
    for _ in range(5):
        for st, s, out in zip(streams, sets, got):
            with torch.cuda.stream(st):
                keep.append(expert_call(hs, ctx, *s, out, 2))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("apart", [10, 20, 23, 24, 25, 26, 27, 28, 32])
@pytest.mark.parametrize("n, e, top", [(8, 4, 2), (8, 70, 2), (40, 6, 3), (100, 16, 2), (100, 6, 2), (300, 4, 2)])
def test_hidden_values_far_below_others_of_their_token(hs, ctx, gen, apart, n, e, top):
    """Sixteen hidden values side by side are 2^apart and more above a token's others, which alone reach the outputs: their output
    weights are positive as they are, so that what is lost of them adds up.  In every form that the number of tokens asks for."""
    ch, f = 64, 40
    x, router, w_in, w_out = inputs(gen, n, ch, f, e, torch.float16)
    gate, up = w_in[:, :f].float(), w_in[:, f:].float()
    up[:, 16:] = gate[:, 16:]                                # silu(a) a > 0; of a = 2^-6 and less about a^2 / 2
    up[:, :16] *= 2.0 ** 12
    gate[:, 16:] *= 2.0 ** -6
    up[:, 16:] *= 2.0 ** (12 - apart + 7)
    w_in = torch.cat((gate, up), 1).to(torch.float16)
    w_out = w_out.float().abs() * 2.0 ** min(14, apart - 11)      # outputs of about one
    w_out[:, :, :16] = 0
    check(hs, ctx, x, router, w_in, w_out.to(torch.float16), top, what=f"2^{apart}")
