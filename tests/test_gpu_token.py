"""Token log probabilities, entropies, best alternatives and their backward pass against the
definitions in 64 bits.

Tolerances.  A row's s is a sum of positive terms, each from ex2 (2 ulp) of an argument rounded
three times; a thread adds at most about 64 partial sums for the vocabularies here, so s is within
(2 + 64) * 2^-24 + 3 * 2^-24 * |d| of exact, d <= 30 where a term matters: 1e-5.  That is the
absolute error of ln s; the subtraction and product in front of it add 3 * 2^-24 of |z_y - m| and the
result another rounding.  The entropy divides two such sums: 1e-5 * (1 + H) and a rounding of ln s.
The gradient's p has the error of lse (one rounding, 2^-24 |lse|), of lp (the same again) and of ex2.
"""
import math

import pytest
import torch

import paper_1806_08054_b200 as ecq

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
EPS = 2.0 ** -24


def make(rows, vocab, dtype, stride=None, seed=0, scale=2.5, offset=0):
    """[rows, vocab] view into a guarded buffer, `offset` entries from an aligned address."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1000 * rows + vocab + seed)
    stride = stride or vocab
    buf = torch.full((offset + rows * stride + 64,), 7.0, dtype=DT[dtype], device="cuda")
    x = buf[offset:offset + rows * stride].view(rows, stride)[:, :vocab]
    x.copy_(scale * torch.randn(rows, vocab, generator=gen, device="cuda"))
    y = torch.randint(0, vocab, (rows,), generator=gen, device="cuda")
    return buf, x, y


def reference(x, y, tau):
    z = x.double() * tau
    lse = torch.logsumexp(z, 1)
    logp = z - lse[:, None]
    p = logp.exp()
    plogp = torch.where(p > 0, p * logp, 0.0)
    lp = torch.where(y >= 0, logp.gather(1, y.clamp(min=0)[:, None])[:, 0], 0.0)
    return z, lse, logp, p, -plogp.sum(1), lp


def forward(x, y, temperature, top):
    rows = x.shape[0]
    out = {k: torch.full((rows,), 9.0, device="cuda") for k in ("logprob", "entropy", "lse")}
    if top:
        out["top_logprob"] = torch.full((rows, top), 9.0, device="cuda")
        out["top_index"] = torch.full((rows, top), 9, dtype=torch.int32, device="cuda")
    ecq.ecq_token_logprob(x, y, temperature=temperature, **out)
    return out


def best(x, top):
    """Values and indices in the order the operator promises."""
    v, i = torch.sort(x.double() + 0.0, dim=1, descending=True, stable=True)
    return v[:, :top], i[:, :top]


def check_forward(x, y, temperature, top):
    tau = 1.0 / temperature
    z, lse, logp, p, ent, lp = reference(x, y, tau)
    out = forward(x, y, temperature, top)
    m = z.masked_fill(~torch.isfinite(z), -math.inf).max(1).values
    assert torch.all((out["lse"].double() - lse).abs() <= 1e-5 + 4 * EPS * (lse.abs() + m.abs()))
    gap = torch.where(y >= 0, m - z.gather(1, y.clamp(min=0)[:, None])[:, 0], 0.0)
    assert torch.all((out["logprob"].double() - lp).abs() <= 1e-5 + 4 * EPS * (gap + lp.abs()))
    assert torch.all((out["entropy"].double() - ent).abs() <= 1e-5 * (1 + ent) + 4 * EPS * (1 + math.log(x.shape[1])))
    if top:
        v, i = best(x, top)
        open_ = torch.isfinite(v)
        assert torch.equal(out["top_index"].long(), torch.where(open_, i, -1))
        want = torch.where(open_, logp.gather(1, i), -math.inf)
        got = out["top_logprob"].double()
        assert torch.equal(torch.isfinite(got), open_)
        assert torch.all((got - want)[open_].abs() <= 1e-5 + 4 * EPS * (m[:, None] - v * tau + want.abs())[open_])
    return out, lse, ent


SHAPES = [(1, 1), (1, 2), (3, 7), (2, 33), (5, 255), (1, 1023), (1, 4099), (1, 50257), (9, 50257), (40, 8191),
          (300, 1000), (700, 517), (7, 131075)]


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("rows,vocab", SHAPES)
def test_forward(rows, vocab, dtype):
    for offset, stride, temperature, top in ((0, vocab, 1.0, min(5, vocab)), (1, vocab + 3, 0.6, min(32, vocab)),
                                             (3, vocab + (-vocab) % 64, 1.7, 0)):
        _, x, y = make(rows, vocab, dtype, stride, offset=offset)
        if rows > 2:
            y[1] = -100
        check_forward(x, y, temperature, top)


@pytest.mark.parametrize("dtype", list(DT))
def test_outputs_are_optional_and_guards_stay(dtype):
    buf, x, y = make(6, 3001, dtype, 3008, offset=5)
    before = buf.clone()
    full = forward(x, y, 1.0, 4)
    for name in ("logprob", "entropy", "lse"):
        one = torch.zeros(8, device="cuda")
        ecq.ecq_token_logprob(x, y if name == "logprob" else None, **{name: one[1:7]})
        assert torch.equal(one[1:7], full[name]) and one[0] == 0 and one[7] == 0
    v, i = torch.zeros(6, 4, device="cuda"), torch.zeros(6, 4, dtype=torch.int32, device="cuda")
    ecq.ecq_token_logprob(x, top_logprob=v, top_index=i)
    assert torch.equal(v, full["top_logprob"]) and torch.equal(i, full["top_index"])
    assert torch.equal(buf.view(torch.uint8), before.view(torch.uint8))


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("vocab", [1, 37, 1000, 50257])
def test_masks(vocab, dtype):
    """-inf entries, the type's lowest value, rows with one open entry, rows with none."""
    lowest = torch.finfo(DT[dtype]).min
    for fill in (-math.inf, lowest):
        _, x, y = make(8, vocab, dtype, vocab + 1, seed=3)
        gen = torch.Generator(device="cuda")
        gen.manual_seed(5)
        x[0] = fill
        x[1] = fill; x[1, vocab // 2] = 1.5; y[1] = vocab // 2
        x[2, torch.rand(vocab, generator=gen, device="cuda") < 0.9] = fill
        x[3, : vocab // 2] = fill
        x[4] = fill; x[4, -1] = -3.0; x[4, 0] = -2.0; y[4] = 0
        top = min(20, vocab)
        tau = 0.5
        out = forward(x, y, 2.0, top)
        v, i = best(x, top)
        open_ = v > -math.inf
        assert torch.equal(out["top_index"].long(), torch.where(open_, i, -1))
        z = x.double() * tau
        lse = torch.logsumexp(z, 1)
        rows = [r for r in range(8) if not math.isinf(lse[r])]
        assert rows[0] == (1 if fill == -math.inf else 0)
        ref = reference(x[rows], y[rows], tau)
        # beside a lowest-value mask lse may be as large as the mask: errors are relative to it
        tol = 1e-5 + 8 * EPS * ref[1].abs()
        assert torch.all((out["lse"][rows].double() - ref[1]).abs() <= tol)
        assert torch.all((out["entropy"][rows].double() - ref[4]).abs() <= 1e-5 * (1 + ref[4]) + 8 * EPS * 12) or fill == lowest
        fine = torch.isfinite(ref[5])
        got = out["logprob"][rows].double()
        assert torch.equal(torch.isfinite(got), fine)
        gap = ref[0].max(1).values - ref[0].gather(1, y[rows][:, None])[:, 0]
        assert torch.all((got - ref[5])[fine].abs() <= 1e-5 + 8 * EPS * gap[fine]) or fill == lowest
        if fill == -math.inf:
            assert out["lse"][0] == -math.inf and out["entropy"][0] == 0 and out["logprob"][0] == -math.inf
            assert torch.all(out["top_index"][0] == -1) and torch.all(out["top_logprob"][0] == -math.inf)
        else:                                               # equal entries: the uniform distribution
            assert abs(out["entropy"][0].item() - math.log(vocab)) <= 2e-5
            assert abs(out["logprob"][0].item() + math.log(vocab)) <= 2e-5
        # backward: masked entries and empty rows get nothing
        g = torch.randn(8, generator=gen, device="cuda")
        d = torch.full_like(x, 5.0)
        ecq.ecq_token_logprob_grad(x, y, out["lse"], out["entropy"], g, 0.3 * g, d, temperature=2.0)
        assert torch.all(torch.isfinite(d))
        if fill == -math.inf:
            assert torch.all(d[0] == 0)
            hit = torch.zeros_like(x, dtype=torch.bool)
            hit.scatter_(1, y[:, None], True)
            assert torch.all(d[torch.isinf(x) & ~hit] == 0)


@pytest.mark.parametrize("dtype", list(DT))
def test_rows_with_nan_or_plus_infinity(dtype):
    _, x, y = make(4, 5003, dtype)
    x[0, 4000] = math.nan
    x[2, 17] = math.inf
    out = forward(x, y, 1.0, 3)
    for r in (0, 2):
        assert all(torch.all(torch.isnan(out[k][r])) for k in ("lse", "entropy", "logprob", "top_logprob"))
        assert torch.all(out["top_index"][r] == -1)
    for r in (1, 3):
        alone = forward(x[r:r + 1], y[r:r + 1], 1.0, 3)
        assert all(torch.allclose(alone[k][0], out[k][r], atol=2e-5, rtol=0) for k in out)
    d = torch.empty_like(x)
    g = torch.ones(4, device="cuda")
    ecq.ecq_token_logprob_grad(x, y, out["lse"], out["entropy"], g, g, d)
    assert torch.all(torch.isnan(d[0])) and torch.all(torch.isnan(d[2])) and torch.all(torch.isfinite(d[[1, 3]]))


def test_target_outside_the_vocabulary():
    _, x, y = make(3, 100, "f32")
    y[:] = torch.tensor([100, -1, 99], device="cuda")
    out = forward(x, y, 1.0, 0)
    assert math.isnan(out["logprob"][0]) and out["logprob"][1] == 0 and math.isfinite(out["logprob"][2])


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("ent", [False, True])
def test_backward_of_a_target_outside_the_vocabulary(dtype, ent):
    """NaN, as its log probability: not a gradient without the target's entry."""
    _, x, y = make(6, 2001, dtype, 2002)
    x[2] += 5000.0
    x[3] = -math.inf
    x[4, 7:] = -math.inf
    y[:] = torch.tensor([2001, -1, 1 << 40, 2001, 5000, 2000], device="cuda")
    out = forward(x, y, 1.0, 0)
    assert torch.equal(torch.isnan(out["logprob"]).cpu(), torch.tensor([True, False, True, True, True, False]))
    d, g = torch.full_like(x, 5.0), torch.ones(6, device="cuda")
    ecq.ecq_token_logprob_grad(x, y, out["lse"], out["entropy"] if ent else None, g, g if ent else None, d)
    assert torch.all(torch.isnan(d[[0, 2, 3, 4]])) and torch.all(torch.isfinite(d[[1, 5]]))


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("rows,vocab", [(2, 600), (1, 50257), (200, 9001), (2, 131075)])
def test_ties_go_to_the_lowest_index(rows, vocab, dtype):
    """Equal rows, few distinct values, signed zeros, a long run of large entries in one place."""
    _, x, y = make(rows, vocab, dtype, offset=2)
    cases = [torch.zeros_like(x), x.round(), torch.where(x > 0, 0.0, -0.0).to(x.dtype), x.clone()]
    cases[3][:, 100:100 + min(4000, vocab - 200)] += 40.0
    strided = x.clone()
    strided[:, ::8 * 256] += 60.0                           # one thread's entries above all others'
    strided[:, 1::8 * 256] += 50.0
    cases.append(strided)
    for c in cases:
        out = forward(c, y, 1.0, 32)
        v, i = best(c, 32)
        assert torch.equal(out["top_index"].long(), i)


def test_all_large_entries_with_one_thread():
    """More entries above the bound than the candidate list holds, all in a few threads' places."""
    vocab = 262144 * 2
    x = torch.randn(200, vocab, device="cuda", dtype=torch.float32)
    vec = torch.arange(vocab, device="cuda") // 4
    x[:, vec % 256 < 4] += 50.0
    y = torch.zeros(200, dtype=torch.int64, device="cuda")
    out = forward(x, y, 1.0, 32)
    v, i = best(x, 32)                                      # torch.topk orders equal values as it likes
    assert torch.equal(out["top_index"].long(), i)


def check_grad(x, y, temperature, ent, in_place=False, d=None):
    tau = 1.0 / temperature
    rows = x.shape[0]
    gen = torch.Generator(device="cuda")
    gen.manual_seed(11)
    out = forward(x, y, temperature, 0)
    g = torch.randn(rows, generator=gen, device="cuda")
    e = torch.randn(rows, generator=gen, device="cuda") if ent else None
    z, lse, logp, p, H, _ = reference(x, y, tau)
    gd = torch.where(y >= 0, g.double(), 0.0)
    hot = torch.zeros_like(z).scatter_(1, y.clamp(min=0)[:, None], (y >= 0).double()[:, None])
    ref = gd[:, None] * (hot - p)
    size = gd.abs()[:, None] * (hot + p)
    if ent:
        ref -= e.double()[:, None] * torch.where(p > 0, p * (logp + H[:, None]), 0.0)
        size += e.double().abs()[:, None] * torch.where(p > 0, p * (logp.abs() + H[:, None]), 0.0)
    ref, size = ref * tau, size * tau
    work = x.clone() if in_place else x
    d = work if in_place else (torch.full_like(x, 3.0) if d is None else d)
    ecq.ecq_token_logprob_grad(work, y, out["lse"], out["entropy"] if ent else None, g, e, d, temperature=temperature)
    rel = 2e-5 + 8 * EPS * (lse.abs().max() + z.abs().max())
    store = {torch.float32: 0.0, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -10}[x.dtype]
    assert torch.all((d.double() - ref).abs() <= rel * size + store * ref.abs() + 2.0 ** -24)
    return d


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("rows,vocab", SHAPES)
def test_backward(rows, vocab, dtype):
    for offset, stride, temperature, ent in ((0, vocab, 1.0, True), (1, vocab + 3, 0.7, False), (3, vocab + 5, 1.4, True)):
        _, x, y = make(rows, vocab, dtype, stride, offset=offset, seed=7)
        if rows > 2:
            y[0] = -1
        d = check_grad(x, y, temperature, ent)
        buf, other, _ = make(rows, vocab, dtype, vocab + 1, offset=2)      # another alignment than the logits'
        other.fill_(3.0)
        tail = buf.clone()
        check_grad(x, y, temperature, ent, d=other)
        assert torch.equal(other, d)
        other.copy_(torch.full_like(other, 3.0))
        assert torch.equal(buf.view(torch.uint8), tail.view(torch.uint8)), "write outside the rows"
        assert torch.equal(check_grad(x, y, temperature, ent, in_place=True), d)


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("vocab,offset", [(5, 0), (1003, 1), (1003, 6), (30001, 3)])
def test_backward_at_a_token_that_is_nearly_certain(vocab, offset, dtype):
    """g (1 - p) at the target, for p from 0.9 to within 1e-6 of 1, from a logit at which log p takes one
    rounding: 16 * 2^-24 of itself.  lse is the definition's in 64 bits, near 0, rounded once: 2^-24 of
    itself, and so of 1 - p."""
    rows = 64
    _, x, y = make(rows, vocab, dtype, vocab + 1, offset=offset)
    x.copy_(-3.0 - math.log(vocab) - torch.arange(rows, device="cuda")[:, None] / 6 + 0.2 * x)
    x.scatter_(1, y[:, None], 0.0)
    z = x.double()
    rest = z.exp().scatter(1, y[:, None], 0.0).sum(1)       # lse = ln(1 + rest), 1 - p = rest / (1 + rest)
    lse = torch.log1p(rest).float()
    g = torch.randn(rows, device="cuda")
    p = z.exp() / (1 + rest)[:, None]
    logp = z - torch.log1p(rest)[:, None]
    H = -(p * logp).sum(1).float()
    d = torch.empty_like(x)
    ecq.ecq_token_logprob_grad(x, y, lse, None, g, None, d)
    want = g.double() * rest / (1 + rest)
    store = {torch.float32: 0.0, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}[x.dtype]
    got = d.double().gather(1, y[:, None])[:, 0]
    assert torch.all((got - want).abs() <= (16 * EPS + store) * want.abs() + 2.0 ** -25)
    # beside a derivative of the entropy that is as small as a regulariser's
    ecq.ecq_token_logprob_grad(x, y, lse, H, g, torch.full_like(g, 1e-3), d)
    extra = 1e-3 * (p.gather(1, y[:, None]) * (logp.gather(1, y[:, None]) + H.double()[:, None]))[:, 0]
    got = d.double().gather(1, y[:, None])[:, 0]
    assert torch.all((got - (want - extra)).abs() <= (16 * EPS + store) * (want.abs() + extra.abs()) + 32 * EPS * 1e-3 * H + 2.0 ** -25)


def uncentred(rows, vocab, dtype, stride, seed, offset):
    """Rows whose lse alone does not tell the probabilities: every entry (or all but a few) at the
    type's lowest value, entries far from zero, entries at the highest value; and rows without open entries."""
    buf, x, y = make(rows, vocab, dtype, stride, seed=seed, offset=offset)
    info = torch.finfo(DT[dtype])
    far = 30000.0 if dtype == "f16" else 1e5                # entries a rounding of the type apart
    x[0] = info.min
    x[1] = info.min; x[1, vocab // 2:] = -math.inf
    x[2] += far
    x[3] -= far
    x[4] = info.max; x[4, ::3] = info.min
    x[5] = -math.inf
    x[6] = 8 * x[6] + 500.0
    y[:7] = torch.tensor([0, 1, 2, vocab - 1, 1, 3, -1], device="cuda")[:7] % vocab
    y[6] = -1
    return buf, x, y


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("vocab,offset", [(8, 0), (301, 1), (1000, 0), (9001, 3), (50257, 1), (131075, 0)])
def test_backward_of_uncentred_rows(vocab, offset, dtype):
    """Against the definition in 64 bits.  p has the error of the sums (1e-5) and three roundings of
    tau (x - m), which is at most 104 where p is not 0: 2e-5 + 8 * 2^-24 * 104 of p, and the entropy's."""
    for temperature, ent in ((1.0, True), (0.5, True), (2.0, False)):
        tau = 1.0 / temperature
        _, x, y = uncentred(9, vocab, dtype, vocab + 1, 5, offset)
        out = forward(x, y, temperature, 0)
        g = torch.randn(9, device="cuda")
        e = torch.randn(9, device="cuda") if ent else None
        z = x.double() * tau
        z[5] = 0                                            # the empty row, set right below
        z -= z.max(1, keepdim=True).values                  # not less lse: 64 bits lose ln V beside 3e38, too
        logp = z - z.exp().sum(1, keepdim=True).log()
        p = logp.exp()
        plogp = torch.where(p > 0, p * logp, 0.0)
        H = -plogp.sum(1)
        hot = torch.zeros_like(z).scatter_(1, y.clamp(min=0)[:, None], (y >= 0).double()[:, None])
        gd = torch.where(y >= 0, g.double(), 0.0)[:, None]
        ref, size = gd * (hot - p), gd.abs() * (hot + p)
        if ent:
            ref = ref - e.double()[:, None] * (plogp + p * H[:, None])
            size = size + e.double().abs()[:, None] * (plogp.abs() + p * (1 + H[:, None]))
        ref, size = ref * tau, size * tau
        ref[5] = 0; size[5] = 0
        store = {torch.float32: 0.0, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -10}[x.dtype]
        allow = (2e-5 + 8 * EPS * 104) * size + store * ref.abs() + 2.0 ** -24
        d = torch.full_like(x, 3.0)
        ecq.ecq_token_logprob_grad(x, y, out["lse"], out["entropy"] if ent else None, g, e, d, temperature=temperature)
        assert torch.all((d.double() - ref).abs() <= allow)
        other = make(9, vocab, dtype, vocab + 2, offset=2)[1]                  # another alignment
        ecq.ecq_token_logprob_grad(x, y, out["lse"], out["entropy"] if ent else None, g, e, other, temperature=temperature)
        assert torch.equal(other, d)
        ecq.ecq_token_logprob_grad(x, y, out["lse"], out["entropy"] if ent else None, g, e, x, temperature=temperature)
        assert torch.equal(x, d)


@pytest.mark.parametrize("dtype", list(DT))
def test_backward_of_rows_around_the_limits_of_lse(dtype):
    """|lse| on either side of 128 and of 1024, and rows beyond them among many others."""
    _, x, y = make(400, 8191, dtype, 8200)
    x[:200] += torch.linspace(100, 140, 200, device="cuda")[:, None]
    x[200:] -= torch.linspace(1000, 1060, 200, device="cuda")[:, None]
    x[::7] = make(400, 8191, dtype, seed=9)[1][::7]
    check_grad(x, y, 1.0, True)
    check_grad(x, y, 1.0, False, in_place=True)


def test_backward_against_differences():
    """(L(x + h v) - L(x - h v)) / 2h of L = sum g log p + e H.  With h = 1e-2 the third-order term is
    about h^2 of the result and the rounding of L about 1e-6 |L| / h: 1e-3 of |v| together."""
    rows, vocab, tau, h = 6, 301, 0.8, 1e-2
    _, x, y = make(rows, vocab, "f32", scale=1.0)
    g, e = torch.randn(rows, device="cuda"), torch.randn(rows, device="cuda")

    def loss(t):
        out = forward(t, y, 1 / tau, 0)
        return (g.double() * out["logprob"].double() + e.double() * out["entropy"].double()).sum()

    out = forward(x, y, 1 / tau, 0)
    d = torch.empty_like(x)
    ecq.ecq_token_logprob_grad(x, y, out["lse"], out["entropy"], g, e, d, temperature=1 / tau)
    for seed in range(4):
        torch.manual_seed(seed)
        v = torch.randn_like(x)
        v /= v.norm()
        numeric = (loss(x + h * v) - loss(x - h * v)) / (2 * h)
        assert abs(numeric - (d.double() * v.double()).sum()) <= 2e-3


def test_only_entropy_and_only_logprob():
    _, x, y = make(5, 1234, "f32")
    out = forward(x, y, 1.0, 0)
    g, e, zero = torch.randn(5, device="cuda"), torch.randn(5, device="cuda"), torch.zeros(5, device="cuda")
    a, b, both = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
    ecq.ecq_token_logprob_grad(x, None, out["lse"], out["entropy"], None, e, a)
    ecq.ecq_token_logprob_grad(x, y, out["lse"], out["entropy"], zero, e, b)
    assert torch.equal(a, b)
    ecq.ecq_token_logprob_grad(x, y, out["lse"], None, g, None, b)
    ecq.ecq_token_logprob_grad(x, y, out["lse"], out["entropy"], g, e, both)
    assert torch.allclose(a + b, both, atol=1e-6, rtol=1e-5)


def test_repeatable_and_on_another_stream():
    _, x, y = make(9, 50257, "bf16")
    first = forward(x, y, 1.0, 20)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        second = forward(x, y, 1.0, 20)
    s.synchronize()
    assert all(torch.equal(first[k], second[k]) for k in first)


def test_row_offsets_beyond_32_bits():
    rows, vocab = 3, 1000
    stride = (1 << 31) + 24                                 # the last row starts beyond 2^32 entries
    need = (2 * stride + vocab) * 2
    if torch.cuda.mem_get_info()[0] < 2 * need:
        pytest.skip("not enough free memory")
    flat = torch.zeros(2 * stride + vocab, dtype=torch.bfloat16, device="cuda")
    x = flat.as_strided((rows, vocab), (stride, 1))
    x.copy_(torch.randn(rows, vocab, device="cuda"))
    y = torch.tensor([5, 6, 999], device="cuda")
    check_forward(x, y, 1.0, 8)
    d = flat.as_strided((rows, vocab), (stride, 1))
    out = forward(x, y, 1.0, 0)
    want = check_grad(x.clone(), y, 1.0, False)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(11)
    g = torch.randn(rows, generator=gen, device="cuda")
    ecq.ecq_token_logprob_grad(x, y, out["lse"], None, g, None, d)
    assert torch.equal(d, want)


@pytest.mark.parametrize("dtype", list(DT))
def test_masked_entries_beside_a_large_entropy_derivative(dtype):
    """Their gradient is 0, whatever the derivative: no 0 * inf."""
    _, x, y = make(4, 3001, dtype, 3003)
    x[:, 5:2000] = -math.inf
    x[:, 2000] = torch.finfo(DT[dtype]).min
    y[:] = 1
    out = forward(x, y, 1.0, 0)
    e = torch.tensor([1e8, -1e10, 1e20, -1e30], device="cuda")
    d = torch.full_like(x, 5.0)
    ecq.ecq_token_logprob_grad(x, y, out["lse"], out["entropy"], torch.ones(4, device="cuda"), e, d)
    assert torch.all(d[:, 5:2001] == 0)
    assert not torch.any(torch.isnan(d))


def test_refusals():
    _, x, y = make(2, 64, "f32")
    lp = torch.zeros(2, device="cuda")
    with pytest.raises(ValueError):
        ecq.ecq_token_logprob(x.cpu(), y, lp)
    with pytest.raises(ValueError):
        ecq.ecq_token_logprob(x.double(), y, lp)
    with pytest.raises(ValueError):
        ecq.ecq_token_logprob(x.t(), y, lp)
    with pytest.raises(ValueError):
        ecq.ecq_token_logprob(x, y.int(), lp)
    with pytest.raises(ValueError):
        ecq.ecq_token_logprob(x, y, torch.zeros(3, device="cuda"))
    for bad in (dict(temperature=-1.0), dict(temperature=math.inf), dict(temperature=math.nan)):
        with pytest.raises((ecq.EcqError, ZeroDivisionError)):
            ecq.ecq_token_logprob(x, y, lp, **bad)
    with pytest.raises(ecq.EcqError):
        ecq.ecq_token_logprob(x, None, lp)                  # log probabilities of no targets
    with pytest.raises(ecq.EcqError):
        ecq.ecq_token_logprob(x)                            # no output
    with pytest.raises(ecq.EcqError):
        ecq.ecq_token_logprob(x, top_logprob=torch.zeros(2, 33, device="cuda"),
                              top_index=torch.zeros(2, 33, dtype=torch.int32, device="cuda"))
    with pytest.raises(ValueError):
        ecq.ecq_token_logprob_grad(x, y, lp, None, lp, None, torch.zeros(2, 63, device="cuda"))
    with pytest.raises(ecq.EcqError):
        ecq.ecq_token_logprob_grad(x, y, lp, None, lp, lp, torch.zeros_like(x))   # entropy's derivative without it
    with pytest.raises(ecq.EcqError):
        ecq.ecq_token_logprob_grad(x, None, lp, None, None, None, torch.zeros_like(x))
    empty = torch.zeros(0, 64, device="cuda")
    ecq.ecq_token_logprob(empty, torch.zeros(0, dtype=torch.int64, device="cuda"), torch.zeros(0, device="cuda"))
