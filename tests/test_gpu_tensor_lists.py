"""Norms, clipping, packing and updates of lists of tensors against their definitions in 64 bits.

Tolerances.  u = 2^-24 is half a step of fp32.  A sum of fp32 squares is formed in fp64, one of 16-bit squares in runs of eight in fp32: at
most 8 roundings of u each, halved by the square root, so a norm is off by NORM = 1 u (its rounding) or 5 u.  The factor adds one rounding
to that, the product another, the tensor's type half a step of its own; a gradual underflow costs half the smallest step."""
import math

import numpy as np
import pytest
import torch

import draco_inputs as di

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF_STEP = {"f32": U, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
SMALLEST = {"f32": 2.0 ** -150, "bf16": 2.0 ** -134, "f16": 2.0 ** -25}
PAD = 16
SENTINEL = 77.0


def _dr():
    import paper_1803_09877_b200 as dr
    return dr


class List:
    """Tensors of the given sizes, each in memory of its own, `shift` elements behind a 16-byte boundary, with sentinels around it."""

    def __init__(self, sizes, types, shifts=None, seed=0, sigma=0.05, absent=(), like=None):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.types, self.sizes = types, sizes
        self.memory, self.tensors = [], []
        for i, (n, t) in enumerate(zip(sizes, types)):
            m = torch.full((PAD + 8 + n + PAD,), SENTINEL, dtype=TYPES[t], device="cuda")
            s = PAD + (shifts[i % len(shifts)] if shifts else 0)
            v = m[s:s + n]
            if like is None:
                v.copy_(torch.randn(n, generator=g, device="cuda") * sigma * (1 + i % 3))
            self.memory.append((m, s, n))
            self.tensors.append(None if i in absent else v)

    def around_is_untouched(self):
        return all(bool((m[:s] == SENTINEL).all()) and bool((m[s + n:] == SENTINEL).all()) for m, s, n in self.memory)

    def wide(self):
        """Values in 64 bits; zeros where absent."""
        return [np.zeros(n) if v is None else v.double().cpu().numpy() for v, n in zip(self.tensors, self.sizes)]

    def bits(self):
        return [m.clone() for m, _, _ in self.memory]

    def has_bits(self, other):
        return all(torch.equal(m.view(torch.uint8), o.view(torch.uint8)) for (m, _, _), o in zip(self.memory, other))

    @property
    def norm_tolerance(self):
        return U * (1 if all(t == "f32" for t in self.types) else 5) * (1 + 1e-6)


def _norm64(parts, kind):
    if kind == "2":
        return math.sqrt(sum(float(np.dot(p, p)) for p in parts))
    return max([float(np.abs(p).max()) for p in parts if p.size], default=0.0)


def _kind(kind):
    return _dr().NORM_2 if kind == "2" else _dr().NORM_MAX


def _near(got, want, rel):
    assert abs(float(got) - want) <= rel * want, (float(got), want, rel)


def _scaled_ok(got, value, factor, t, off):
    """got = value * factor, `factor` off by at most `off`, product and type rounded once each."""
    want = value * factor
    bound = np.abs(want) * ((1 + off) * (1 + U) * (1 + HALF_STEP[t]) - 1 if t != "f32" else off + U + off * U) * (1 + 1e-9) + SMALLEST[t] + 2.0 ** -150
    bad = np.abs(got - want) > bound
    assert not bad.any(), (t, int(bad.sum()), float(np.abs(got - want).max()))


EDGES = [0, 1, 2, 3, 7, 8, 9, 127, 1017, 1023, 1024, 1025, 2040, 2047, 2048, 2049, 4097, 0, 12_345]
LISTS = {
    "one": ([1], ["f32"]),
    "empty": ([0, 0], ["f32", "bf16"]),
    "edges_f32": (EDGES, ["f32"] * len(EDGES)),
    "edges_bf16": (EDGES, ["bf16"] * len(EDGES)),
    "edges_f16": (EDGES, ["f16"] * len(EDGES)),
    "mixed": (EDGES + [70_001, 5], (["bf16", "f32", "f16"] * 7)[: len(EDGES) + 2]),
    "large": ([3_000_001, 64, 2_500_000], ["bf16", "f32", "f32"]),
    "hundred": ([37 * (i % 5) + i for i in range(100)], ["f16", "f32"] * 50),
    # beyond what one cluster takes
    "long_f32": (EDGES + [400_003], ["f32"] * (len(EDGES) + 1)),
    "long_bf16": ([900_001] + EDGES, ["bf16"] * (len(EDGES) + 1)),
    "long_mixed": (EDGES + [300_007, 250_001, 9], (["f16", "f32", "bf16"] * 8)[: len(EDGES) + 3]),
    "thousand": ([257 + 64 * (i % 3) for i in range(1000)], ["bf16"] * 1000),
    "many": ([i % 7 for i in range(4500)], ["f32", "bf16", "f16"] * 1500),
}
SHIFTS = {"aligned": [0], "all": [0, 1, 2, 3, 4, 5, 6, 7], "three": [3]}


def _layout(l):
    return _dr().Layout(l.sizes, [TYPES[t] for t in l.types])


@pytest.mark.parametrize("kind", ["2", "max"])
@pytest.mark.parametrize("shift", sorted(SHIFTS))
@pytest.mark.parametrize("name", sorted(LISTS))
def test_norm(name, shift, kind):
    sizes, types = LISTS[name]
    absent = {2, 5} if len(sizes) > 6 else set()
    l = List(sizes, types, SHIFTS[shift], seed=11, absent=absent)
    before, lay = l.bits(), _layout(l)
    norm, again = torch.full((2, 1), -1.0, device="cuda")
    each = torch.full((len(sizes) + 1,), -1.0, device="cuda")
    lay.norm(l.tensors, norm, kind=_kind(kind))
    lay.norm(l.tensors, again, each=each[:-1], kind=_kind(kind))
    parts = l.wide()
    tol = 0.0 if kind == "max" else l.norm_tolerance
    _near(norm, _norm64(parts, kind), tol)
    _near(again, _norm64(parts, kind), tol)
    for e, p in zip(each.tolist(), parts):
        _near(e, _norm64([p], kind), tol)
    assert each[-1].item() == -1.0
    assert l.has_bits(before)
    for _ in range(3):                                   # the same inputs, the same bits
        third = torch.zeros(1, device="cuda")
        lay.norm(l.tensors, third, kind=_kind(kind))
        assert third.item() == norm.item()


@pytest.mark.parametrize("separately", [False, True])
@pytest.mark.parametrize("where", ["in place", "same shifts", "other shifts"])
@pytest.mark.parametrize("kind", ["2", "max"])
@pytest.mark.parametrize("name", sorted(LISTS))
def test_clip(name, kind, where, separately):
    sizes, types = LISTS[name]
    absent = {2, 5} if len(sizes) > 6 else set()
    l = List(sizes, types, SHIFTS["all"], seed=12, absent=absent)
    out = None if where == "in place" else List(sizes, types, SHIFTS["all" if where == "same shifts" else "three"], like=l, absent=absent)
    parts, before, lay = l.wide(), l.bits(), _layout(l)
    want, each = _norm64(parts, kind), [_norm64([p], kind) for p in parts]
    # some tensors are above the limit and some below it
    limit = float(np.float32(np.median([e for e in each if e] or [1.0]) if separately else want / 3))
    norm = torch.full((1,), -1.0, device="cuda")
    each_got = torch.full((len(sizes),), -1.0, device="cuda") if separately else None
    lay.clip(l.tensors, limit, out=out.tensors if out else None, norm=norm, each=each_got, separately=separately, kind=_kind(kind))
    tol = 0.0 if kind == "max" else l.norm_tolerance
    _near(norm, want, tol)
    target = out or l
    for i, (x, p) in enumerate(zip(target.tensors, parts)):
        v = each[i] if separately else want
        if separately:
            _near(each_got[i], v, tol)
        if x is None or not p.size:
            continue
        # a factor of its own, or 1 where the norm is a rounding away from the limit
        factor = limit / v if v > limit else 1.0
        _scaled_ok(x.double().cpu().numpy(), p, factor, types[i], tol + U)
        if v < limit * (1 - 1e-5):
            assert np.array_equal(x.double().cpu().numpy(), p)
    assert target.around_is_untouched()
    if out:
        assert l.has_bits(before)
        assert all(bool((m == SENTINEL).all()) for i, (m, _, _) in enumerate(out.memory) if i in absent)


@pytest.mark.parametrize("limit", [None, 0.5, 1e9])
@pytest.mark.parametrize("row_shift", [0, 1, 2, 3])
@pytest.mark.parametrize("shift", sorted(SHIFTS))
@pytest.mark.parametrize("name", sorted(LISTS))
def test_pack(name, shift, row_shift, limit):
    sizes, types = LISTS[name]
    absent = {2, 5, 18} if len(sizes) > 18 else set()
    l = List(sizes, types, SHIFTS[shift], seed=13, sigma=0.3, absent=absent)
    parts, before, lay = l.wide(), l.bits(), _layout(l)
    d = sum(sizes)
    memory = torch.full((PAD + 4 + d + PAD,), SENTINEL, device="cuda")
    row = memory[PAD + row_shift:PAD + row_shift + d]
    norm = torch.full((1,), -1.0, device="cuda")
    v = _norm64(parts, "2")
    if limit is None:
        lay.pack(l.tensors, row)
        factor, off = 1.0, 0.0
    else:
        lay.pack(l.tensors, row, max_norm=limit, norm=norm)
        _near(norm, v, l.norm_tolerance)
        factor, off = (limit / v, l.norm_tolerance + U) if v > limit else (1.0, 0.0)
    want = np.concatenate(parts)
    got = row.cpu().numpy().astype(np.float64)
    if factor == 1.0:
        assert np.array_equal(got, want)
    else:
        _scaled_ok(got, want, factor, "f32", off)
    assert bool((memory[:PAD + row_shift] == SENTINEL).all()) and bool((memory[PAD + row_shift + d:] == SENTINEL).all())
    assert l.has_bits(before)


@pytest.mark.parametrize("limit", [None, 0.5, 1e9])
@pytest.mark.parametrize("with_master", [False, True])
@pytest.mark.parametrize("shift", sorted(SHIFTS))
@pytest.mark.parametrize("name", sorted(LISTS))
def test_update(name, shift, with_master, limit):
    sizes, types = LISTS[name]
    absent = {2, 5, 18} if len(sizes) > 18 else set()
    w = List(sizes, types, SHIFTS[shift], seed=14, absent=absent)
    d = sum(sizes)
    g = torch.Generator(device="cuda").manual_seed(15)
    u = torch.randn(max(d, 1), generator=g, device="cuda")[:d]
    master = torch.randn(d + 8, generator=g, device="cuda") * 0.05 if with_master else None
    old, old_u = w.wide(), u.double().cpu().numpy()
    old_master = master.double().cpu().numpy() if with_master else None
    memory, lay, scale = w.bits(), _layout(w), 0.5
    norm = torch.full((1,), -1.0, device="cuda")
    m = master[:d] if with_master else None
    v = math.sqrt(float(np.dot(old_u, old_u)))
    if limit is None:
        lay.update(w.tensors, u, scale, master=m)
        factor = 1.0
    else:
        lay.update(w.tensors, u, scale, max_norm=limit, master=m, norm=norm)
        _near(norm, v, U * (1 + 1e-6))
        factor = limit / v if v > limit else 1.0
    at = 0
    for i, (x, p) in enumerate(zip(w.tensors, old)):
        n = sizes[i]
        if x is None:
            assert torch.equal(w.memory[i][0], memory[i])
            if with_master:
                assert np.array_equal(master[at:at + n].double().cpu().numpy(), old_master[at:at + n])
        elif n:
            step = scale * factor * old_u[at:at + n]
            want = (old_master[at:at + n] if with_master else p) - step
            # norm, factor and scale rounded once each; the fused result once
            fp32 = np.abs(step) * 3 * U * (1 + 1e-6) + np.abs(want) * U + 2.0 ** -149
            got = x.double().cpu().numpy()
            if with_master:
                now = master[at:at + n]
                assert (np.abs(now.double().cpu().numpy() - want) <= fp32).all()
                assert torch.equal(x, now.to(TYPES[types[i]]))
            else:
                assert (np.abs(got - want) <= fp32 + (np.abs(want) + fp32) * HALF_STEP[types[i]] + SMALLEST[types[i]]).all()
        at += n
    if with_master:
        assert np.array_equal(master[d:].double().cpu().numpy(), old_master[d:])
    assert w.around_is_untouched()
    assert np.array_equal(u.double().cpu().numpy(), old_u)


@pytest.mark.parametrize("t,value", [("f32", 1e-30), ("f32", 3e38), ("f32", 1e-45), ("bf16", 1e-30), ("bf16", 1e-22), ("bf16", 1e30), ("bf16", 3e38), ("bf16", 1e-40),
                                     ("f16", 65504.0), ("f16", 6e-8), ("bf16", 0.0), ("f32", 0.0), ("f16", 0.0)])
@pytest.mark.parametrize("shift", [0, 3])
def test_norms_of_extreme_values(t, value, shift):
    """Squares that fp32 cannot hold; a sum beyond fp32 is infinite."""
    n = 6001
    l = List([n], [t], [shift], like=True)
    l.tensors[0].fill_(value)
    x = float(l.tensors[0][0])
    want = x * math.sqrt(n)
    norm, lay = torch.full((1,), -1.0, device="cuda"), _layout(l)
    lay.norm(l.tensors, norm)
    if want > 3.4028235e38:
        assert norm.item() == math.inf
        before = l.bits()
        lay.clip(l.tensors, 1.0, norm=norm)
        assert norm.item() == math.inf and l.has_bits(before)
    else:
        assert abs(norm.item() - want) <= 5 * U * want + 2.0 ** -150
    lay.norm(l.tensors, norm, kind=_dr().NORM_MAX)
    assert norm.item() == x
    one = List([n], [t], [shift], like=True)                 # one such value among zeros
    one.tensors[0].zero_()[n // 2] = value
    lay.norm(one.tensors, norm)
    assert abs(norm.item() - x) <= 5 * U * x + 2.0 ** -150


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("kind", ["2", "max"])
@pytest.mark.parametrize("t", sorted(TYPES))
@pytest.mark.parametrize("at", [0, 5, 2500, -1])
@pytest.mark.parametrize("n", [5001, 700_001])
def test_a_norm_that_is_not_finite_bounds_nothing(t, kind, bad, at, n):
    sizes, types = [3, n, 64], [t] * 3
    l = List(sizes, types, [0, 1], seed=16)
    l.tensors[1][at] = bad
    before, lay, norm = l.bits(), _layout(l), torch.zeros(1, device="cuda")

    def as_told():
        got, want = norm.item(), math.nan if math.isnan(bad) else math.inf
        assert math.isnan(got) if math.isnan(want) else got == want

    lay.norm(l.tensors, norm, kind=_kind(kind))
    as_told()
    norm.zero_()
    lay.clip(l.tensors, 1e-3, norm=norm, kind=_kind(kind))
    as_told()
    assert l.has_bits(before)
    each = torch.zeros(3, device="cuda")
    lay.clip(l.tensors, 1e-3, each=each, separately=True, kind=_kind(kind))
    assert torch.equal(l.memory[1][0].view(torch.uint8), before[1].view(torch.uint8))
    assert not torch.equal(l.tensors[0], before[0][PAD:PAD + 3]) and math.isfinite(each[0].item()) and not math.isfinite(each[1].item())
    for x, (m, _, _) in zip(before, l.memory):
        m.copy_(x)
    row = torch.zeros(sum(sizes), device="cuda")
    norm.zero_()
    lay.pack(l.tensors, row, max_norm=1e-3, norm=norm, kind=_kind(kind))
    as_told()
    assert torch.equal(torch.nan_to_num(row, nan=5.0), torch.nan_to_num(torch.cat([x.float() for x in l.tensors]), nan=5.0))
    u = torch.zeros(sum(sizes), device="cuda")
    u[at] = bad
    master = torch.ones(sum(sizes), device="cuda")
    for m in (None, master):
        norm.zero_()
        lay.update(l.tensors, u, 1.0, max_norm=1.0, master=m, norm=norm, kind=_kind(kind))
        as_told()
        assert l.has_bits(before) and bool((master == 1.0).all())
    lay.update(l.tensors, u, 1.0, master=master, kind=_kind(kind))                     # not asked for the norm: applied as it is
    assert not bool(torch.isfinite(master).all())


def test_limits_at_their_ends():
    dr = _dr()
    l = List([4, 5], ["f32", "bf16"], like=True)
    l.tensors[0].copy_(torch.tensor([1.0, -2.0, 2.0, 0.0]))
    l.tensors[1].copy_(torch.tensor([4.0, 0.0, 0.0, 0.0, 0.0]))                        # the norm is 5
    lay, norm, start = _layout(l), torch.zeros(1, device="cuda"), l.bits()
    lay.clip(l.tensors, 5.0, norm=norm)
    assert norm.item() == 5.0 and l.has_bits(start)
    lay.clip(l.tensors, math.inf, norm=norm)
    assert norm.item() == 5.0 and l.has_bits(start)
    lay.clip(l.tensors, 1.25)
    assert l.tensors[0].tolist() == [0.25, -0.5, 0.5, 0.0] and l.tensors[1].tolist() == [1.0, 0.0, 0.0, 0.0, 0.0]
    lay.clip(l.tensors, 0.5, kind=dr.NORM_MAX, norm=norm)
    assert norm.item() == 1.0 and l.tensors[0].tolist() == [0.125, -0.25, 0.25, 0.0]
    lay.clip(l.tensors, 0.0, norm=norm)
    assert norm.item() == float(np.float32(math.sqrt(0.25 + 0.140625))) and not l.tensors[0].any() and not l.tensors[1].any()
    lay.clip(l.tensors, 0.0, norm=norm)
    assert norm.item() == 0.0


def test_tensors_in_other_orders_of_their_dimensions():
    """Norms and clipping go by memory, whatever the order of the dimensions."""
    dr = _dr()
    x = torch.randn(8, 5, 7, 3, device="cuda").to(memory_format=torch.channels_last)
    y = torch.randn(33, 65, device="cuda").t()
    lay, norm = dr.Layout.of([x, y]), torch.zeros(1, device="cuda")
    want = math.sqrt(float(x.double().square().sum() + y.double().square().sum()))
    lay.norm([x, y], norm)
    _near(norm, want, 1.01 * U)
    out = [torch.empty_like(x), torch.empty_like(y)]
    lay.clip([x, y], 1.0, out=out)
    for a, b in zip((x, y), out):
        _scaled_ok(b.double().cpu().numpy(), a.double().cpu().numpy(), 1.0 / want, "f32", 2.01 * U)
    with pytest.raises(dr.DracoError, match="strides"):
        lay.clip([x, y], 1.0, out=[torch.empty_like(x), torch.empty(y.shape, device="cuda")])
    with pytest.raises(dr.DracoError, match="contiguous"):
        lay.pack([x, y], torch.empty(lay.d, device="cuda"))


def test_refusals():
    dr = _dr()
    from paper_1803_09877_b200 import binding
    l = List([10, 20, 30], ["f32", "bf16", "f16"], like=True)
    a, b, c = l.tensors
    lay, norm, row = _layout(l), torch.zeros(1, device="cuda"), torch.zeros(60, device="cuda")
    before = l.bits()

    def refused(call, match):
        with pytest.raises(dr.DracoError, match=match):
            call()

    refused(lambda: lay.norm([a, b], norm), "2 tensors, not 3")
    refused(lambda: lay.norm([a, b, c[:-1]], norm), "not 30")
    refused(lambda: lay.norm([a, c[:20], c], norm), "float16, not 20 of type 1")
    refused(lambda: lay.norm([a.cpu(), b, c], norm), "is on cpu")
    refused(lambda: lay.norm([torch.zeros(20, device="cuda")[::2], b, c], norm), "not dense")
    refused(lambda: lay.norm([torch.zeros(10, dtype=torch.complex64, device="cuda").conj().imag, b, c], norm), "not dense")
    refused(lambda: lay.norm([torch._neg_view(a), b, c], norm), "negated")
    refused(lambda: lay.norm([a, b, c], None), "invalid argument")
    refused(lambda: lay.norm([a, b, c], torch.zeros(1, dtype=torch.float64, device="cuda")), "norm")
    refused(lambda: lay.norm([a, b, c], norm, each=torch.zeros(2, device="cuda")), "each")
    refused(lambda: lay.norm([a, b, c], norm, kind=2), "invalid argument")
    refused(lambda: lay.norm([a.data_ptr() + 2, b, c], norm), "invalid argument")       # not on its element's boundary
    refused(lambda: lay.norm([a, b.data_ptr() + 1, c], norm), "invalid argument")
    for limit in (-1.0, math.nan, -math.inf):
        refused(lambda: lay.clip([a, b, c], limit), "invalid argument")
        refused(lambda: lay.pack([a, b, c], row, max_norm=limit), "invalid argument")
        refused(lambda: lay.update([a, b, c], row, 1.0, max_norm=limit), "invalid argument")
    refused(lambda: lay.clip([a, b, c], 1.0, each=torch.zeros(3, device="cuda")), "invalid argument")
    refused(lambda: lay.clip([a, b, c], 1.0, out=[a, None, c]), "invalid argument")
    refused(lambda: lay.clip([a, None, c], 1.0, out=[a, b, c]), "invalid argument")
    refused(lambda: lay.update([a, b, c], row, math.nan), "invalid argument")
    refused(lambda: lay.update([a, b, c], None, 1.0), "invalid argument")
    refused(lambda: lay.update([a, b, c], row[:-1], 1.0), "not 60")
    refused(lambda: lay.update([a, b, c], torch.zeros(61, device="cuda")[1:], 1.0), "invalid argument")      # 16-byte alignment
    refused(lambda: lay.update([a, b, c], row, 1.0, master=row), "invalid argument")
    refused(lambda: lay.update([row[50:], b, c], row, 1.0), "invalid argument")
    refused(lambda: lay.update([row[50:], b, c], torch.zeros(60, device="cuda"), 1.0, master=row), "invalid argument")
    refused(lambda: lay.pack([a, b, c], None), "invalid argument")
    refused(lambda: lay.pack([row[:10], b, c], row), "invalid argument")
    refused(lambda: lay.pack([a, b, c], torch.zeros(60, device="cuda", dtype=torch.float16)), "row")
    # the same tensor twice: read twice, written never
    same = dr.Layout([10, 10, 0, 0], dr.F32)
    other, empty = torch.zeros(10, device="cuda"), torch.zeros(0, device="cuda")
    refused(lambda: same.clip([a, a, empty, empty], 1.0), "invalid argument")
    refused(lambda: same.clip([a, other, empty, empty], 1.0, out=[other, a, empty, empty]), "invalid argument")
    refused(lambda: same.clip([a, a, empty, empty], 1.0, out=[other, other, empty, empty]), "invalid argument")
    refused(lambda: same.update([a, a, empty, empty], torch.zeros(20, device="cuda"), 1.0), "invalid argument")
    a.fill_(1.0)
    same.norm([a, a, empty, empty], norm)
    assert norm.item() == float(np.float32(math.sqrt(20.0)))
    a.copy_(before[0][PAD:PAD + 10])
    assert l.has_bits(before)
    assert binding.lib.draco_strerror(binding.ELIMIT).startswith(b"size exceeds")
    lay.close()
    refused(lambda: lay.norm([a, b, c], norm), "invalid argument")


def test_some_outputs_in_place():
    """An output may be its own input, the others elsewhere."""
    for sizes in ([100, 37, 2000], [400_000, 37, 300_001]):
        l = List(sizes, ["f32", "bf16", "f16"], [1], seed=91)
        out = List(sizes, ["f32", "bf16", "f16"], [2], like=l)
        parts, lay = l.wide(), _layout(l)
        v = _norm64(parts, "2")
        targets = [l.tensors[0], out.tensors[1], l.tensors[2]]
        untouched = out.bits()
        lay.clip(l.tensors, 0.5, out=targets)
        for x, p, t in zip(targets, parts, l.types):
            _scaled_ok(x.double().cpu().numpy(), p, 0.5 / v, t, l.norm_tolerance + U)
        assert np.array_equal(l.tensors[1].double().cpu().numpy(), parts[1]) and l.around_is_untouched() and out.around_is_untouched()
        assert torch.equal(out.memory[0][0], untouched[0]) and torch.equal(out.memory[2][0], untouched[2])


def test_as_many_tensors_as_there_may_be():
    dr = _dr()
    from paper_1803_09877_b200 import binding
    n = binding.MAX_TENSORS
    x = torch.ones(n, device="cuda")
    lay, address = dr.Layout([1] * n, dr.F32), x.data_ptr()
    addresses = [address + 4 * i for i in range(n)]
    norm, row = torch.zeros(1, device="cuda"), torch.zeros(n, device="cuda")
    lay.norm(addresses, norm)
    assert norm.item() == math.sqrt(n)
    lay.clip(addresses, math.sqrt(n) / 4)
    lay.pack(addresses, row)
    assert bool((row == 0.25).all())
    lay.update(addresses, row, 2.0)
    assert bool((x == -0.25).all())


def test_two_lists_on_two_streams():
    """Layouts have scratch of their own: calls on two of them may overlap."""
    dr = _dr()
    lists = [List([200_000, 31, 5000], ["bf16", "f32", "f16"], seed=20 + k) for k in range(2)]
    lays, streams = [_layout(l) for l in lists], [torch.cuda.Stream() for _ in lists]
    norms, rows = torch.zeros(2, 1, device="cuda"), torch.zeros(2, 205_032, device="cuda")
    torch.cuda.synchronize()
    for _ in range(20):
        for l, lay, st, n, r in zip(lists, lays, streams, norms, rows):
            lay.pack(l.tensors, r[:lay.d], max_norm=1.0, norm=n, stream=st)
            lay.norm(l.tensors, n, stream=st)
    torch.cuda.synchronize()
    for l, n, r, lay in zip(lists, norms, rows, lays):
        v = _norm64(l.wide(), "2")
        _near(n, v, l.norm_tolerance)
        _scaled_ok(r[:lay.d].double().cpu().numpy(), np.concatenate(l.wide()), 1.0 / v, "f32", 6 * U)


@pytest.mark.parametrize("n", [40, 4_000_000])
def test_a_layouts_first_calls_captured(n):
    """Nothing that a call needs is made, loaded or allocated by an earlier one."""
    code = f"""
import torch, paper_1803_09877_b200 as dr
x, w = torch.full(({n},), 3.0, device="cuda"), torch.zeros({n}, device="cuda", dtype=torch.bfloat16)
row, norm, each, g = torch.zeros({n}, device="cuda"), torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda"), torch.cuda.CUDAGraph()
lx, lw = dr.Layout([{n}], dr.F32), dr.Layout.of([w])
with torch.cuda.graph(g):
    lx.norm([x], norm, each=each)
    lx.pack([x], row, max_norm=1.0)
    lw.update([w], row, 1.0, max_norm=0.5)
    lx.clip([x], 2.0, out=[row])
g.replay()
torch.cuda.synchronize()
n = {n} ** 0.5
assert abs(norm.item() - 3 * n) < 1e-6 * n and each.item() == norm.item()
assert abs(w[7].item() + 0.5 / n) < 0.01 / n and abs(row[5].item() - 2 / n) < 1e-6 / n
"""
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", code], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr


def test_native_and_python_lists_are_the_same(monkeypatch):
    """The natively listed addresses, those that binding.py lists, and torch's own function in the place of the built one."""
    dr = _dr()
    from paper_1803_09877_b200 import binding
    l = List([1000, 7, 0, 64], ["bf16", "f32", "f16", "f32"], [0, 3], seed=81, absent={3})
    lay, results = _layout(l), []
    tensors = [torch.nn.Parameter(l.tensors[0]), l.tensors[1], l.tensors[2], None]

    def run(kind=list):
        norm, row, each = torch.zeros(1, device="cuda"), torch.full((1071,), 5.0, device="cuda"), torch.zeros(4, device="cuda")
        lay.norm(kind(tensors), norm, each=each)
        lay.pack(kind(tensors), row, max_norm=0.5)
        out = List(l.sizes, l.types, [0, 3], like=l, absent={3})
        lay.clip(tensors, 0.25, out=out.tensors)
        results.append([norm, row, each] + out.tensors[:3])

    run()
    run(tuple)
    run(iter)
    run(lambda ts: [None if t is None else t.data_ptr() for t in ts])
    own = getattr(torch.Tensor, "__dlpack_c_exchange_api__", None)
    if own is not None and binding._native is not binding._CtypesCalls:
        binding._native.set_exchange(torch.Tensor, torch.nn.Parameter, own)
        run()
        binding._native.set_exchange(torch.Tensor, torch.nn.Parameter, binding._exchange(torch))
    monkeypatch.setattr(binding, "_native", binding._CtypesCalls)
    run()
    for other in results[1:]:
        for a, b in zip(results[0], other):
            assert torch.equal(a, b)


def test_a_captured_step_on_new_values():
    """Clip, pack and update captured together; replays work on what the tensors then hold, and eager calls go on in between."""
    sizes, types = [30_000, 10, 4097, 1], ["bf16", "f32", "f16", "f32"]
    l, w = List(sizes, types, [0, 3], seed=31), List(sizes, types, [1, 0], seed=32)
    lay, side = _layout(l), torch.cuda.Stream()
    d = sum(sizes)
    row, master, norms = torch.zeros(d, device="cuda"), torch.zeros(d, device="cuda"), torch.zeros(3, 1, device="cuda")
    each = torch.zeros(4, device="cuda")

    def step():
        lay.norm(l.tensors, norms[0], each=each)
        lay.clip(l.tensors, 0.5, separately=True)
        lay.norm(l.tensors, norms[1])
        lay.pack(l.tensors, row, max_norm=0.25, norm=norms[2])
        lay.update(w.tensors, row, 0.5, max_norm=0.125, master=master)

    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        step()
    fresh = [List(sizes, types, [0, 3], seed=40 + k) for k in range(3)]
    for f in fresh:
        for a, b in zip(l.tensors, f.tensors):
            a.copy_(b)
        master.fill_(0.5)
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in [row, master, norms, each] + l.tensors + w.tensors]
        for a, b in zip(l.tensors, f.tensors):
            a.copy_(b)
        master.fill_(0.5)
        step()
        torch.cuda.synchronize()
        for x, y in zip(got, [row, master, norms, each] + l.tensors + w.tensors):
            assert torch.equal(x, y)
        assert float(row.norm()) == pytest.approx(0.25, rel=1e-2)


@pytest.mark.parametrize("shifts", ["aligned", "all"])
@pytest.mark.parametrize("types", [["bf16", "f32", "f16", "bf16"], ["f32"] * 4, ["bf16"] * 4])
def test_long_lists(types, shifts):
    """Long enough for second passes in several waves of blocks."""
    sizes = [23_000_001, 17, 12_000_000, 14_000_002]
    l = List(sizes, types, SHIFTS[shifts], seed=71)
    lay, d = _layout(l), sum(sizes)
    parts = [x.double() for x in l.tensors]
    v = math.sqrt(float(sum(torch.dot(p, p) for p in parts)))
    norm, row = torch.zeros(1, device="cuda"), torch.full((d + 3,), SENTINEL, device="cuda")
    off = l.norm_tolerance + U

    def near(got, want, t, off):
        bound = want.abs() * ((1 + off) * (1 + U) * (1 + HALF_STEP[t]) - 1 if t != "f32" else off + U + off * U) * (1 + 1e-9) + SMALLEST[t] + 2.0 ** -150
        assert bool(((got.double() - want).abs() <= bound).all())

    lay.pack(l.tensors, row[1:d + 1], max_norm=1.0, norm=norm)
    _near(norm, v, l.norm_tolerance)
    near(row[1:d + 1], torch.cat(parts) / v, "f32", off)
    assert row[0].item() == SENTINEL and bool((row[d + 1:] == SENTINEL).all())
    out = List(sizes, types, SHIFTS["three"], like=l)
    lay.clip(l.tensors, 1.0, out=out.tensors)
    for x, p, t in zip(out.tensors, parts, types):
        near(x, p / v, t, off)
    assert out.around_is_untouched()
    lay.clip(l.tensors, 1.0)
    for x, p, t in zip(l.tensors, parts, types):
        near(x, p / v, t, off)
    assert l.around_is_untouched()
    u = row[:d].clone()
    u[0] = 0.0
    r = float(u.double().square().sum().sqrt())
    for master in (None, torch.randn(d, device="cuda")):
        old = [x.double() for x in l.tensors] if master is None else list(master.double().split(sizes))
        lay.update(l.tensors, u, 2.0, max_norm=0.5, master=master, norm=norm)
        _near(norm, r, U * (1 + 1e-6))
        for x, o, step, t in zip(l.tensors, old, u.double().split(sizes), types):
            step = step * (2.0 * 0.5 / r)
            fp32 = step.abs() * 3 * U * (1 + 1e-6) + (o - step).abs() * U + 2.0 ** -149
            assert bool(((x.double() - (o - step)).abs() <= fp32 + ((o - step).abs() + fp32) * HALF_STEP[t] + SMALLEST[t]).all())
        if master is not None:
            assert torch.equal(torch.cat([x.float() for x in l.tensors]), torch.cat([m.to(TYPES[t]).float() for m, t in zip(master.split(sizes), types)]))
    assert l.around_is_untouched()


def test_offsets_beyond_32_bits():
    dr = _dr()
    sizes = [2_200_000_001, 13, 2_200_000_003]
    lay = dr.Layout(sizes, dr.BF16)
    memory = torch.full((sum(sizes) + 64,), 0.0, dtype=torch.bfloat16, device="cuda")
    tensors, at = [], 0
    for n in sizes:
        tensors.append(memory[at:at + n])
        at += n
    marks = [0, 1, 2_147_483_648, 2_200_000_000, 2_200_000_001, 2_200_000_013, 2_200_000_014, 4_294_967_296, 4_294_967_301, sum(sizes) - 1]
    memory[marks] = 2.0
    norm, row = torch.zeros(1, device="cuda"), torch.empty(lay.d, device="cuda")
    lay.pack(tensors, row, max_norm=math.sqrt(10.0), norm=norm)
    assert norm.item() == float(np.float32(math.sqrt(40.0)))
    assert int(row.count_nonzero()) == len(marks) and float((row[marks] - 1.0).abs().max()) <= 4 * U
    row.zero_()[marks] = 1.0
    lay.update(tensors, row, 1.0, max_norm=math.sqrt(2.5))
    assert float((memory[marks].float() - 1.5).abs().max()) == 0.0 and int(memory.count_nonzero()) == len(marks)
    lay.clip(tensors, math.sqrt(2.5), norm=norm)
    assert norm.item() == pytest.approx(math.sqrt(22.5), rel=1e-6)
    assert float((memory[marks].float() - 0.5).abs().max()) <= 0.5 * 2.0 ** -8 and int(memory.count_nonzero()) == len(marks)


@pytest.mark.parametrize("code", ["REP", "CYC", "CYC_PACKED"])
def test_an_iteration_from_gradient_tensors_to_weights(code):
    """n workers' gradient lists packed into the rows of G, clipped each by its own norm; encoded, attacked, located and decoded; the sum,
    bounded, taken off a list of bf16 weights by way of their fp32 copy.  Odd d: rows of G start off the 16-byte grid."""
    dr = _dr()
    n, s = 15, 2
    sizes = [5000, 31, 12_000, 1, 257]
    types = ["bf16", "f32", "bf16", "f32", "f16"]
    d = sum(sizes)
    assert d % 4
    workers = [List(sizes, types, [0], seed=60 + k, absent={3} if k == 4 else ()) for k in range(n)]
    weights = List(sizes, ["bf16"] * 5, [0], seed=59)
    lay, wlay = _layout(workers[0]), _layout(weights)
    G, norms = torch.empty((n, d), device="cuda"), torch.empty((n, 1), device="cuda")
    for k, l in enumerate(workers):
        lay.pack(l.tensors, G[k], max_norm=1.0, norm=norms[k])
    rows = []
    for k, l in enumerate(workers):
        parts = l.wide()
        v = _norm64(parts, "2")
        _near(norms[k], v, l.norm_tolerance)
        assert v > 1.0
        rows.append(np.concatenate(parts) / v)
    exact = np.sum(rows, axis=0)
    cyc, vlen = code != "REP", (d + 1) // 2 if code == "CYC_PACKED" else d
    plan = dr.Plan(n, s, d, getattr(dr, code))
    Z = torch.empty((n, 2 * vlen if cyc else d), device="cuda")
    adv = di.choose_adversaries(61, n, s)
    f = torch.from_numpy(di.projection_vector(62, vlen)).cuda() if cyc else None
    flags, u = torch.empty(n, dtype=torch.uint8, device="cuda"), torch.empty(d, device="cuda")
    plan.encode(G, Z)
    plan.corrupt(Z, adv, [dr.ADV_REVGRAD] * s, [100.0] * s, seed=63)
    plan.locate_decode(Z, f, flags, u)
    assert sorted(np.flatnonzero(flags.cpu().numpy())) == adv.tolist()
    master = torch.cat([x.float() for x in weights.tensors])
    old = master.double().cpu().numpy()
    norm = torch.zeros(1, device="cuda")
    wlay.update(weights.tensors, u, 0.5, max_norm=1.0, master=master, norm=norm)
    v = math.sqrt(float(np.dot(exact, exact)))
    # the code's own accuracy at n = 15, s = 2 with complex64 vectors is 1e-4 of the largest entry
    err = 1e-4 * np.abs(exact).max()
    assert abs(norm.item() - v) <= math.sqrt(d) * err
    want = old - 0.5 * min(1.0, 1.0 / v) * exact
    assert np.abs(master.double().cpu().numpy() - want).max() <= err + 0.5 * math.sqrt(d) * err / v * np.abs(exact).max() + 1e-6
    assert torch.equal(torch.cat(weights.tensors), master.bfloat16())
    assert all(l.around_is_untouched() for l in workers) and weights.around_is_untouched()


def _exchanges():
    """The ways to read a list's tensors: the built module, torch's own function, and ctypes, by name; the usual one last."""
    from paper_1803_09877_b200 import binding
    native, usual = binding._native, binding._exchange(torch)
    own = getattr(torch.Tensor, "__dlpack_c_exchange_api__", None)

    def put(calls, exchange):
        binding._native = calls
        if calls is not binding._CtypesCalls and exchange is not None:
            calls.set_exchange(torch.Tensor, torch.nn.Parameter, exchange)

    yield "ctypes", lambda: put(binding._CtypesCalls, None)
    yield "torch's own", lambda: put(native, own)
    yield "usual", lambda: put(native, usual)


def test_negated_views_are_refused_by_every_exchange():
    dr = _dr()
    x, other = torch.ones(4, device="cuda"), torch.zeros(4, device="cuda")
    negated, part = torch._neg_view(x), torch.ones(1, dtype=torch.complex64, device="cuda").conj().imag
    lay, one, norm = dr.Layout.of([x]), dr.Layout([1], dr.F32), torch.zeros(1, device="cuda")
    for name, put in _exchanges():
        put()
        try:
            for l, v in ((lay, negated), (one, part)):
                row = other[:l.d]
                for call in (lambda: l.norm([v], norm), lambda: l.clip([v], 0.5), lambda: l.clip([v], 0.5, out=[row]), lambda: l.pack([v], row),
                             lambda: l.update([v], row, 1.0), lambda: l.pack([row], v), lambda: l.update([row], v, 1.0)):
                    with pytest.raises(dr.DracoError, match="negated"):
                        call()
        finally:
            for _, back in _exchanges():
                pass
            back()
    assert bool((x == 1.0).all()) and not other.any() and not norm.any()


def test_writes_to_a_lazy_clone_leave_its_source():
    dr = _dr()
    for name, put in _exchanges():
        put()
        try:
            for write in ("clip", "out", "row", "param", "master"):
                x, y = torch.full((1000,), 3.0, device="cuda"), torch.full((1000,), 3.0, device="cuda")
                clone, lay = torch._lazy_clone(x), dr.Layout.of([x])
                if write == "clip":
                    lay.clip([clone], 1.0)
                elif write == "out":
                    lay.clip([y], 1.0, out=[clone])
                elif write == "row":
                    lay.pack([y], clone, max_norm=1.0)
                elif write == "param":
                    lay.update([clone], y, 0.5)
                else:
                    lay.update([y.clone()], y, 0.5, master=clone)
                assert bool((x == 3.0).all()) and bool((y == 3.0).all()) and not bool((clone == 3.0).any()), (name, write)
        finally:
            for _, back in _exchanges():
                pass
            back()


@pytest.mark.parametrize("kind", ["2", "max"])
@pytest.mark.parametrize("types", [["bf16"], ["f16"], ["f32"], ["bf16", "f32", "f16"]])
@pytest.mark.parametrize("sizes", [[1], [7], [8], [9], [15], [16], [17], [100], [257], [1000, 33, 511], [2047, 2048, 2049], [4096, 4097, 12_345], [100_003, 5],
                                   [37 * (i % 9) + i for i in range(120)], [400_003, 1, 70_001], [257 + 64 * (i % 3) for i in range(600)], [3_000_017, 999]])
def test_results_do_not_depend_on_where_the_tensors_lie(sizes, types, kind):
    """The same values at other offsets from the 16-byte grid: the same bits, so that equal gradients make equal rows, whoever packs them."""
    types = (types * len(sizes))[:len(sizes)]
    l = List(sizes, types, [0], seed=92, sigma=1.0)
    lay, d = _layout(l), sum(sizes)
    limit = 0.37 * _norm64(l.wide(), kind)
    want = None
    for shifts in ([0], [1], [2], [3], [4], [5], [6], [7], [0, 1, 2, 3, 4, 5, 6, 7], [7, 4, 2]):
        at = List(sizes, types, shifts, like=l)
        for x, y in zip(at.tensors, l.tensors):
            x.copy_(y)
        norms, each = torch.zeros(3, 1, device="cuda"), torch.zeros(2, len(sizes), device="cuda")
        row = torch.zeros(d + 3, device="cuda")[shifts[0] % 4:][:d]
        lay.norm(at.tensors, norms[0], kind=_kind(kind))
        lay.norm(at.tensors, norms[1], each=each[0], kind=_kind(kind))
        lay.pack(at.tensors, row, max_norm=limit, norm=norms[2], kind=_kind(kind))
        got = [norms, each, row]
        for separately in (False, True):
            out = List(sizes, types, shifts[::-1], like=l)
            lay.clip(at.tensors, limit / (2 if separately else 1), out=out.tensors, separately=separately, kind=_kind(kind))
            got += out.tensors
        lay.clip(at.tensors, limit, each=each[1], separately=True, kind=_kind(kind))
        got = [x.clone() for x in got + at.tensors]
        want = want or got
        for x, y in zip(got, want):
            assert torch.equal(x, y), shifts


def test_replicas_of_a_group_that_pack_their_own_copies_agree():
    """The repetition code's vote compares bits: honest members whose gradients lie elsewhere in memory are no disagreement."""
    dr = _dr()
    n, s, sizes, types = 9, 1, [700, 31, 1000, 257], ["bf16", "f16", "bf16", "f32"]
    d = sum(sizes)
    plan, lay = dr.Plan(n, s, d, dr.REP), dr.Layout(sizes, [TYPES[t] for t in types])
    flags, u = torch.empty(n, dtype=torch.uint8, device="cuda"), torch.empty(d, device="cuda")
    for seed in range(40):
        l = List(sizes, types, [0], seed=200 + seed, sigma=1.0)
        R = torch.empty((n, d), device="cuda")
        for k in range(n):
            mine = List(sizes, types, [k % 8, 3, (2 * k + 1) % 8], like=l)
            for x, y in zip(mine.tensors, l.tensors):
                x.copy_(y)
            lay.pack(mine.tensors, R[k], max_norm=1.0)
        assert all(torch.equal(R[0], R[k]) for k in range(n))
        plan.locate_decode(R, None, flags, u)
        assert not flags.any() and plan.info()["no_majority"] == 0


@pytest.mark.parametrize("kind", ["2", "max"])
def test_an_error_of_another_call_is_not_taken_for_a_launch_of_this_one(kind):
    """A list of several launches: refused after the first of them, its layout would count blocks wrongly from then on."""
    import ctypes
    from paper_1803_09877_b200 import binding
    runtime = ctypes.CDLL("libcudart.so.12")
    sizes = [1 + i % 900 for i in range(4500)]
    l = List(sizes, ["bf16", "f32", "f16"] * 1500, [0, 1], seed=93)
    lay, d = _layout(l), sum(sizes)
    v, norm, row = _norm64(l.wide(), kind), torch.zeros(3, 1, device="cuda"), torch.zeros(d, device="cuda")
    torch.cuda.synchronize()
    stream = torch.cuda.current_stream().cuda_stream
    binding._current_stream()
    assert runtime.cudaSetDevice(9999) != 0                # an error that nobody has looked at yet
    lay.norm(l.tensors, norm[0], kind=_kind(kind), stream=stream)
    lay.pack(l.tensors, row, max_norm=v / 2, norm=norm[1], kind=_kind(kind), stream=stream)
    left = runtime.cudaGetLastError()
    lay.norm(l.tensors, norm[2], kind=_kind(kind))
    assert left != 0                                       # and is still there for whoever asks
    tol = 0.0 if kind == "max" else l.norm_tolerance
    for n in norm:
        _near(n, v, tol)
    _scaled_ok(row.double().cpu().numpy(), np.concatenate(l.wide()), 0.5, "f32", tol + U)


@pytest.mark.parametrize("call", ["norm", "pack", "clip", "clip separately", "update"])
def test_two_threads_with_one_layout_on_one_stream(call):
    """A call's launches stay together: between a measurement and what is scaled by it another thread's measurement would be that of another list."""
    import threading
    sizes, types, times = [150_000, 31, 40_000], ["bf16", "f32", "f32"], 150
    lists = [List(sizes, types, [0], seed=94 + k, sigma=0.1 * 5 ** k) for k in range(2)]
    lay, d, stream = _layout(lists[0]), sum(sizes), torch.cuda.Stream()
    flat = [torch.cat([x.float() for x in l.tensors]) for l in lists]
    norms, each = torch.zeros(2, times + 1, 1, device="cuda"), torch.zeros(2, times + 1, 3, device="cuda")
    rows = torch.zeros(2, times + 1, d, device="cuda")
    outs = [[List(sizes, types, [0], like=l).tensors for _ in range(times + 1)] for l in lists]

    def go(k, i):
        norm = norms[k, i]
        if call == "norm":
            lay.norm(lists[k].tensors, norm, each=each[k, i], stream=stream)
        elif call == "pack":
            lay.pack(lists[k].tensors, rows[k, i], max_norm=1.0, norm=norm, stream=stream)
        elif call == "update":
            lay.update(outs[k][i], flat[k], 0.5, max_norm=1.0, norm=norm, stream=stream)
        else:
            lay.clip(lists[k].tensors, 1.0, out=outs[k][i], norm=norm, separately="separately" in call, stream=stream)

    torch.cuda.synchronize()
    for k in range(2):
        go(k, times)                                       # one after the other
    torch.cuda.synchronize()
    threads = [threading.Thread(target=lambda k=k: [go(k, i) for i in range(times)]) for k in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    for k in range(2):
        assert norms[k, times].item() > 1.0
        for x in (norms[k], each[k], rows[k]):
            assert bool((x == x[times]).all())
        for i in range(times):
            assert all(torch.equal(a, b) for a, b in zip(outs[k][i], outs[k][times]))


def test_autograd_is_told_of_what_a_call_writes():
    dr = _dr()
    for name, put in _exchanges():
        put()
        try:
            x, w = torch.nn.Parameter(torch.full((100,), 3.0, device="cuda")), torch.nn.Parameter(torch.full((50,), 2.0, device="cuda", dtype=torch.bfloat16))
            lay = dr.Layout.of([x, w])
            vectors = {"out0": torch.zeros(100, device="cuda"), "out1": torch.zeros(50, device="cuda", dtype=torch.bfloat16), "row": torch.zeros(150, device="cuda"),
                       "u": torch.ones(150, device="cuda"), "master": torch.ones(150, device="cuda"), "norm": torch.zeros(1, device="cuda"),
                       "each": torch.zeros(2, device="cuda"), "x": x, "w": w}
            v = vectors
            calls = [(lambda: lay.norm([x, w], v["norm"], each=v["each"]), "norm each"),
                     (lambda: lay.clip([x, w], 1.0, out=[v["out0"], v["out1"]], norm=v["norm"]), "out0 out1 norm"),
                     (lambda: lay.clip((x, w), 1.0, each=v["each"], separately=True), "x w each"),
                     (lambda: lay.pack([x, w], v["row"], norm=v["norm"]), "row norm"),
                     (lambda: lay.update([x, None], v["u"], 0.5, norm=v["norm"]), "x norm"),
                     (lambda: lay.update(iter([x, w]), v["u"], 0.5, master=v["master"]), "x w master")]
            for call, written in calls:
                before = {k: t._version for k, t in vectors.items()}
                call()
                for k, t in vectors.items():
                    assert (t._version > before[k]) == (k in written.split()), (name, written, k)
            loss = (x * x).sum() + (w.float() * w.float()).sum()
            lay.update([x, w], v["u"], 0.5)
            with pytest.raises(RuntimeError, match="modified by an inplace operation"):
                loss.backward()
            before = x._version
            with pytest.raises(dr.DracoError):                 # refused: not written
                lay.update([x, w], v["u"], math.nan)
            assert x._version == before
            with torch.inference_mode():
                i = torch.full((100,), 3.0, device="cuda")
            lay.clip([i, None], 3.0)                           # has no version
            assert float(i.norm()) == pytest.approx(3.0, rel=1e-5)
        finally:
            for _, back in _exchanges():
                pass
            back()


@pytest.mark.parametrize("sizes", [[100] * 2000 + [20_000_001, 17, 12_000_000], [20_000_001, 17, 12_000_000] + [100] * 2000, [64 + i % 5 for i in range(20_000)]])
@pytest.mark.parametrize("kind", ["2", "max"])
def test_lists_of_several_launches_of_unequal_length(sizes, kind):
    """A short first launch before a long second one, the other way round, and many launches of short tensors: one factor for all of them."""
    dr = _dr()
    d = sum(sizes)
    g = torch.Generator(device="cuda").manual_seed(95)
    memory = torch.empty(d, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    tensors, wide = list(memory.split(sizes)), memory.double()
    v = float(wide.square().sum().sqrt()) if kind == "2" else float(wide.abs().max())
    lay, norm, row = dr.Layout(sizes, dr.BF16), torch.zeros(1, device="cuda"), torch.zeros(d, device="cuda")
    tol = 0.0 if kind == "max" else 5 * U * (1 + 1e-6)

    def near(got, want, t):
        rel = (1 + tol + U) * (1 + U) * (1 + (HALF_STEP[t] if t != "f32" else 0.0)) - 1
        assert bool(((got.double() - want).abs() <= want.abs() * rel * (1 + 1e-9) + SMALLEST[t]).all())

    lay.pack(tensors, row, max_norm=v / 2, norm=norm, kind=_kind(kind))
    _near(norm, v, tol)
    near(row, wide * 0.5, "f32")
    norm.zero_()
    lay.update(tensors, row, 0.0, max_norm=v / 4, norm=norm, kind=_kind(kind))
    assert torch.equal(memory.double(), wide) and abs(norm.item() - v / 2) <= 1e-6 * v
    lay.clip(tensors, v / 2, norm=norm, kind=_kind(kind))
    _near(norm, v, tol)
    near(memory, wide * 0.5, "bf16")
