"""Performance cases of the operators on lists of tensors: what stands between a model's many gradient tensors and the flat fp32 vectors
that the code works on.

    norm     the global norm of a list of gradients, or the norm of each of them
    clip     the same, and every gradient scaled by min(1, max_norm / norm), all by the global norm or each by its own
    pack     a list of gradients of any type -> the fp32 row of G that ``Plan.encode`` reads, clipped on the way
    update   the decoded sum u -> w <- w - scale * min(1, max_norm / |u|) * u for a list of parameters, with or without an fp32 master copy

A norm is the 2-norm or the largest magnitude.  Where it is not finite, clip and pack leave the values as they are and update leaves the
weights.  A gradient may be absent (None): it adds nothing to the norm, its part of a packed row is zero.

The tensors of one type lie in one buffer, as the buckets of a data-parallel program hold them: ``tight`` back to back, so that most start
off the 16-byte grid, or else each on a multiple of 16 bytes.
"""
import math
import random

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
MAX_BYTES = 2.1e9           # of a drawn case: the largest listed one
INF = float("inf")
UPDATE_SCALE = 0.25


def listed():
    return [
        # the gradients of a small convolutional text model (154 k parameters), logged every iteration: latency is all there is
        dict(name="norm_f32_154k", op="norm", kind="2", each=False, types="f32", count=8, total=154_000, tight=False, absent=0, limit=INF),
        # a network of 60.2 M parameters in 465 tensors, half of them vectors of normalisation layers
        dict(name="norm_bf16_60.2M", op="norm", kind="2", each=False, types="bf16", count=465, total=60_200_000, tight=False, absent=0, limit=INF),
        # what 45 workers computed, one norm a worker: rows of G
        dict(name="norm_rows_n45_11.7M", op="norm", kind="2", each=True, types="f32", count=-45, total=45 * 11_700_000, tight=True, absent=0, limit=INF),
        # a small model's gradients, always above the limit
        dict(name="clip_f32_100k", op="clip", kind="2", each=False, types="f32", count=6, total=100_000, tight=False, absent=0, limit=1.0),
        # 62 tensors of three types with sizes as they come, a few of them without a gradient
        dict(name="clip_mixed_11.7M", op="clip", kind="2", each=False, types="mixed", count=62, total=11_700_000, tight=True, absent=9, limit=0.25),
        # an ordinary iteration of a trained network: the norm is below the limit, and the gradients stay
        dict(name="clip_below_bf16_60.2M", op="clip", kind="2", each=False, types="bf16", count=465, total=60_200_000, tight=False, absent=0, limit=1e6),
        # every worker's row bounded by itself before the encoder reads G; rows off the 16-byte grid
        dict(name="clip_rows_n15_1M", op="clip", kind="2", each=True, types="f32", count=-15, total=15 * 1_000_003, tight=True, absent=0, limit=1.0),
        # one worker's half-precision gradients into its row of G; 431 k parameters, sizes as they come, by the largest magnitude
        dict(name="pack_f16_431k", op="pack", kind="max", each=False, types="f16", count=10, total=431_080, tight=True, absent=4, limit=0.0078125),
        # the largest model: 138 M parameters in a few tensors
        dict(name="pack_bf16_138M", op="pack", kind="2", each=False, types="bf16", count=38, total=138_000_000, tight=False, absent=0, limit=1.0),
        # the server's update of a small fp32 model
        dict(name="update_f32_1M", op="update", kind="2", each=False, types="f32", count=12, total=1_000_000, tight=False, absent=0, limit=1.0),
        # half-precision weights updated in place, sizes as they come
        dict(name="update_f16_5M", op="update", kind="2", each=False, types="f16", count=80, total=5_000_011, tight=True, absent=0, limit=1.0),
        # mixed precision: fp32 master weights and their bf16 copies
        dict(name="update_master_bf16_60.2M", op="update", kind="2", each=False, types="bf16", count=465, total=60_200_000, tight=False, absent=0, limit=1.0,
             master=True),
    ]


def draw(rng):
    """One more case: totals from 500 to 138 M, 1 to 600 tensors, or the rows of G."""
    while True:
        op = rng.choice(["norm", "clip", "clip", "pack", "update"])
        each = op in ("norm", "clip") and rng.random() < 0.3
        types = rng.choice(["f32", "bf16", "f16", "mixed"])
        total = int(math.exp(rng.uniform(math.log(500), math.log(138e6))))
        count = int(math.exp(rng.uniform(0.0, math.log(600))))
        if each and rng.random() < 0.5:
            count, types = -rng.randint(3, 64), "f32"
            total = total // -count * -count
        count = min(count, total)
        kind = rng.choice(["2", "2", "2", "max"])
        limit = rng.choice([1.0, 0.25, 1e6]) if kind == "2" else rng.choice([0.0078125, 1e6])
        case = dict(op=op, kind=kind, each=each, types=types, count=count, total=total, tight=rng.random() < 0.5,
                    absent=rng.choice([0, 0, 5]) if count > 5 else 0, limit=INF if op == "norm" else limit)
        if op == "update" and rng.random() < 0.5:
            case["master"] = True
        if total >= 500 and work(case)["bytes"] <= MAX_BYTES:
            return case


def _sizes(case):
    """Numbers of elements: equal rows (a negative count), or matrices and vectors in turn."""
    total, count = case["total"], case["count"]
    if count < 0:
        return [total // -count] * -count
    rng = random.Random(total * 1009 + count)
    share = [math.exp(rng.uniform(-2.5, 2.5)) if i % 2 == 0 else 0.0 for i in range(count)]
    sizes = [rng.choice([1, 10, 64, 256, 1000, 2048]) if i % 2 else 0 for i in range(count)]
    if not case["tight"]:
        sizes = [-(-n // 8) * 8 for n in sizes]
    if sum(sizes) > total // 4:
        sizes = [min(n, 1) for n in sizes]
    left, weight = total - sum(sizes), sum(share)
    for i in range(0, count, 2):
        n = int(left * share[i] / weight)
        sizes[i] = n if case["tight"] else n // 8 * 8
    sizes[0] += total - sum(sizes)
    return sizes


def _types(case):
    count = abs(case["count"])
    if case["types"] != "mixed":
        return [case["types"]] * count
    return [("bf16", "bf16", "f32", "f16")[i // 2 % 4] for i in range(count)]


def _present(case):
    return [not case["absent"] or i % case["absent"] != case["absent"] - 1 for i in range(abs(case["count"]))]


def _views(case):
    """Buffers by type, and each tensor as a view of its buffer."""
    at, place = {}, []
    for n, t in zip(_sizes(case), _types(case)):
        start = at.get(t, 0)
        if not case["tight"]:
            start = -(-start // 8) * 8
        place.append((t, start, n))
        at[t] = start + n
    buffers = {t: torch.zeros(n, dtype=TYPES[t], device="cuda") for t, n in at.items()}
    return buffers, [buffers[t][a:a + n] for t, a, n in place]


def _filled(case, gen, sigma):
    """The same with values: a scale of its own for each tensor."""
    buffers, views = _views(case)
    for t in sorted(buffers):
        buffers[t].normal_(generator=gen)
    scales = (torch.rand(len(views), generator=gen, device="cuda") * 4 - 2).exp_().mul_(sigma).tolist()
    for v, s in zip(views, scales):
        v.mul_(s)
    return buffers, [v if p else None for v, p in zip(views, _present(case))]


def _inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    d = case["total"]
    st = dict(case=case)
    if case["op"] == "update":
        st["u"] = torch.empty(d, dtype=torch.float32, device="cuda").normal_(generator=gen)
        if case.get("master"):
            st["master"] = torch.empty(d, dtype=torch.float32, device="cuda").normal_(0.0, 0.05, generator=gen)
        st["buffers"], st["tensors"] = _filled(case, gen, 0.05)
    else:
        st["buffers"], st["tensors"] = _filled(case, gen, 0.01)
    return st


def prepare(case, seed):
    st = _inputs(case, seed)
    if case["op"] == "clip" and case["limit"] < 1e6:          # below the limit: in place
        st["out_buffers"], out = _views(case)
        st["out"] = [o if g is not None else None for o, g in zip(out, st["tensors"])]
    if case["op"] == "pack":
        st["row"] = torch.empty(case["total"], dtype=torch.float32, device="cuda")
    st["norm"] = torch.empty(1, dtype=torch.float32, device="cuda")
    if case["each"]:
        st["each"] = torch.empty(abs(case["count"]), dtype=torch.float32, device="cuda")
    if own:
        import paper_1803_09877_b200 as dr
        st["kind"] = dr.NORM_2 if case["kind"] == "2" else dr.NORM_MAX
        st["layout"] = dr.Layout(_sizes(case), [TYPES[t] for t in _types(case)])
    return st


def run(st):
    return _own(st) if own else _plain(st)


def _own(st):
    case, lay = st["case"], st["layout"]
    op, limit, kind, each = case["op"], case["limit"], st["kind"], st.get("each")
    if op == "norm":
        lay.norm(st["tensors"], st["norm"], each=each, kind=kind)
        return _result(st)
    if op == "clip":
        lay.clip(st["tensors"], limit, out=st.get("out"), norm=st["norm"], each=each, separately=case["each"], kind=kind)
        return _result(st, st.get("out_buffers", st["buffers"]))
    if op == "pack":
        lay.pack(st["tensors"], st["row"], max_norm=limit, norm=st["norm"], kind=kind)
        return _result(st, dict(row=st["row"]))
    lay.update(st["tensors"], st["u"], UPDATE_SCALE, max_norm=limit, master=st.get("master"), norm=st["norm"], kind=kind)
    return _result(st, dict(st["buffers"], master=st["master"]) if "master" in st else st["buffers"])


def _result(st, buffers=None):
    out = dict(buffers or {}, norm=st["norm"])
    if "each" in st:
        out["each"] = st["each"]
    return out


def _norms(tensors, kind):
    """One norm a tensor and that of all, in 64 bits: sums of many squares."""
    zero = torch.zeros((), dtype=torch.float64, device="cuda")
    parts = [zero if t is None or t.numel() == 0 else t.double().square().sum() if kind == "2" else t.abs().max().double() for t in tensors]
    parts = torch.stack(parts)
    return (parts.sqrt(), parts.sum().sqrt()) if kind == "2" else (parts, parts.max())


def _factor(norm, limit):
    return torch.where((norm > limit) & torch.isfinite(norm.float()), limit / norm, 1.0).float()


def _plain(st):
    case = st["case"]
    op, limit = case["op"], case["limit"]
    if op == "update":
        _, norm = _norms([st["u"]], case["kind"])
        step = torch.where(torch.isfinite(norm.float()), UPDATE_SCALE * _factor(norm, limit), 0.0)
        at = 0
        for w, n in zip(st["tensors"], _sizes(case)):
            if w is not None:
                source = st["master"][at:at + n] if "master" in st else w.float()
                new = source - step * st["u"][at:at + n]
                if "master" in st:
                    source.copy_(new)
                w.copy_(new)
            at += n
        st["norm"].copy_(norm)
        return _result(st, dict(st["buffers"], master=st["master"]) if "master" in st else st["buffers"])
    each, norm = _norms(st["tensors"], case["kind"])
    st["norm"].copy_(norm)
    if "each" in st:
        st["each"].copy_(each)
    if op == "norm":
        return _result(st)
    c = _factor(each if case["each"] else norm, limit)
    if op == "clip":
        for i, (t, o) in enumerate(zip(st["tensors"], st.get("out", st["tensors"]))):
            if t is not None:
                o.copy_(t.float() * (c[i] if case["each"] else c))
        return _result(st, st.get("out_buffers", st["buffers"]))
    at = 0
    for t, n in zip(st["tensors"], _sizes(case)):
        st["row"][at:at + n] = 0.0 if t is None else t.float() * c
        at += n
    return _result(st, dict(row=st["row"]))


def work(case):
    """Bytes: every gradient once, what is written once, u and the weights of an update.  A list below its limit is read only."""
    data = sum(BYTES[t] * n for n, t, p in zip(_sizes(case), _types(case), _present(case)) if p)
    there = sum(n for n, p in zip(_sizes(case), _present(case)) if p)
    out = 4 + (4 * abs(case["count"]) if case["each"] else 0)
    op = case["op"]
    if op == "norm":
        return {"bytes": data + out, "flops": 2.0 * there}
    if op == "clip":
        below = case["limit"] >= 1e6
        return {"bytes": data + out + (0 if below else data), "flops": (2.0 if below else 3.0) * there}
    if op == "pack":
        return {"bytes": data + 4 * case["total"] + out, "flops": 3.0 * there}
    weights = 8 * there + data if case.get("master") else 2 * data
    return {"bytes": 4 * case["total"] + weights + out, "flops": 4.0 * there}


def exact(case, seed):
    """The definitions in 64 bits."""
    st = _inputs(case, seed)
    out = {}

    def p_norm(squares_or_maxima):
        v = torch.tensor(squares_or_maxima, dtype=torch.float64)
        return float(v.sum()) ** 0.5 if case["kind"] == "2" else float(v.max())

    def measure(x):
        if x is None or x.numel() == 0:
            return 0.0
        total = 0.0
        for c in x.split(1 << 24):
            c = c.to(torch.float64)
            total = total + float(torch.dot(c, c)) if case["kind"] == "2" else max(total, float(c.abs().max()))
        return total

    def bounded(v):
        return case["limit"] / v if v > case["limit"] else 1.0

    if case["op"] == "update":
        v = p_norm([measure(st["u"])])
        step = UPDATE_SCALE * bounded(v)
        new = {t: b.to(torch.float64) for t, b in st["buffers"].items()}
        master = st["master"].to(torch.float64) if "master" in st else None
        u, at = st["u"].to(torch.float64), 0
        for w, n in zip(st["tensors"], _sizes(case)):
            if w is not None and n:
                b = new[next(t for t in TYPES if TYPES[t] == w.dtype)]
                part = b[w.storage_offset():w.storage_offset() + n]
                if master is None:
                    part -= step * u[at:at + n]
                else:
                    master[at:at + n] -= step * u[at:at + n]
                    part.copy_(master[at:at + n])
            at += n
        out.update(new)
        if master is not None:
            out["master"] = master
        out["norm"] = torch.tensor([v], dtype=torch.float64)
        return out
    parts = [measure(x) for x in st["tensors"]]
    v = p_norm(parts)
    each = [p_norm([p]) for p in parts]
    out["norm"] = torch.tensor([v], dtype=torch.float64)
    if case["each"]:
        out["each"] = torch.tensor(each, dtype=torch.float64)
    if case["op"] == "norm":
        return out
    factors = [bounded(e) for e in each] if case["each"] else [bounded(v)] * len(parts)
    if case["op"] == "pack":
        row, at = torch.zeros(case["total"], dtype=torch.float64, device="cuda"), 0
        for x, n, c in zip(st["tensors"], _sizes(case), factors):
            if x is not None:
                row[at:at + n] = x.to(torch.float64) * c
            at += n
        out["row"] = row
        return out
    for t, b in st["buffers"].items():
        out[t] = b.to(torch.float64) if case["limit"] >= 1e6 else torch.zeros(b.numel(), dtype=torch.float64, device="cuda")
    for x, c in zip(st["tensors"], factors):
        if x is not None and x.numel():
            b = out[next(t for t in TYPES if TYPES[t] == x.dtype)]
            b[x.storage_offset():x.storage_offset() + x.numel()] = x.to(torch.float64) * c
    return out
