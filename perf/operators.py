"""Operators of layers with normalised rows and 8-bit products, and of clipped gradient steps, as measurable cases.

Kinds of a case
  norm       root-mean-square norm of rows, with a residual's addition, as rows of the storage type and / or 8-bit codes
  norm_grad  its backward pass: the rows' gradient and the gain's
  codes      rows (of activations, or of errors behind a ReLU) as 8-bit codes with a scale for each 128 columns
  transform  a layer's weights as codes, and its rows of codes times them (forward, or the input gradient: the same product)
  weights    weight gradient from codes of inputs and of errors
  clip       norm of all gradients, limited, into buffers of their own
  step       the same norm, and the gradient step with limited gradients
"""
import math

import torch

own = False

_EPS = 1e-5
_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # a handful of nodes asked for by a serving program, features as they come (odd width), fp32
        dict(name="norm_few_nodes", kind="norm", rows=200, width=75, dtype="f32", residual=False, codes=False),
        # all nodes of the large graph, hidden width 512, residual added, codes for the next product
        dict(name="norm_large_codes", kind="norm", rows=2_449_029, width=512, dtype="bf16", residual=True, codes=True),
        # backward of the citation-sized network's hidden rows in fp32, with the gradient of the residual stream
        dict(name="norm_grad", kind="norm_grad", rows=169_343, width=256, dtype="f32", residual=True),
        # backward of wide bf16 rows whose width is no power of two
        dict(name="norm_grad_wide", kind="norm_grad", rows=1_000_003, width=1000, dtype="bf16", residual=True),
        # errors of a class layer: 47 columns in fp32, most rows no training nodes
        dict(name="codes_class_errors", kind="codes", rows=410_003, width=47, dtype="f32", gate=False),
        # errors of a hidden layer of the large graph, behind the ReLU
        dict(name="codes_hidden_errors", kind="codes", rows=2_449_029, width=512, dtype="bf16", gate=True),
        # a hidden layer of the citation-sized network: weights of this step to codes, product, ReLU
        dict(name="transform_step", kind="transform", rows=169_343, inputs=256, outputs=256, dtype="bf16", relu=True, add=False),
        # the widest layer the package takes
        dict(name="transform_wide", kind="transform", rows=262_181, inputs=2048, outputs=2048, dtype="bf16", relu=True, add=False),
        # weight gradient of a hidden layer of the citation-sized network
        dict(name="weights_medium", kind="weights", rows=169_343, inputs=256, outputs=256),
        # weight gradient over all nodes of the large graph
        dict(name="weights_large", kind="weights", rows=2_449_029, inputs=512, outputs=512),
        # the six weight matrices of the 100-256-256-47 network with two taps: norm and step
        dict(name="step_network", kind="step", tensors=6, sizes="100-256-256-47", total=0, dtype="f32", limit=0.5),
        # many tensors of all sizes, 300 million elements
        dict(name="clip_many", kind="clip", tensors=403, sizes="spread", total=300_000_007, dtype="f32", limit=0.05),
    ]


_MOST = None


def _cost(c):
    w = work(c)
    return max(w["bytes"], w["flops"] / 50)


def draw(rng):
    """One more case of the same ranges: 1 to 1.2 million rows, widths of 8 to 2048 (odd ones included), 1 to 600 tensors
    of 1 element to tens of millions."""
    global _MOST
    if _MOST is None:
        _MOST = {}
        for c in listed():
            _MOST[c["kind"]] = max(_MOST.get(c["kind"], 0), _cost(c))
    log_uniform = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))  # noqa: E731
    while True:
        kind = rng.choice(["norm", "norm_grad", "codes", "transform", "transform", "weights", "clip", "step"])
        rows, width = log_uniform(1, 1_200_000), log_uniform(8, 2048)
        other = log_uniform(8, 2048)
        dtype = rng.choice(["f32", "bf16"])
        if rng.random() < 0.4:
            width = max(16, width // 16 * 16)
        if kind == "norm":
            c = dict(kind=kind, rows=rows, width=width, dtype=dtype, residual=rng.random() < 0.6, codes=rng.random() < 0.6)
        elif kind == "norm_grad":
            c = dict(kind=kind, rows=rows, width=width, dtype=dtype, residual=rng.random() < 0.6)
        elif kind == "codes":
            c = dict(kind=kind, rows=rows, width=width, dtype=dtype, gate=rng.random() < 0.5)
        elif kind == "transform":
            add = rng.random() < 0.3
            c = dict(kind=kind, rows=rows, inputs=width, outputs=other, dtype=dtype, relu=not add and rng.random() < 0.5, add=add)
        elif kind == "weights":
            c = dict(kind=kind, rows=rows, inputs=width, outputs=other)
        else:
            tensors = log_uniform(1, 600)
            c = dict(kind=kind, tensors=tensors, sizes="spread", total=max(tensors, log_uniform(1_000, 200_000_000)),
                     dtype=dtype if kind == "clip" else "f32", limit=round(math.exp(rng.uniform(math.log(0.05), math.log(5.0))), 3))
        # (a step's only listed case is a small network's: the limit of its cost is that of clipping)
        if _cost(c) <= _MOST["clip" if kind == "step" else kind]:
            return c


# ---------------------------------------------------------------------------------------------------------------
# what a program has in hand
# ---------------------------------------------------------------------------------------------------------------

def _up(n, m):
    return (n + m - 1) // m * m


def _tensor_sizes(c):
    """Elements of every tensor of a clip or step case."""
    if c["sizes"] != "spread":
        w = [int(v) for v in c["sizes"].split("-")]
        return [w[l] * w[l + 1] for l in range(len(w) - 1) for _ in range(2)]
    n, total = c["tensors"], c["total"]
    shares = [math.exp(6.0 * math.sin(1.0 + 2.399963 * i)) for i in range(n)]       # from one to 160,000 times the smallest
    scale = (total - n) / sum(shares)
    sizes = [1 + int(s * scale) for s in shares]
    sizes[-1] += total - sum(sizes)
    return sizes


def _exponent(a):
    """Smallest e with a 2^-e <= 448 = 0.875 2^9, at least -127; 0 for a = 0."""
    m, p = torch.frexp(a)
    e = p - 9 + (m > 0.875).to(p.dtype)
    return torch.where(a > 0, e.clamp(min=-127), torch.zeros_like(e))


def _blocks(v, n):
    """v with its last dimension in blocks of n, zeros behind the last column."""
    w = v.shape[-1]
    if w % n:
        v = torch.nn.functional.pad(v, (0, n - w % n))
    return v.reshape(*v.shape[:-1], -1, n)


def _inverse(e):
    """2^-e for -127 <= e <= 126 by its bits (a power computed by a function may be off by a last bit, which moves ties)."""
    return ((127 - e) << 23).to(torch.int32).view(torch.float32)


def _rows_to_codes(v):
    """fp32 rows -> (codes as e4m3 [rows, width], scales as e8m0 [rows, blocks])."""
    w = v.shape[-1]
    b = _blocks(v, 128)
    e = _exponent(b.abs().amax(-1))
    q = (b * _inverse(e).unsqueeze(-1)).to(torch.float8_e4m3fn)
    return q.reshape(v.shape[0], -1)[:, :w], (e + 127).to(torch.uint8).view(torch.float8_e8m0fnu)


def _weights_to_codes(h):
    """fp32 matrix -> (codes as e4m3 [r, c], scales as e8m0 [blocks of r, blocks of c]), blocks of 128 x 128."""
    r, c = h.shape
    p = torch.nn.functional.pad(h, (0, -c % 128, 0, -r % 128))
    b = p.reshape(p.shape[0] // 128, 128, p.shape[1] // 128, 128)
    e = _exponent(b.abs().amax((1, 3)))
    q = (b * _inverse(e)[:, None, :, None]).to(torch.float8_e4m3fn)
    return q.reshape(p.shape)[:r, :c], (e + 127).to(torch.uint8).view(torch.float8_e8m0fnu)


def _value(codes, scales, like):
    """What rows of codes stand for, in the type `like`."""
    w = codes.shape[1]
    return (_blocks(codes.to(like), 128) * scales.to(like).unsqueeze(-1)).reshape(codes.shape[0], -1)[:, :w]


def _stored(codes, scales, width):
    """Codes and scales in the buffers that the calls take: code rows of whole 16 bytes, scale rows of whole 4."""
    n = codes.shape[0]
    c = torch.zeros((n, _up(width, 16)), dtype=torch.uint8, device="cuda")
    c[:, :width] = codes.contiguous().view(torch.uint8)
    s = torch.full((n, _up(-(-width // 128), 4)), 127, dtype=torch.uint8, device="cuda")
    s[:, :scales.shape[1]] = scales.view(torch.uint8)
    return c, s


def _code_buffers(rows, width, scale_rows=None):
    c = torch.zeros((rows, _up(width, 16)), dtype=torch.uint8, device="cuda")
    s = torch.zeros((rows if scale_rows is None else scale_rows, _up(-(-width // 128), 4)), dtype=torch.uint8, device="cuda")
    return c, s


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    kind = case["kind"]
    t = _TYPES[case.get("dtype", "f32")]

    def normal(*shape, dtype=torch.float32, scale=1.0):
        return torch.randn(*shape, generator=g, device="cuda", dtype=dtype).mul_(scale)

    def activations(n, w, dtype):
        """Rows of different size, as a layer without norm leaves them."""
        size = torch.exp(torch.randn(n, 1, generator=g, device="cuda") * 0.7)
        return normal(n, w, dtype=dtype).mul_(size.to(dtype))

    def errors(n, w, dtype):
        """Gradients: small, and none at four rows in ten (nodes whose class is not known)."""
        on = (torch.rand(n, 1, generator=g, device="cuda") > 0.4).to(dtype)
        return normal(n, w, dtype=dtype, scale=1.0 / max(1, n)).mul_(on)

    s = dict(case=case)
    if kind in ("norm", "norm_grad"):
        n, w = case["rows"], case["width"]
        s["gain"] = 1.0 + normal(w, scale=0.2)
        if kind == "norm":
            s["x"] = activations(n, w, t)
            s["residual"] = activations(n, w, t) if case["residual"] else None
            s["total"] = torch.empty((n, w), dtype=t, device="cuda") if case["residual"] else None
            s["inv"] = torch.empty(n, device="cuda")
            if case["codes"]:
                s["codes"], s["scales"] = _code_buffers(n, w)
            else:
                s["y"] = torch.empty((n, w), dtype=t, device="cuda")
        else:
            s["u"] = activations(n, w, t)
            s["inv"] = torch.cat([torch.rsqrt(p.float().square().mean(-1) + _EPS) for p in s["u"].split(1 << 18)])
            s["dy"] = errors(n, w, t)
            s["du"] = errors(n, w, t) if case["residual"] else None
            s["dx"] = torch.empty((n, w), dtype=t, device="cuda")
            s["dgain"] = torch.empty(w, device="cuda")
            s["workspace"] = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")
    elif kind == "codes":
        n, w = case["rows"], case["width"]
        s["x"] = errors(n, w, t)
        s["gate"] = normal(n, w, dtype=t).clamp_(min=0) if case["gate"] else None
        s["codes"], s["scales"] = _code_buffers(n, w)
    elif kind == "transform":
        n, fi, fo = case["rows"], case["inputs"], case["outputs"]
        parts = [_stored(*_rows_to_codes(activations(m, fi, torch.float32)), fi) for m in [1 << 18] * (n >> 18) + [n & ((1 << 18) - 1)] if m]
        s["codes"], s["scales"] = (torch.cat(p) for p in zip(*parts))
        s["h"] = normal(fi, fo, scale=math.sqrt(2.0 / (fi + fo)))
        s["turned"], s["turned_scales"] = _code_buffers(fo, fi, -(-fo // 128))
        s["plain"], s["plain_scales"] = _code_buffers(fi, fo, -(-fi // 128))
        s["c"] = normal(n, fo, dtype=t) if case["add"] else torch.empty((n, fo), dtype=t, device="cuda")
    elif kind == "weights":
        n, fi, fo = case["rows"], case["inputs"], case["outputs"]
        for name, w, of in (("y", fi, activations), ("d", fo, errors)):
            parts = [_stored(*_rows_to_codes(of(m, w, torch.float32)), w) for m in [1 << 18] * (n >> 18) + [n & ((1 << 18) - 1)] if m]
            s[name], s[name + "_scales"] = (torch.cat(p) for p in zip(*parts))
        s["dh"] = torch.empty((fi, fo), device="cuda")
        s["workspace"] = torch.empty(1 << 30, dtype=torch.uint8, device="cuda")
    else:
        sizes = _tensor_sizes(case)
        each = [normal(1, scale=0.5).abs().item() / math.sqrt(sum(sizes)) for _ in range(4)]
        s["grads"] = [normal(m, dtype=t, scale=each[i % 4]) for i, m in enumerate(sizes)]
        s["others"] = [normal(m) for m in sizes] if kind == "step" else [torch.empty(m, dtype=t, device="cuda") for m in sizes]
        s["norm"] = torch.empty(2, device="cuda")
        s["workspace"] = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
        if own:            # the tables of addresses that a program makes once for its tensors; the plain form has none
            from paper_2406_17611_amd import binding as vb
            s["lists"] = vb.TensorList(s["grads"]), vb.TensorList(s["others"])
    return s


# ---------------------------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------------------------

def run(s):
    return _call(s) if own else _plain(s)


def _call(s):
    from paper_2406_17611_amd import binding as vb
    c = s["case"]
    kind = c["kind"]
    e4m3, e8m0 = torch.float8_e4m3fn, torch.float8_e8m0fnu
    if kind == "norm":
        vb.rms_norm_fwd(s["x"], s["gain"], _EPS, residual=s["residual"], total=s["total"], y=s.get("y"), codes=s.get("codes"),
                        scales=s.get("scales"), inv_rms=s["inv"])
        out = dict(inv=s["inv"])
        if c["residual"]:
            out["total"] = s["total"]
        if c["codes"]:
            out["codes"], out["scales"] = s["codes"].view(e4m3)[:, :c["width"]], s["scales"].view(e8m0)[:, :-(-c["width"] // 128)]
        else:
            out["y"] = s["y"]
        return out
    if kind == "norm_grad":
        vb.rms_norm_bwd(s["dy"], s["u"], s["gain"], s["inv"], s["dx"], s["dgain"], dtotal=s["du"], workspace=s["workspace"])
        return dict(dx=s["dx"], dgain=s["dgain"])
    if kind == "codes":
        vb.quantize_rows(s["x"], s["codes"], s["scales"], gate=s["gate"])
        return dict(codes=s["codes"].view(e4m3)[:, :c["width"]], scales=s["scales"].view(e8m0)[:, :-(-c["width"] // 128)])
    if kind == "transform":
        fi, fo = c["inputs"], c["outputs"]
        vb.quantize_weights(s["h"], s["turned"], s["turned_scales"], s["plain"], s["plain_scales"])
        vb.scaled_transform(s["codes"], s["scales"], s["turned"], s["turned_scales"], fi, s["c"], accumulate=c["add"],
                            act=vb.ACT_RELU if c["relu"] else vb.ACT_IDENTITY)
        return dict(c=s["c"], turned=s["turned"].view(e4m3)[:, :fi], turned_scales=s["turned_scales"].view(e8m0)[:, :-(-fi // 128)],
                    plain=s["plain"].view(e4m3)[:, :fo], plain_scales=s["plain_scales"].view(e8m0)[:, :-(-fo // 128)])
    if kind == "weights":
        vb.scaled_bwd_weight(s["y"], s["y_scales"], s["d"], s["d_scales"], s["dh"], workspace=s["workspace"])
        return dict(dh=s["dh"])
    grads, others = s["lists"]
    if kind == "clip":
        vb.clip_gradients(grads, c["limit"], s["norm"], into=others, workspace=s["workspace"])
        return dict(norm=s["norm"], grads=_joined(s["others"]))
    vb.sgd_step_clipped(others, grads, 1e-3, c["limit"], s["norm"], workspace=s["workspace"])
    return dict(norm=s["norm"], weights=_joined(s["others"]))


def _joined(tensors):
    """At most 32 outputs: the largest tensors as they are."""
    if len(tensors) <= 32:
        return list(tensors)
    at = sorted(range(len(tensors)), key=lambda i: -tensors[i].numel())
    return [tensors[i] for i in at[:16]] + [tensors[i] for i in at[-16:]]


def _plain(s):
    c = s["case"]
    kind = c["kind"]
    if kind == "norm":
        t = s["x"].dtype
        u = (s["x"].float() + s["residual"].float()).to(t) if c["residual"] else s["x"]
        v = u.float()
        inv = torch.rsqrt(v.square().mean(-1) + _EPS)
        y = v * inv.unsqueeze(-1) * s["gain"]
        out = dict(inv=inv)
        if c["residual"]:
            out["total"] = u
        if c["codes"]:
            out["codes"], out["scales"] = _rows_to_codes(y)
        else:
            out["y"] = y.to(t)
        return out
    if kind == "norm_grad":
        t = s["dy"].dtype
        inv = s["inv"].unsqueeze(-1)
        xh, dy = s["u"].float() * inv, s["dy"].float()
        h = dy * s["gain"]
        dx = inv * (h - xh * (h * xh).mean(-1, keepdim=True))
        if c["residual"]:
            dx = dx + s["du"].float()
        return dict(dx=dx.to(t), dgain=(dy * xh).sum(0))
    if kind == "codes":
        v = s["x"].float()
        if c["gate"]:
            v = torch.where(s["gate"] > 0, v, torch.zeros_like(v))
        codes, scales = _rows_to_codes(v)
        return dict(codes=codes, scales=scales)
    if kind == "transform":
        fi = c["inputs"]
        q, e = _weights_to_codes(s["h"])
        w = q.float() * e.float().repeat_interleave(128, 0)[:q.shape[0]].repeat_interleave(128, 1)[:, :q.shape[1]]
        v = _value(s["codes"].view(torch.float8_e4m3fn)[:, :fi], _scales(s["scales"], fi), torch.float32) @ w
        if c["add"]:
            v = s["c"].float() + v
        if c["relu"]:
            v = v.clamp(min=0)
        s["c"].copy_(v)
        return dict(c=s["c"], turned=q.t(), turned_scales=e.t(), plain=q, plain_scales=e)
    if kind == "weights":
        v = [_value(s[k].view(torch.float8_e4m3fn)[:, :w], _scales(s[k + "_scales"], w), torch.float32)
             for k, w in (("y", c["inputs"]), ("d", c["outputs"]))]
        return dict(dh=v[0].t() @ v[1])
    norm = torch.stack([x.double().square().sum() for x in s["grads"]]).sum().sqrt()
    factor = torch.clamp(c["limit"] / norm, max=1.0)
    s["norm"].copy_(torch.stack([norm, factor]))
    f = s["norm"][1]
    if kind == "clip":
        for into, x in zip(s["others"], s["grads"]):
            into.copy_(x.float() * f)
        return dict(norm=s["norm"], grads=_joined(s["others"]))
    for w, x in zip(s["others"], s["grads"]):
        w.copy_(w - 1e-3 * f * x)
    return dict(norm=s["norm"], weights=_joined(s["others"]))


def _scales(stored, width):
    """Stored exponents of real columns as scales."""
    return stored.view(torch.float8_e8m0fnu)[:, :-(-width // 128)]


# ---------------------------------------------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------------------------------------------

def work(case):
    kind = case["kind"]
    e = 2 if case.get("dtype") == "bf16" else 4
    coded = lambda n, w: n * (w + -(-w // 128))  # noqa: E731
    if kind == "norm":
        n, w = case["rows"], case["width"]
        b = n * w * e * (3 if case["residual"] else 1) + (coded(n, w) if case["codes"] else n * w * e) + 4 * n + 4 * w
        return {"bytes": b, "flops": 5.0 * n * w}
    if kind == "norm_grad":
        n, w = case["rows"], case["width"]
        return {"bytes": n * w * e * (4 if case["residual"] else 3) + 4 * n + 8 * w, "flops": 9.0 * n * w}
    if kind == "codes":
        n, w = case["rows"], case["width"]
        return {"bytes": n * w * e * (2 if case["gate"] else 1) + coded(n, w), "flops": 2.0 * n * w}
    if kind == "transform":
        n, fi, fo = case["rows"], case["inputs"], case["outputs"]
        return {"bytes": coded(n, fi) + n * fo * e * (2 if case["add"] else 1) + 6 * fi * fo, "flops": 2.0 * n * fi * fo}
    if kind == "weights":
        n, fi, fo = case["rows"], case["inputs"], case["outputs"]
        return {"bytes": coded(n, fi) + coded(n, fo) + 4 * fi * fo, "flops": 2.0 * n * fi * fo}
    n = sum(_tensor_sizes(case))
    # the limit is known when all gradients have been read once: they are read again
    return {"bytes": n * e * 3 if kind == "clip" else n * 16, "flops": 4.0 * n}


# ---------------------------------------------------------------------------------------------------------------
# the definition in 64 bits
# ---------------------------------------------------------------------------------------------------------------

def _nearest_code(v):
    """fp64 values of magnitude 448 at most -> nearest numbers of 4 exponent and 3 fraction bits, ties to even."""
    p = torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -20))).clamp(min=-6)
    unit = _power(p - 3)
    return torch.round(v / unit) * unit


def _power(p):
    """2^p in fp64, exactly."""
    return ((p.to(torch.int64) + 1023) << 52).view(torch.float64)


def _exact_scale(a):
    e = torch.ceil(torch.log2(a.clamp(min=2.0 ** -1000) / 448.0))
    e = torch.where(a > _power(e) * 448.0, e + 1, e)
    e = torch.where(a <= _power(e - 1) * 448.0, e - 1, e).clamp(min=-127)
    return torch.where(a > 0, _power(e), torch.ones_like(a))


def _exact_codes(v):
    codes, scales = torch.empty_like(v), []
    for j in range(0, v.shape[1], 128):
        s = _exact_scale(v[:, j:j + 128].abs().amax(1))
        codes[:, j:j + 128] = _nearest_code(v[:, j:j + 128] / s[:, None])
        scales.append(s)
    return codes, torch.stack(scales, 1)


def _exact_values(stored, scales, width):
    v = stored.view(torch.float8_e4m3fn)[:, :width].to(torch.float64)
    for j in range(0, width, 128):
        v[:, j:j + 128] *= _power(scales[:, j // 128].to(torch.float64) - 127)[:, None]
    return v


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    step = 1 << 18
    f64 = torch.float64
    parts = lambda *t: zip(*(x.split(step) if x is not None else [None] * (-(-case["rows"] // step)) for x in t))  # noqa: E731
    join = lambda got: {k: torch.cat([g[k] for g in got]) for k in got[0]}  # noqa: E731
    if kind == "norm":
        got = []
        for x, r in parts(s["x"], s["residual"]):
            u = x.to(f64)
            if r is not None:
                u = (u + r.to(f64)).to(x.dtype).to(f64)
            inv = (u.pow(2).sum(1) / case["width"] + _EPS).pow(-0.5)
            y = u * inv[:, None] * s["gain"].to(f64)
            o = dict(inv=inv)
            if r is not None:
                o["total"] = u.to(x.dtype)
            if case["codes"]:
                codes, scales = _exact_codes(y)
                o["codes"], o["scales"] = codes.to(torch.float32), scales
            else:
                o["y"] = y
            got.append(o)
        return join(got)
    if kind == "norm_grad":
        got, dgain = [], torch.zeros(case["width"], dtype=f64, device="cuda")
        for dy, u, du in parts(s["dy"], s["u"], s["du"]):
            # the norm's derivative applied to h: (h - u (u . h) / (w (mean u^2 + eps))) / rms, 1 / rms as it was saved
            inv = s["inv"][sum(len(g) for g in got):][:len(u)].to(f64)[:, None]
            u, dy = u.to(f64), dy.to(f64)
            h = dy * s["gain"].to(f64)
            dx = h * inv - u * inv.pow(3) * ((u * h).sum(1, keepdim=True) / case["width"])
            if du is not None:
                dx += du.to(f64)
            dgain += torch.einsum("nw,nw->w", dy, u * inv)
            got.append(dx)
        return dict(dx=torch.cat(got), dgain=dgain)
    if kind == "codes":
        got = []
        for x, gate in parts(s["x"], s["gate"]):
            v = x.to(f64)
            if gate is not None:
                v = v * (gate > 0)
            codes, scales = _exact_codes(v)
            got.append(dict(codes=codes.to(torch.float32), scales=scales))
        return join(got)
    if kind == "transform":
        fi, fo = case["inputs"], case["outputs"]
        h = s["h"].to(f64)
        codes, scales = torch.empty_like(h), torch.empty((-(-fi // 128), -(-fo // 128)), dtype=f64, device="cuda")
        w = torch.empty_like(h)
        for i in range(scales.shape[0]):
            for j in range(scales.shape[1]):
                at = (slice(128 * i, 128 * i + 128), slice(128 * j, 128 * j + 128))
                scales[i, j] = _exact_scale(h[at].abs().max())
                codes[at] = _nearest_code(h[at] / scales[i, j])
                w[at] = codes[at] * scales[i, j]
        got = []
        for q, e, c in parts(s["codes"], s["scales"], s["c"]):
            v = torch.mm(_exact_values(q, e, fi), w)
            if case["add"]:
                v = v + c.to(f64)
            got.append(torch.relu(v) if case["relu"] else v)
        return dict(c=torch.cat(got), turned=codes.t(), turned_scales=scales.t(), plain=codes, plain_scales=scales)
    if kind == "weights":
        dh = torch.zeros((case["inputs"], case["outputs"]), dtype=f64, device="cuda")
        for y, ys, d, ds in parts(s["y"], s["y_scales"], s["d"], s["d_scales"]):
            dh += torch.mm(_exact_values(y, ys, case["inputs"]).t(), _exact_values(d, ds, case["outputs"]))
        return dict(dh=dh)
    square = 0.0
    for g in s["grads"]:
        square += float(torch.linalg.vector_norm(g.to(f64))) ** 2
    norm = math.sqrt(square)
    factor = min(1.0, case["limit"] / norm) if norm else 1.0
    out = dict(norm=torch.tensor([norm, factor], dtype=f64, device="cuda"))
    if kind == "clip":
        out["grads"] = [factor * g.to(f64) for g in _joined(s["grads"])]
    else:
        out["weights"] = [w.to(f64) - 1e-3 * factor * g.to(f64) for w, g in zip(_joined(s["others"]), _joined(s["grads"]))]
    return out
