"""Operators of a voxel network's training and attention as they are measured: rotary positions over three axes,
group norm with an activation over packed scans, and activation checkpoints in 8 bits.

A case is a dict of plain values.  Its ``op`` is

* ``rope`` -- rotation of the heads of q and k by their voxels' coordinates (``heads`` and ``kv_heads`` heads of
  ``head_dim`` channels, ``sections`` pairs for x, y and z, pairs of neighbours or of ``halves``); with ``train`` the
  gradients' rotation back too; ``packed`` hands q and k over as views of one row-major buffer;
* ``gn`` -- group norm of the voxels of each scan with an activation; with ``train`` its backward too, the residual
  branch's gradient added where ``res`` is set, reading a checkpoint in 8 bits of the input where ``ckpt`` is;
* ``ckpt`` -- rows into 8 bits and back (``out`` = 0), or the weight gradient [channels][out] of a linear layer from
  the rows in 8 bits.

Rows are spread unevenly over the scans (``lengths``); ``empty`` is the index of a scan with no voxel, or -1.  The
plain forms are elementary torch operations in 32 bits, angles in 64, rounded once at the end.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
EPS = 1e-5
BLOCK = 32  # channels that share an exponent in a checkpoint


def listed():
    return [
        # the query tokens of a few scans, in single precision: launches and latency
        rope("rope_tokens_f32", 40, 8, 0, 32, (6, 6, 4), "f32"),
        # four sweeps at stride 16, q and k side by side in one buffer
        rope("rope_stage16_bf16", 11263, 8, 8, 32, (6, 6, 4), "bf16", packed=True),
        # a training step at stride 8, shared key heads, a part of a head's channels rotated, pairs of halves
        rope("rope_train_stage8_f16", 26881, 4, 2, 64, (8, 8, 8), "f16", halves=True, train=True),
        # a whole sweep at full resolution, forward and backward
        rope("rope_train_sweep_bf16", 88119, 8, 8, 32, (6, 6, 4), "bf16", train=True),
        # the voxels around one object, in single precision
        gn("gn_object_f32", 701, 1, 96, 8, "f32", "relu"),
        # the full-resolution voxels of a batch of four sweeps
        gn("gn_batch_bf16", 300007, 4, 96, 8, "bf16", "relu"),
        # training steps: one sweep at stride 1 with a residual branch, and a batch at stride 8 from a checkpoint
        gn("gn_train_sweep_bf16", 88119, 1, 96, 8, "bf16", "silu", train=True, res=True),
        gn("gn_train_stage8_ckpt_f16", 26881, 4, 256, 16, "f16", "silu", train=True, ckpt=True),
        # the saved rows of a batch of sweeps, and what their backward reads
        ckpt("ckpt_batch_bf16", 300007, 96, 0, "bf16"),
        # a linear layer's weight gradient: an object's voxels, a sweep, a batch at stride 8
        ckpt("ckpt_wgrad_object_f32", 701, 96, 96, "f32"),
        ckpt("ckpt_wgrad_sweep_bf16", 88119, 96, 96, "bf16"),
        ckpt("ckpt_wgrad_stage8_f16", 26881, 256, 256, "f16"),
    ]


def rope(name, rows, heads, kv_heads, head_dim, sections, dtype, halves=False, packed=False, train=False):
    sx, sy, sz = sections
    return dict(name=name, op="rope", rows=rows, heads=heads, kv_heads=kv_heads, head_dim=head_dim, sx=sx, sy=sy, sz=sz,
                dtype=dtype, halves=halves, packed=packed, train=train)


def gn(name, rows, scans, channels, groups, dtype, act, train=False, res=False, ckpt=False, empty=-1):
    return dict(name=name, op="gn", rows=rows, scans=scans, channels=channels, groups=groups, dtype=dtype, act=act,
                train=train, res=res, ckpt=ckpt, empty=empty)


def ckpt(name, rows, channels, out, dtype):
    return dict(name=name, op="ckpt", rows=rows, channels=channels, out=out, dtype=dtype)


def draw(rng):
    def size(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    dtype = rng.choice(("bf16", "bf16", "f16", "f32"))
    op = rng.choice(("rope", "gn", "gn", "ckpt", "ckpt"))
    if op == "rope":
        kv = rng.choice((0, 1, 2, 3, 4, 8))
        heads = max(kv, 1) * (rng.choice((1, 2, 4)) if kv <= 2 else 1)
        D = rng.choice((16, 24, 32, 32, 64, 96, 128))
        pairs = D // 2 if rng.random() < 0.6 else rng.randint(3, D // 2)
        sy = sz = pairs // 3
        if rng.random() < 0.2:  # the plane alone
            sy, sz = pairs // 2, 0
        most = min(88119, 88119 * 512 // ((heads + kv) * D))
        case = rope("", size(1, most), heads, kv, D, (pairs - sy - sz, sy, sz), dtype, halves=rng.random() < 0.4,
                    packed=kv > 0 and rng.random() < 0.4, train=rng.random() < 0.5)
    elif op == "gn":
        C = rng.choice((19, 32, 48, 64, 96, 96, 128, 256))
        groups = rng.choice([g for g in (1, 2, 3, 4, 8, 16, 19, 32, C) if C % g == 0])
        scans = rng.choice((1, 1, 2, 4, 8))
        train = rng.random() < 0.5
        # ReLU's gradient jumps where z changes its sign, and one of millions of z lies within a rounding of 0
        case = gn("", size(1, 300007 * 32 // C if train else 300007 * 96 // max(C, 96)), scans, C, groups, dtype,
                  rng.choice(("silu", "none")) if train else rng.choice(("relu", "silu", "none")), train=train,
                  res=train and rng.random() < 0.5, ckpt=train and rng.random() < 0.5,
                  empty=rng.randrange(scans) if scans > 1 and rng.random() < 0.3 else -1)
    else:
        C = rng.choice((19, 32, 64, 96, 96, 128, 256))
        out = rng.choice((0, 0, 19, 32, 64, 96, 128, 256))
        most = 300007 * 96 // max(C, 96) if not out else min(88119, 88119 * 128 * 128 // (max(C, 64) * max(out, 64)))
        case = ckpt("", size(1, most), C, out, dtype)
    del case["name"]
    return case


def lengths(case):
    """Voxels of each scan: uneven, all of the case's rows in all."""
    n = case["scans"]
    weight = [0.0 if b == case["empty"] else 1.0 + 0.4 * math.sin(1.7 * b + 0.6) for b in range(n)]
    total, out, done = sum(weight), [], 0
    for b in range(n):
        end = round(case["rows"] * sum(weight[: b + 1]) / total)
        out.append(end - done)
        done = end
    return out


def sections(case):
    return case["sx"], case["sy"], case["sz"]


# -- inputs ------------------------------------------------------------------

class Draws:
    """Seeded values on the GPU."""

    def __init__(self, seed):
        self.gen = torch.Generator(device="cuda")
        self.gen.manual_seed(int(seed) * 1_000_003 + 31)

    def normal(self, *shape, std=1.0, dtype=torch.float32):
        return (torch.randn(*shape, generator=self.gen, device="cuda") * std).to(dtype)

    def features(self, m, C, dtype):
        """Channels of unequal spread around unequal means, as a residual stream's."""
        x = self.normal(m, C) * (0.3 + 2.0 * torch.rand(C, generator=self.gen, device="cuda")) + self.normal(C)
        return x.to(dtype)

    def voxels(self, n):
        """Coordinates (b, x, y, z) of a sweep: wide and flat, far from the origin where a map's frame is kept."""
        xy = torch.randint(-1024, 1024, (n, 2), generator=self.gen, device="cuda")
        xy += torch.randint(-20000, 20000, (1, 2), generator=self.gen, device="cuda")
        z = torch.randint(-40, 60, (n, 1), generator=self.gen, device="cuda")
        return torch.cat([torch.zeros_like(z), xy, z], 1).to(torch.int32)


def frequencies(case):
    """Radians a voxel: from a wavelength of some voxels to one of hundreds, for each axis."""
    return torch.tensor([math.pow(100.0, -i / s) for s in sections(case) for i in range(s)], dtype=torch.float32,
                        device="cuda")


def data(case, seed):
    r, dt, m = Draws(seed), DTYPES[case["dtype"]], case["rows"]
    if case["op"] == "rope":
        H, K, D = case["heads"], case["kv_heads"], case["head_dim"]
        d = dict(coords=r.voxels(m), freqs=frequencies(case), k=None, dk=None)
        if case["packed"]:  # q, k and v side by side, as one product for all three leaves them
            d["q"], d["k"] = torch.split(r.normal(m, H + 2 * K, D, dtype=dt), [H, K, K], dim=1)[:2]
        else:
            d["q"] = r.normal(m, H, D, dtype=dt)
            if K:
                d["k"] = r.normal(m, K, D, dtype=dt)
        if case["train"]:
            d["dq"] = r.normal(m, H, D, dtype=dt)
            if K:
                d["dk"] = r.normal(m, K, D, dtype=dt)
        return d
    C = case["channels"]
    d = dict(x=r.features(m, C, dt))
    if case["op"] == "ckpt":
        if case["out"]:
            d["da"] = r.normal(m, case["out"], dtype=dt)
        return d
    d["lens"] = lengths(case)
    off = [0]
    for n in d["lens"]:
        off.append(off[-1] + n)
    d["off"] = torch.tensor(off, dtype=torch.int32, device="cuda")
    d["gamma"], d["beta"] = 1.0 + r.normal(C, std=0.1), r.normal(C, std=0.1)
    if case["train"]:
        d["dy"] = r.normal(m, C, dtype=dt)
        d["dres"] = r.normal(m, C, dtype=dt) if case["res"] else None
    return d


def prepare(case, seed):
    d = data(case, seed)
    d["case"] = case
    if not own:
        return d
    from paper_2007_16100_amd import spv
    if case["op"] == "rope":
        d["params"] = spv.make_rope_params(case["head_dim"], d["freqs"], sections(case), halves=case["halves"])
    elif case["op"] == "gn":
        sizes = (case["rows"], case["channels"], case["groups"], case["scans"])
        d["ws"] = (spv.Workspace.for_group_norm_backward if case["train"] else spv.Workspace.for_group_norm)(*sizes)
    elif case["out"]:
        d["ws"] = spv.Workspace.for_linear_backward8(case["rows"], case["channels"], case["out"])
    return d


# -- one pass ----------------------------------------------------------------

def run(state):
    return globals()[("own_" if own else "plain_") + state["case"]["op"]](state)


def own_rope(d):
    from paper_2007_16100_amd import spv
    out = spv.spv_rope(d["params"], d["coords"], d["q"], d["k"])
    if not d["case"]["train"]:
        return out
    grads = spv.spv_rope(d["params"], d["coords"], d["dq"], d["dk"], inverse=True)
    return [out, grads] if d["k"] is None else [*out, *grads]


def own_gn(d):
    from paper_2007_16100_amd import spv
    case = d["case"]
    args = dict(gamma=d["gamma"], beta=d["beta"], act=case["act"])
    if not case["train"]:
        return spv.spv_group_norm(d["ws"], d["x"], d["off"], case["groups"], eps=EPS, **args)
    if case["ckpt"]:
        y, stat, x = spv.spv_group_norm(d["ws"], d["x"], d["off"], case["groups"], eps=EPS, want_stat=True,
                                        want_checkpoint=True, **args)
    else:
        y, stat = spv.spv_group_norm(d["ws"], d["x"], d["off"], case["groups"], eps=EPS, want_stat=True, **args)
        x = d["x"]
    dx, dgamma, dbeta = spv.spv_group_norm_backward(d["ws"], d["dy"], x, d["off"], case["groups"], stat, dres=d["dres"],
                                                    **args)
    return dict(y=y, dx=dx, dgamma=dgamma, dbeta=dbeta)


def own_ckpt(d):
    from paper_2007_16100_amd import spv
    saved = spv.spv_checkpoint8(d["x"])
    if not d["case"]["out"]:
        return spv.spv_checkpoint8_read(saved)
    return spv.spv_linear_backward8(d["ws"], saved, d["da"])


def plain_rope(d):
    case = d["case"]
    P, D = sum(sections(case)), case["head_dim"]
    axis = torch.tensor([a for a, s in enumerate(sections(case), 1) for _ in range(s)], device="cuda")
    angle = d["coords"][:, axis].double() * d["freqs"].double()
    cos, sin = torch.cos(angle).float().unsqueeze(1), torch.sin(angle).float().unsqueeze(1)

    def rotate(t, sin):
        x = t.float()
        u, w = (x[..., :P], x[..., P:2 * P]) if case["halves"] else (x[..., 0:2 * P:2], x[..., 1:2 * P:2])
        a, b = u * cos - w * sin, u * sin + w * cos
        turned = torch.cat([a, b], -1) if case["halves"] else torch.stack([a, b], -1).flatten(-2)
        return torch.cat([turned, x[..., 2 * P:]], -1).to(t.dtype)

    out = [rotate(t, sin) for t in (d["q"], d["k"]) if t is not None]
    if case["train"]:
        out += [rotate(t, -sin) for t in (d["dq"], d["dk"]) if t is not None]
    return out if len(out) > 1 else out[0]


def plain_codes(x):
    """The codes of rows in 8 bits (float32 whole numbers) and their scales, in blocks of 32 channels."""
    m, C = x.shape
    nb = -(-C // BLOCK)
    f = torch.zeros(m, nb * BLOCK, device="cuda")
    f[:, :C] = x.float()
    f = f.view(m, nb, BLOCK)
    top = (f.abs().amax(-1, keepdim=True).view(torch.int32) >> 23) - 127  # the largest value's exponent
    e = (top - 6).clamp(min=-24 if x.dtype == torch.float16 else -126)
    code = torch.round(f * ((127 - e) << 23).view(torch.float32)).clamp(-127, 127)
    return code, ((127 + e) << 23).view(torch.float32)


def plain_saved(x):
    """What is read back from 8 bits, in float32."""
    code, scale = plain_codes(x)
    return (code * scale).flatten(1)[:, :x.shape[1]]


def plain_gn(d):
    case, dt = d["case"], d["x"].dtype
    G, C = case["groups"], case["channels"]
    y, dx = torch.empty_like(d["x"]), torch.empty_like(d["x"])
    dgamma, dbeta = torch.zeros(C, device="cuda"), torch.zeros(C, device="cuda")
    saved = plain_saved(d["x"]) if case["ckpt"] else d["x"]

    def activated(xh):
        z = xh * d["gamma"] + d["beta"]
        if case["act"] == "relu":
            return torch.where(z > 0, z, torch.zeros_like(z)), (z > 0).float()
        if case["act"] == "silu":
            s = 1.0 / (1.0 + torch.exp(-z))
            return z * s, s * (1.0 + z * (1.0 - s))
        return z, torch.ones_like(z)

    i = 0
    for n in d["lens"]:
        rows, i = slice(i, i + n), i + n
        if not n:
            continue
        x = d["x"][rows].float().view(n, G, C // G)
        mean = x.mean((0, 2), keepdim=True)
        r = torch.rsqrt(((x - mean) ** 2).mean((0, 2), keepdim=True) + EPS)
        y[rows] = activated(((x - mean) * r).view(n, C))[0].to(dt)
        if not case["train"]:
            continue
        xh = (saved[rows].float().view(n, G, C // G) - mean) * r
        gz = d["dy"][rows].float() * activated(xh.view(n, C))[1]
        dgamma += (gz * xh.view(n, C)).sum(0)
        dbeta += gz.sum(0)
        h = (gz * d["gamma"]).view(n, G, C // G)
        g = r * (h - h.mean((0, 2), keepdim=True) - xh * (h * xh).mean((0, 2), keepdim=True))
        g = g.view(n, C)
        dx[rows] = (g + d["dres"][rows].float() if d["dres"] is not None else g).to(dt)
    return dict(y=y, dx=dx, dgamma=dgamma, dbeta=dbeta) if case["train"] else y


def plain_ckpt(d):
    saved = plain_saved(d["x"])
    if not d["case"]["out"]:
        return saved.to(d["x"].dtype)
    return saved.t() @ d["da"].float()


# -- what a pass cannot do without -------------------------------------------

def work(case):
    e = 4 if case["dtype"] == "f32" else 2
    m = case["rows"]
    if case["op"] == "rope":
        n, times = m * (case["heads"] + case["kv_heads"]) * case["head_dim"], 2 if case["train"] else 1
        return dict(bytes=times * (2 * e * n + 16 * m), flops=times * 3.0 * n)
    C = case["channels"]
    n = m * C
    if case["op"] == "gn":
        if not case["train"]:
            return dict(bytes=2 * e * n + 8 * C, flops=10.0 * n)
        # x and dy read once, y and dx written once
        return dict(bytes=(4 + (1 if case["res"] else 0)) * e * n + 16 * C, flops=35.0 * n)
    held = n + m * -(-C // BLOCK)  # codes and exponents, written once and read once
    if not case["out"]:
        return dict(bytes=2 * e * n + 2 * held, flops=6.0 * n)
    return dict(bytes=e * n + 2 * held + e * m * case["out"] + 4 * C * case["out"], flops=2.0 * n * case["out"])


# -- the same in 64 bits -------------------------------------------------------

def exact(case, seed):
    d = data(case, seed)
    return globals()["exact_" + case["op"]](case, d)


def exact_rope(case, d):
    """A pair as a complex number, turned by its angle."""
    P, out = sum(sections(case)), []
    sides = [(t, 1.0) for t in (d["q"], d["k"])] + ([(t, -1.0) for t in (d["dq"], d["dk"])] if case["train"] else [])
    for t, sign in sides:
        if t is None:
            continue
        y = t.double().clone()
        p = 0
        for a, s in enumerate(sections(case)):
            for _ in range(s):
                i, j = (p, p + P) if case["halves"] else (2 * p, 2 * p + 1)
                turn = sign * d["coords"][:, 1 + a].double() * d["freqs"][p].double()
                z = torch.complex(y[..., i], y[..., j]) * torch.polar(torch.ones_like(turn), turn)[:, None]
                y[..., i], y[..., j] = z.real, z.imag
                p += 1
        out.append(y)
    return out if len(out) > 1 else out[0]


def exact_saved(x):
    """Block by block: steps of the power of two of which 64 to 127 reach the largest value, and the nearest of them."""
    out = x.double().clone()
    for c in range(0, x.shape[1], BLOCK):
        b = out[:, c:c + BLOCK]
        top = b.abs().amax(1, keepdim=True)
        over = torch.where(top > 0, top / torch.frexp(top)[0], torch.ones_like(top))  # the power of two above it
        step = (over / 128.0).clamp(min=math.ldexp(1.0, -24 if x.dtype == torch.float16 else -126))
        b.copy_(torch.round(b / step).clamp(-127, 127) * step)
    return out


def exact_gn(case, d):
    G, x64 = case["groups"], d["x"].double()
    gamma, beta = d["gamma"].double(), d["beta"].double()
    act = dict(relu=torch.relu, silu=torch.nn.functional.silu, none=lambda t: t)[case["act"]]
    y, dx = torch.zeros_like(x64), torch.zeros_like(x64)
    dgamma, dbeta = torch.zeros_like(gamma), torch.zeros_like(beta)
    saved = exact_saved(d["x"]) if case["ckpt"] else x64
    i = 0
    for n in d["lens"]:
        rows, i = slice(i, i + n), i + n
        if not n:
            continue
        x = x64[rows].reshape(n, G, -1)
        var, mean = torch.var_mean(x, dim=(0, 2), correction=0, keepdim=True)
        dev = torch.sqrt(var + EPS)
        y[rows] = act(((x - mean) / dev).reshape(n, -1) * gamma + beta)
        if not case["train"]:
            continue
        # the output as a function of the normalized values, gamma and beta; then through the normalization, whose
        # statistics are the forward's
        xh = ((saved[rows].reshape(n, G, -1) - mean) / dev).reshape(n, -1).requires_grad_()
        leaf = [xh, gamma.clone().requires_grad_(), beta.clone().requires_grad_()]
        h, gg, gb = torch.autograd.grad(act(leaf[0] * leaf[1] + leaf[2]), leaf, d["dy"][rows].double())
        dgamma += gg
        dbeta += gb
        h, xh = h.reshape(n, G, -1), xh.detach().reshape(n, G, -1)
        g = (h - h.mean((0, 2), keepdim=True) - xh * (h * xh).mean((0, 2), keepdim=True)) / dev
        dx[rows] = g.reshape(n, -1)
        if d["dres"] is not None:
            dx[rows] += d["dres"][rows].double()
    return dict(y=y, dx=dx, dgamma=dgamma, dbeta=dbeta) if case["train"] else y


def exact_ckpt(case, d):
    saved = exact_saved(d["x"])
    return torch.mm(saved.t(), d["da"].double()) if case["out"] else saved
