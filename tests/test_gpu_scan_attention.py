"""The attention layer over packed scans against the same layer in float64 with its gradients from autograd, on the
stride-8 and stride-16 voxels that the network's own plan gives."""
import numpy as np
import pytest
import torch

from paper_2007_16100_amd import synth

pytestmark = pytest.mark.gpu
TD = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
# the framework's normwise bounds of chains of layers (16-bit: rounded between the layers)
TOL = {"f32": 1e-5, "bf16": 2e-2, "f16": 4e-3}


@pytest.fixture(scope="module")
def spv():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2007_16100_amd import spv as s
    s.lib()
    return s


@pytest.fixture(scope="module")
def voxels(spv):
    """Coordinates of two cropped sweeps (and an empty scan between them) at strides 8 and 16."""
    from paper_2007_16100_amd.spvcnn import SPVCNN
    a, b = synth.lidar_sweep(1002)[::40], synth.lidar_sweep(1003)[::25]
    xyz = torch.from_numpy(np.concatenate([a, b])).cuda()
    batch = torch.cat([torch.zeros(len(a)), torch.full((len(b),), 2.0)]).to(torch.int32).cuda()
    plan, _ = SPVCNN(synth.spvcnn_params(3, "bf16"), "bf16", 0.05).plan(xyz, batch)
    return plan.coords


def params(C, H, K, D, dtype, seed):
    g = torch.Generator().manual_seed(seed)

    def w(i, o):
        return (torch.randn(i, o, generator=g) / i ** 0.5).to(TD[dtype]).cuda()
    return dict(gamma=(1 + 0.1 * torch.randn(C, generator=g)).cuda(), beta=(0.1 * torch.randn(C, generator=g)).cuda(),
                Wq=w(C, H * D), Wk=w(C, K * D), Wv=w(C, K * D), Wo=w(H * D, C))


def plain(P, x, H, K, off, cap, slopes, coords, tokens=None, token_off=None, token_coords=None):
    """The layer in float64 on the CPU."""
    def ln(t):
        return torch.nn.functional.layer_norm(t, t.shape[1:], P["gamma"], P["beta"], 1e-5)
    own = tokens is None
    t, t_off, t_coords = (x, off, coords) if own else (tokens, token_off, token_coords)
    h = ln(x)
    q, k, v = ln(t) @ P["Wq"], h @ P["Wk"], h @ P["Wv"]
    D = q.shape[1] // H
    rows = []
    for b in range(len(off) - 1):
        i, j = slice(t_off[b], t_off[b + 1]), slice(off[b], off[b + 1])
        heads = []
        for a in range(H):
            g = a // (H // K)
            s = q[i, a * D:(a + 1) * D] @ k[j, g * D:(g + 1) * D].T / D ** 0.5
            s = cap * torch.tanh(s / cap) if cap else s
            if slopes is not None:
                s = s - slopes[a] * (t_coords[i, None, 1:] - coords[None, j, 1:]).abs().sum(-1)
            heads.append(torch.softmax(s, 1) @ v[j, g * D:(g + 1) * D] if s.shape[1] else torch.zeros(s.shape[0], D))
        rows.append(torch.cat(heads, 1))
    return t + torch.cat(rows) @ P["Wo"]


def normwise(got, want):
    return ((got.detach().double().cpu() - want).abs().max() / want.abs().max()).item()


@pytest.mark.parametrize("dtype,C,H,K,cap", [("bf16", 256, 8, 8, 0.0), ("bf16", 96, 3, 1, 5.0), ("f16", 128, 4, 2, 0.0),
                                             ("f32", 64, 2, 2, 3.0)])
def test_layer_and_gradients(spv, voxels, dtype, C, H, K, cap):
    from paper_2007_16100_amd.scan_attention import ScanAttention, scan_offsets
    coords = voxels[4 if C == 256 else 3].contiguous()
    n = coords.shape[0]
    print(f"layer n={n} C={C} H={H} K={K} {dtype}", flush=True)
    off = scan_offsets(coords, 3)
    b = coords[:, 0].cpu()
    assert off.tolist() == [0, int((b < 1).sum()), int((b < 2).sum()), n] and off[1] == off[2]
    slopes = torch.tensor([2.0 ** -(2 + h) for h in range(H)]).cuda()
    P = params(C, H, K, C // H, dtype, C)
    layer = ScanAttention(P, H, K, cap, slopes)
    g = torch.Generator().manual_seed(9)
    x, dy = (torch.randn(n, C, generator=g).to(TD[dtype]).cuda() for _ in range(2))
    saved = {}
    y = layer.forward(x, off, coords, save=saved)
    grads = layer.backward(saved, dy)
    assert torch.equal(y, layer.forward(x, off, coords))

    Pd = {k: t.double().cpu().requires_grad_() for k, t in P.items()}
    xd = x.double().cpu().requires_grad_()
    want = plain(Pd, xd, H, K, off.tolist(), cap, slopes.double().cpu(), coords.double().cpu())
    assert normwise(y, want.detach()) <= TOL[dtype]
    names = list(Pd)
    ref = torch.autograd.grad(want, [Pd[k] for k in names] + [xd], dy.double().cpu())
    for k, r in zip(names + ["x"], ref):
        print(k, normwise(grads[k][: r.shape[0]], r), flush=True)
        # weight gradients are sums over up to a thousand rows
        assert normwise(grads[k][: r.shape[0]], r) <= TOL[dtype] * (2 if k != "x" else 1), k


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_tokens_read_their_scans(spv, voxels, dtype):
    """Two tokens a scan over its voxels; those of the empty scan pass through."""
    from paper_2007_16100_amd.scan_attention import ScanAttention, scan_offsets
    coords = voxels[3].contiguous()
    n, C, H, K = coords.shape[0], 128, 4, 2
    off, t_off = scan_offsets(coords, 3), torch.tensor([0, 2, 4, 6], dtype=torch.int32).cuda()
    P = params(C, H, K, 32, dtype, 77)
    slopes = torch.full((H,), 0.05).cuda()
    g = torch.Generator().manual_seed(4)
    x, tok = torch.randn(n, C, generator=g).to(TD[dtype]).cuda(), torch.randn(6, C, generator=g).to(TD[dtype]).cuda()
    tc = torch.tensor([[b, 3 * i, -b, 0] for b in range(3) for i in range(2)], dtype=torch.int32).cuda()
    y = ScanAttention(P, H, K, 0.0, slopes).forward(x, off, coords, tok, t_off, tc)
    assert torch.equal(y[2:4], tok[2:4])
    Pd = {k: t.double().cpu() for k, t in P.items()}
    want = plain(Pd, x.double().cpu(), H, K, off.tolist(), 0.0, slopes.double().cpu(), coords.double().cpu(),
                 tok.double().cpu(), t_off.tolist(), tc.double().cpu())
    assert normwise(y, want) <= TOL[dtype]
    with pytest.raises(ValueError):
        ScanAttention(P, 3)
