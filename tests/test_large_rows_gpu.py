"""The embedding and the layer norm where a launch has more rows than workgroups along a direction, or more bytes than the
memory-side cache (nontemporal stores); compared on the GPU with elementary torch operations in 64 bits.

Tolerances: a lookup is one product in fp32 and one rounding, which torch's own product makes as well.  The layer norm's are
those of test_layer_norm_offset_gpu.py; h = x + y adds its own rounding, 2^-24 (|x| + |y|) r, to n.
"""
import pytest
import torch

from matrices import DT, half

pytestmark = pytest.mark.gpu

ARITH = 2.0 ** -17
EPS = 1e-5


def padded(rows, H, dtype, pad, seed, mean=0.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    wide = torch.empty((rows, H + pad), dtype=DT[dtype], device="cuda")
    for i in range(0, rows, 1 << 20):   # (no fp32 copy of all of it)
        part = wide[i:i + (1 << 20)]
        part.copy_(torch.randn(part.shape, generator=g, device="cuda") + mean)
    return wide[:, :H]


@pytest.mark.parametrize("rows,V,H,dtype,pad", [(33000, 500, 4099, "bf16", 5), (17000, 500, 4099, "f32", 3), (2_300_000, 70, 60, "bf16", 0),
                                                ((1 << 24) + 1000, 40, 3, "bf16", 0), ((1 << 22) + 77, 40, 130, "f32", 1), (140_000, 90, 1001, "bf16", 1)])
def test_lookup(rows, V, H, dtype, pad):
    import paper_2410_10989_amd as flce
    print(f"case lookup {rows} {V} {H} {dtype}", flush=True)
    table = padded(V, H, dtype, 0, 1)
    tokens = torch.randint(-3, V + 3, (rows,), device="cuda", generator=torch.Generator(device="cuda").manual_seed(2))
    wide = torch.full((rows, H + pad), 77.0, dtype=DT[dtype], device="cuda")
    flce.flce_embedding_fwd(table, tokens, scale=1.7, ignore_index=4, out=wide[:, :H])
    live = (tokens >= 0) & (tokens < V) & (tokens != 4)
    scaled = torch.cat([(table.float() * 1.7).to(DT[dtype]), torch.zeros(1, H, dtype=DT[dtype], device="cuda")])
    want = torch.where(live, tokens, V)
    for i in range(0, rows, 1 << 21):
        assert torch.equal(wide[i:i + (1 << 21), :H], scaled[want[i:i + (1 << 21)]])
    assert (wide[:, H:] == 77.0).all()


def test_gradient_of_more_pieces_than_workgroups():
    """2^27 rows: 2^22 pieces, 2^21 groups of them, and lists of the sort that are taken in turns.  Small whole numbers: every
    order of additions gives the same sums."""
    import paper_2410_10989_amd as flce
    rows, V = (1 << 27) + 77, 300
    g = torch.Generator(device="cuda").manual_seed(3)
    tokens = torch.randint(-1, V + 1, (rows,), device="cuda", generator=g)
    dout = torch.randint(-8, 9, (rows, 1), device="cuda", generator=g, dtype=torch.int32).float()
    ws = torch.empty(flce.flce_embedding_workspace_bytes(rows, V, 1, torch.float32), dtype=torch.uint8, device="cuda")
    got = flce.flce_embedding_bwd(dout, tokens, V, workspace=ws)
    live = (tokens >= 0) & (tokens < V)
    want = torch.bincount(torch.where(live, tokens, V), weights=dout[:, 0].double(), minlength=V + 1)[:V]
    assert want.abs().max() < 2 ** 24 and torch.equal(got[:, 0].double(), want)


def inside(name, got, ref, slack, mag, dtype):
    over = (got.double() - ref).abs() - (half(dtype) * (1 + slack) * ref.abs() + slack * (1 + half(dtype)) * mag + 2.0 ** -126)
    assert got.isfinite().all() and over.max().item() <= 0, (name, over.argmax().item(), over.max().item())


def statistics(h):
    d = h - h.mean(1, keepdim=True)
    r = 1 / torch.sqrt((d * d).mean(1, keepdim=True) + torch.tensor(EPS).double().item())
    return d * r, r, (d.abs() + d.abs().mean(1, keepdim=True) + 2.0 ** -19 * h.abs().mean(1, keepdim=True)) * r


LARGE = [(9000, 4099, "bf16", 5), (4600, 4099, "f32", 3), (300_000, 130, "bf16", 1), (70_000, 1000, "bf16", 0), (2500, 14001, "bf16", 1),
         (1300, 14001, "f32", 0), (20_000, 2001, "bf16", 3), (10_000, 2001, "f32", 0),
         (12_000, 3001, "bf16", 0), (6000, 3001, "f32", 1), (4000, 16401, "bf16", 3), (2100, 16401, "f32", 1), ((1 << 24) + 777, 8, "bf16", 0)]


@pytest.mark.parametrize("rows,H,dtype,pad", LARGE)
def test_layer_norm_forward(rows, H, dtype, pad):
    import paper_2410_10989_amd as flce
    print(f"case forward {rows} {H} {dtype}", flush=True)
    x, y = padded(rows, H, dtype, pad, 4, 0.5), padded(rows, H, dtype, 0, 5)
    gamma, beta = padded(2, H, dtype, 0, 6, 1.0)
    wide = torch.full((2, rows, H + pad), 77.0, dtype=DT[dtype], device="cuda")
    flce.flce_layer_norm_fwd(x, y, gamma, beta, EPS, h=wide[0, :, :H], n=wide[1, :, :H])
    step = max(1, (1 << 26) // H)
    for i in range(0, rows, step):
        a, b = x[i:i + step].double(), y[i:i + step].double()
        inside("h", wide[0, i:i + step, :H], a + b, ARITH, a.abs() + b.abs(), dtype)
        xh, r, mag = statistics(a + b)
        g = gamma.double()
        inside("n", wide[1, i:i + step, :H], xh * g + beta.double(), ARITH,
               g.abs() * (mag + 2.0 ** -7 * (a.abs() + b.abs() + (a.abs() + b.abs()).mean(1, keepdim=True)) * r) + (g * xh).abs() + beta.double().abs(), dtype)
    assert (wide[:, :, H:] == 77.0).all()


@pytest.mark.parametrize("rows,H,dtype,pad", LARGE)
def test_layer_norm_backward(rows, H, dtype, pad):
    """Sums over rows: a workgroup adds up its rows one after the other, 1 / 128 of all of them at most (and 16 of those
    that share its LDS), 2^-24 of the magnitudes each."""
    import paper_2410_10989_amd as flce
    print(f"case backward {rows} {H} {dtype}", flush=True)
    h, dn, dh = padded(rows, H, dtype, pad, 7, 0.5), padded(rows, H, dtype, 0, 8), padded(rows, H, dtype, pad, 9)
    gamma = padded(1, H, dtype, 0, 10, 1.0)[0]
    wide = torch.full((rows, H + pad), 77.0, dtype=DT[dtype], device="cuda")
    _, dgamma, dbeta = flce.flce_layer_norm_bwd(h, dn, dh, gamma, True, EPS, dx=wide[:, :H])
    step = max(1, (1 << 26) // H)
    sums = torch.zeros(4, H, dtype=torch.float64, device="cuda")   # of dgamma and dbeta, and of their magnitudes
    for i in range(0, rows, step):
        n, res = dn[i:i + step].double(), dh[i:i + step].double()
        xh, r, mag = statistics(h[i:i + step].double())
        u, xm = n * gamma.double(), xh.abs() + mag
        dx = res + r * (u - u.mean(1, keepdim=True) - xh * (u * xh).mean(1, keepdim=True))
        inside("dx", wide[i:i + step, :H], dx, ARITH,
               res.abs() + r * (u.abs() + u.abs().mean(1, keepdim=True) + 2 * xm * (u.abs() * xm).mean(1, keepdim=True)), dtype)
        for k, v in enumerate((n * xh, n, n.abs() * xm, n.abs())):
            sums[k] += v.sum(0)
    assert (wide[:, H:] == 77.0).all()
    slack = ARITH + (rows / 128 + 64) * 2.0 ** -24
    inside("dgamma", dgamma, sums[0], slack, sums[2], dtype)
    inside("dbeta", dbeta, sums[1], slack, sums[3], dtype)
