"""Linear layers in 8-bit integers on the GPU: results, operands and kernels that no other test puts together.

The references and tolerances of products and norms are those of test_gpu_int.py; which kernel a
product takes is checked on the CPU (test_int_choice.py).
"""
import numpy as np
import pytest

from harness import dev_bf16, dev_f32, host_f32
from test_gpu_int import Codes, _check_norm, _linear_case, _sync
from workloads import bf16_round

pytestmark = pytest.mark.gpu

# one size for every kernel of a product, as test_int_choice.py has them
FEW = [(1, 520, 272), (16, 4100, 400), (30, 520, 272), (64, 4100, 400)]
SMALL = [(300, 700, 100), (389, 1280, 640), (500, 1500, 1600), (1300, 1300, 1300), (1100, 2570, 272)]
LARGE = [(1000, 5120, 144), (2400, 4000, 272), (2890, 5125, 400)]
LARGE_OTHER = [(1500, 4501, 300), (2300, 4101, 144), (3000, 5000, 400)]

FORMS = ([("bias", "bf16", ""), ("bias", "f32", ""), ("gelu", "bf16", "")] +
         [(e, o, r) for e in ("res", "gate") for o in ("bf16", "f32") for r in ("bf16", "f32")])


@pytest.fixture(scope="module")
def A(gpu):
    from paper_2606_15319_amd import ardit
    return ardit


@pytest.mark.parametrize("epi,out,res", FORMS)
@pytest.mark.parametrize("M,N,K", LARGE)
def test_every_result_of_the_large_tiles(A, M, N, K, epi, out, res):
    _linear_case(A, M, N, K, epi=epi, out=out, res=res, per=999)


@pytest.mark.parametrize("epi,out,res", [("gelu", "bf16", ""), ("res", "f32", "f32"), ("gate", "bf16", "f32")])
@pytest.mark.parametrize("M,N,K", LARGE_OTHER)
def test_the_large_tiles_at_other_widths(A, M, N, K, epi, out, res):
    _linear_case(A, M, N, K, epi=epi, out=out, res=res, per=777, pad=1)


class Product:
    """Operands of one product on the device."""

    def __init__(self, A, M, N, K, kind, per):
        import torch
        g = torch.Generator(device="cuda")
        g.manual_seed(M + N + K)
        self.A, self.M, self.N, self.kp = A, M, N, -(-K // 16) * 16
        self.K, self.per = K, per
        q = lambda r: torch.randint(-127, 128, (r, self.kp), device="cuda", generator=g).to(torch.int8)
        s = lambda n: 0.001 + 0.001 * torch.rand(n, device="cuda", generator=g)
        rn = lambda *n: torch.randn(n, device="cuda", generator=g)
        self.x, self.w, self.sx, self.sw = q(M), q(N), s(M), s(N)
        self.x[:, K:] = 0
        self.b, self.r = rn(N).bfloat16(), rn(M, N) if kind == "f32" else rn(M, N).bfloat16()
        self.mod, self.tab = rn(-(-M // per), 6, N), rn(6, N)
        self.type = A.F32 if kind == "f32" else A.BF16

    def run(self, y, res, gate, table):
        A = self.A
        kw = dict(mod=self.mod, mod_table=table, gate_row=2, rows_per_stream=self.per) if gate else {}
        A.ardit_int_linear(None, A.linear_desc(self.M, self.N, self.K, self.x, self.kp, self.sx, self.w, self.kp, self.sw,
                                               bias=self.b, res=res, res_type=self.type, ldr=self.N, **kw),
                           y, self.type, self.N)
        _sync()


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("gate", [False, True])
@pytest.mark.parametrize("M,N,K", FEW + SMALL + LARGE + LARGE_OTHER[:1])
def test_a_residual_under_the_result(A, M, N, K, gate, kind):
    """y over res: the bits of a result with a tensor of its own, in every kernel."""
    import torch
    p = Product(A, M, N, K, kind, max(1, M // 3))
    y = torch.empty_like(p.r)
    p.run(y, p.r, gate, p.tab)
    over = p.r.clone()
    p.run(over, over, gate, p.tab)
    assert torch.equal(y, over) and not torch.equal(y, p.r)


@pytest.mark.parametrize("M,N,K", FEW[1:2] + SMALL[1:3] + LARGE)
def test_a_gate_without_a_table(A, M, N, K):
    """mod alone is mod + 0."""
    import torch
    p = Product(A, M, N, K, "f32", max(1, M // 2))
    y, z = torch.empty_like(p.r), torch.empty_like(p.r)
    p.run(y, p.r, True, None)
    p.run(z, p.r, True, torch.zeros_like(p.tab))
    assert torch.equal(y, z)
    p.run(z, p.r, True, p.tab)
    assert not torch.equal(y, z)


# long rows, of which most hold a code that is decided again
@pytest.mark.parametrize("gate", [False, True])
@pytest.mark.parametrize("delta", ["bf16", "f32"])
@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("rows,dim,pad,by,per", [(65, 5120, 0, "mod", 30), (40, 5119, 0, "gain", None), (24, 8192, 0, "mod", 24),
                                                 (60, 1536, 8, "shift", 7), (50, 1535, 1, "plain", 50)])
def test_norm_of_a_sum_that_is_not_kept(A, rows, dim, pad, by, per, f32, delta, gate):
    _check_norm(A, rows, dim, f32=f32, delta=delta, gate=gate, by=by, per=per, pad=pad, kind="loud", keep=False)


@pytest.mark.parametrize("value", [np.inf, -np.inf, np.nan])
@pytest.mark.parametrize("where", ["gain", "shift", "scale", "gate", "table"])
@pytest.mark.parametrize("dim", [512, 77])
def test_norm_with_a_vector_that_is_no_number(A, where, value, dim):
    """An infinity or a NaN in a vector of stream 1: its rows have NaN scales and zero codes, the others what
    they have without it."""
    import torch
    rng = np.random.default_rng(3)
    per, rows = 9, 26
    x, d = (rng.standard_normal((rows, dim)).astype(np.float32) for _ in range(2))
    mod, tab = rng.standard_normal((3, 6, dim)).astype(np.float32), rng.standard_normal((6, dim)).astype(np.float32)
    gain = bf16_round(rng.standard_normal(dim).astype(np.float32)).astype(np.float32)
    xd, dd = dev_f32(x), dev_f32(d)

    def norm(mod, tab, gain):
        keep = [dev_f32(mod), dev_f32(tab), dev_bf16(gain)]
        kw = dict(gain=keep[2]) if where == "gain" else dict(shift_row=3, scale_row=4)
        c = Codes(rows, dim)
        h = torch.empty((rows, dim), device="cuda")
        A.ardit_int_norm(None, rows, dim,
                         A.norm_desc(xd, A.F32, dim, delta=dd, delta_type=A.F32, ldd=dim, h=h, ldh=dim, mod=keep[0],
                                     mod_table=keep[1], rows_per_stream=per, gate_row=5, **kw), c.q, c.ld, c.s)
        q, s = c.host()
        return q.copy(), s.copy(), host_f32(h)

    plain = norm(mod, tab, gain)
    assert np.isfinite(plain[1]).all()
    m, t, g = mod.copy(), tab.copy(), gain.copy()
    if where == "gain":
        g[dim // 2] = value
    elif where == "table":
        t[4, dim - 1] = value
    else:
        m[1, {"shift": 3, "scale": 4, "gate": 5}[where], dim - 1] = value
    got = norm(m, t, g)
    hit = np.ones(rows, bool) if where in ("gain", "table") else np.arange(rows) // per == 1
    assert np.isnan(got[1][hit]).all() and not got[0][hit].any()
    assert np.array_equal(got[0][~hit], plain[0][~hit]) and np.array_equal(got[1][~hit], plain[1][~hit])
    same = np.ones((rows, dim), bool)
    if where == "gate":
        same[hit, dim - 1] = False
        assert not np.isfinite(got[2][~same]).any()
    assert np.array_equal(got[2][same], plain[2][same])
