"""Products in 8-bit integers: the quantisation of rows and the product with a
scale for each token and channel, against plain 64-bit restatements.

Tolerances (derived from the arithmetic):
* quantised rows: whole numbers, equal; the scale is one float32 division, equal.
* product, bf16: the integer sums are exact below 2^24 (K 127^2 < 2^24 for K <=
  1040; random rows stay below it at every K here), the scales, the bias and the
  residual add a few roundings of 2^-24 of the largest term, the output is rounded once: per element
  2^-8 |y| + 2^-20 (|product| + |bias| + |resid|).  GELU: the fast exponential is
  good to 2^-20 relative over its range here, within the same bound.
* product, fp32: per element 2^-20 of the same terms.
* sums past 2^24 (every number +-127): each of the K / 16 additions of the tensor core
  may drop 2^-23 of the sum: 2^-23 K / 16 relative.
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a CUDA GPU", allow_module_level=True)

from paper_2604_20289_gb300 import xcache as xb  # noqa: E402

DEV = torch.device("cuda")
F64 = torch.float64


def tdt(dtype):
    return torch.bfloat16 if dtype == "bf16" else torch.float32


def rand(shape, seed, std=1.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return std * torch.randn(*shape, generator=g, device=DEV)


def plain_quantize(x):
    """(whole numbers, scale) in 64 bits."""
    x = x.to(F64)
    a = x.abs().amax(dim=1, keepdim=True)
    q = torch.where(a > 0, torch.round(127 * x / a), torch.zeros_like(x))
    return q, (a.float() / torch.full_like(a, 127, dtype=torch.float32)).squeeze(1)


def quantize(x, dtype):
    q = torch.full(x.shape, 55, dtype=torch.int8, device=DEV)
    s = torch.full((x.shape[0],), -1.0, device=DEV)
    xb.op_quantize_rows(dtype, x, q, s)
    return q, s


# ------------------------------------------------------------- quantisation
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,K", [(1, 16), (3, 48), (5, 1024), (7, 1040), (130, 4096), (9, 4112), (33, 8192), (4, 8208),
                                 (2, 16384), (3, 20000), (2, 131072)])
def test_rows_are_quantised(dtype, M, K):
    x = (rand((M, K), K + M) * torch.exp(2 * rand((M, 1), K))).to(tdt(dtype))
    q, s = quantize(x, dtype)
    rq, rs = plain_quantize(x)
    assert torch.equal(q.to(F64), rq)
    assert torch.equal(s, rs)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,K", [(5, 12288), (5, 24576), (5, 12016), (5, 24032), (305, 2064), (305, 8208), (609, 2064), (700, 272), (1300, 12288)])
def test_rows_at_the_ends_of_shared_memory_and_of_few(dtype, M, K):
    """Rows that fill the shared memory of a CTA, or just do not, and row counts on either side of the rules."""
    x = (rand((M, K), M + K) * torch.exp(2 * rand((M, 1), K))).to(tdt(dtype))
    q, s = quantize(x, dtype)
    rq, rs = plain_quantize(x)
    assert torch.equal(q.to(F64), rq)
    assert torch.equal(s, rs)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_halves_go_to_even_numbers(dtype):
    """Every x = a (k + 1/2) / 127 that the type holds, and its neighbours: a = 127 2^e, where the halves are exact, and
    x = a / 2 for every a of 8 bits, which is 63.5 steps."""
    rows = []
    for a in (127.0, 127.0 * 2 ** 20, 127.0 * 2 ** -30):
        k = torch.arange(-127, 127, device=DEV, dtype=F64) + 0.5
        rows.append(torch.cat([torch.tensor([a], device=DEV, dtype=F64), k * a / 127, torch.zeros(1, device=DEV, dtype=F64)]))
    for m in range(128, 256):
        row = torch.zeros(256, device=DEV, dtype=F64)
        row[0], row[1], row[2] = m, m / 2, -m / 2
        rows.append(row)
    x = torch.stack(rows).to(tdt(dtype))
    if dtype == "f32":                                 # and the values next to the halves
        up = torch.nextafter(x, torch.full_like(x, 1e30))
        x = torch.cat([x, torch.cat([x[:, :1], up[:, 1:]], dim=1)])
    q, s = quantize(x, dtype)
    rq, rs = plain_quantize(x)
    assert torch.equal(q.to(F64), rq) and torch.equal(s, rs)
    assert q[3 + 5, 1].item() == 64 and q[3 + 5, 2].item() == -64      # 63.5 -> 64


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_sizes_at_the_ends_of_the_range(dtype):
    x = torch.zeros(8, 64, device=DEV)
    big = torch.finfo(tdt(dtype)).max
    x[0, 3], x[0, 5], x[0, 7] = big, -big / 2, big / 254
    x[1, 0], x[1, 1] = 1e-38, -3e-39
    x[2, 0], x[2, 1] = 2.0 ** -133, 2.0 ** -132        # subnormal in both types
    x[4, 9] = float("inf")
    x[5, 9], x[5, 10] = float("nan"), 1.0
    x[6, 0], x[6, 1] = 1e30, 1e-30
    x[7] = -0.0
    x = x.to(tdt(dtype))
    q, s = quantize(x, dtype)
    fine = [0, 1, 2, 3, 6, 7]
    rq, rs = plain_quantize(x[fine])
    assert torch.equal(q[fine].to(F64), rq)
    assert torch.equal(s[fine], rs)
    assert s[4].isnan() and s[5].isnan() and not q[4].any() and not q[5].any()


def test_no_rows():
    q, s = quantize(torch.empty(0, 32, dtype=torch.bfloat16, device=DEV), "bf16")
    assert q.shape == (0, 32) and s.shape == (0,)


# ------------------------------------------------------------------ product
EPI = {"bias": xb.XC_EPI_BIAS, "gelu": xb.XC_EPI_GELU, "resid": xb.XC_EPI_RESID_GATE}


def operands(dtype, M, N, K, seed=0):
    x = (rand((M, K), seed) * torch.exp(0.5 * rand((M, 1), seed + 1))).to(tdt(dtype))
    q, s = plain_quantize(rand((N, K), seed + 2, K ** -0.5).bfloat16())
    return dict(x=x, wq=q.to(torch.int8), ws=s, bias=rand((N,), seed + 3, 0.05), gate=1 + 0.2 * rand((N,), seed + 4),
                resid=rand((M, N), seed + 5).to(tdt(dtype)))


def plain_linear(o, epi, a_scale=None, rows=None):
    """(y, the size of its terms) in 64 bits."""
    if a_scale is None:
        q, s = plain_quantize(o["x"])
    else:
        q, s = o["x"].to(F64), a_scale
    p = (q @ o["wq"].to(F64).t()) * s.to(F64)[:, None] * o["ws"].to(F64)
    y = p + o["bias"].to(F64)
    size = p.abs() + o["bias"].abs().to(F64)
    if epi == "gelu":
        y = 0.5 * y * (1 + torch.tanh((2 / np.pi) ** 0.5 * (y + 0.044715 * y ** 3)))
    elif epi == "resid":
        y = o["resid"].to(F64) + o["gate"].to(F64) * y
        size = size * o["gate"].abs().to(F64) + o["resid"].abs().to(F64)
    return y, size


def run_linear(dtype, o, epi, a_scale=None, **kw):
    out = torch.full((o["x"].shape[0], o["wq"].shape[0]), 7.0, dtype=tdt(dtype), device=DEV)
    more = dict(gate=o["gate"], resid=o["resid"]) if epi == "resid" else {}
    xb.op_linear_i8(dtype, EPI[epi], o["x"], o["wq"], o["ws"], o["bias"], out, a_scale=a_scale, **more, **kw)
    return out


def near(out, ref, size):
    half = 2.0 ** -8 if out.dtype is torch.bfloat16 else 0.0
    off = (out.to(F64) - ref).abs() - half * ref.abs() - 2.0 ** -20 * size
    assert off.max().item() <= 0, f"over the bound by {off.max().item():.3e} at {divmod(off.argmax().item(), out.shape[1])}"


SHAPES = [(1, 128, 128), (4, 5, 16), (1, 1, 16), (3, 100, 48), (16, 128, 64), (17, 256, 80), (33, 130, 5120), (64, 1024, 640),
          (100, 384, 1040), (128, 4000, 144), (129, 640, 256), (250, 200, 2048), (257, 72, 512), (300, 1536, 1536), (513, 129, 96),
          (1031, 1000, 304), (40, 3000, 13824), (2000, 2560, 192)]


@pytest.mark.parametrize("dtype,epi", [("bf16", "bias"), ("bf16", "gelu"), ("bf16", "resid"), ("f32", "bias"), ("f32", "resid"),
                                       ("f32", "gelu")])
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_product(dtype, epi, M, N, K):
    o = operands(dtype, M, N, K, seed=M + N + K)
    out = run_linear(dtype, o, epi)
    near(out, *plain_linear(o, epi))
    assert xb.op_device_error() == 0


@pytest.mark.parametrize("M,N,K", [(12960, 1536, 1536), (4, 15360, 5120), (331, 5120, 13824), (4320, 6000, 1040)])
def test_product_large(M, N, K):
    o = operands("bf16", M, N, K)
    near(run_linear("bf16", o, "gelu"), *plain_linear(o, "gelu"))
    assert xb.op_device_error() == 0


@pytest.mark.parametrize("M,N,K", [(3, 200, 48), (300, 1536, 1024)])
def test_product_of_tokens_quantised_before(M, N, K):
    o = operands("bf16", M, N, K)
    want = run_linear("bf16", o, "resid")
    q, s = quantize(o["x"], "bf16")
    o["x"] = q
    assert torch.equal(run_linear("bf16", o, "resid", a_scale=s), want)


def test_all_8_bit_numbers():
    """-128 too, on either side."""
    M, N, K = 37, 300, 1024
    g = torch.Generator(device=DEV).manual_seed(5)
    o = operands("f32", M, N, K)
    o["x"] = torch.randint(-128, 128, (M, K), generator=g, device=DEV).to(torch.int8)
    o["wq"] = torch.randint(-128, 128, (N, K), generator=g, device=DEV).to(torch.int8)
    s = torch.full((M,), 1.0, device=DEV)
    o["ws"], o["bias"] = torch.full((N,), 1.0, device=DEV), torch.zeros(N, device=DEV)
    assert torch.equal(run_linear("f32", o, "bias", a_scale=s).to(F64), plain_linear(o, "bias", s)[0])


def test_sums_past_24_bits():
    M, N, K = 20, 256, 13824
    o = operands("f32", M, N, K)
    o["x"] = torch.full((M, K), 3.0, device=DEV)
    o["x"][::2] *= -1
    o["wq"] = torch.full((N, K), 127, dtype=torch.int8, device=DEV)
    out, (ref, _) = run_linear("f32", o, "bias"), plain_linear(o, "bias")
    assert ((out.to(F64) - ref).abs() / ref.abs()).max().item() <= 2.0 ** -23 * K / 16


@pytest.mark.parametrize("M,N,K", [(4, 300, 13824), (12, 256, 5120), (32, 100, 2064)])
def test_sums_past_24_bits_of_few_tokens(M, N, K):
    """The kernel of few tokens: the same bound, K / 16 additions that may drop 2^-23 of the sum each."""
    o = operands("f32", M, N, K)
    o["x"] = torch.full((M, K), 3.0, device=DEV)
    o["x"][::2] *= -1
    o["wq"] = torch.full((N, K), 127, dtype=torch.int8, device=DEV)
    assert xb.op_linear_i8_workspace_bytes(M, N, K) == 0
    out, (ref, _) = run_linear("f32", o, "bias"), plain_linear(o, "bias")
    assert ((out.to(F64) - ref).abs() / ref.abs()).max().item() <= 2.0 ** -23 * K / 16


def test_a_row_that_is_not_finite_spoils_only_its_own_outputs():
    o = operands("bf16", 40, 256, 512)
    o["x"][7, 100], o["x"][20, 3] = float("nan"), float("-inf")
    out = run_linear("bf16", o, "bias")
    ok = [i for i in range(40) if i not in (7, 20)]
    assert out[7].isnan().all() and out[20].isnan().all()
    o["x"] = o["x"][ok]
    near(out[ok], *plain_linear(o, "bias"))


def test_residual_in_place_and_equal_runs():
    o = operands("bf16", 331, 1160, 2064)
    want = run_linear("bf16", o, "resid")
    for _ in range(3):
        assert torch.equal(run_linear("bf16", o, "resid"), want)
    io = o["resid"].clone()
    xb.op_linear_i8("bf16", xb.XC_EPI_RESID_GATE, o["x"], o["wq"], o["ws"], o["bias"], io, gate=o["gate"], resid=io)
    assert torch.equal(io, want)


def test_no_tokens():
    o = operands("bf16", 0, 256, 64)
    assert run_linear("bf16", o, "bias").shape == (0, 256)


def test_weights_made_by_the_kernel_before_the_product():
    """The product reads its weights before it waits for the kernel ahead of it."""
    M, N, K = 8, 4096, 4096
    o = operands("bf16", M, N, K)
    w = rand((N, K), 9).bfloat16()
    for i in range(20):
        wi = torch.roll(w, i, 0)
        xb.op_quantize_rows("bf16", wi, o["wq"], o["ws"])
        out = run_linear("bf16", o, "bias")
        if i % 5 == 4:
            near(out, *plain_linear(dict(o), "bias"))


def test_every_weight_reaches_its_token():
    """One-hot tokens show each weight by itself; several rounds, as a slot refilled too early shows only now and then."""
    M, N, K = 12960, 1536, 1536
    w = operands("bf16", 1, N, K)["wq"]
    x = torch.zeros(M, K, device=DEV)
    m = torch.arange(M, device=DEV)
    x[m, m % K] = 127.0
    x = x.bfloat16()
    one, zero, out = torch.full((N,), 1 / 127.0, device=DEV), torch.zeros(N, device=DEV), torch.empty(M, N, dtype=torch.bfloat16, device=DEV)
    want = w.t()[m % K].float()
    for _ in range(10):
        xb.op_linear_i8("bf16", xb.XC_EPI_BIAS, x, w, one, zero, out)
        assert torch.equal(torch.round(out.float()), want)


def test_streams_and_graphs():
    o = operands("bf16", 50, 640, 512)
    want = run_linear("bf16", o, "bias")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out = torch.empty_like(want)
    xb.op_linear_i8("bf16", EPI["bias"], o["x"], o["wq"], o["ws"], o["bias"], out, stream=side)
    side.synchronize()
    assert torch.equal(out, want)
    graphs, outs = [], []
    for _ in range(2):                                 # two graphs, each with a workspace of its own
        g = torch.cuda.CUDAGraph()
        outs.append(torch.zeros_like(want))
        with torch.cuda.graph(g):
            xb.op_linear_i8("bf16", EPI["bias"], o["x"], o["wq"], o["ws"], o["bias"], outs[-1])
        graphs.append(g)
    with torch.cuda.stream(side):
        graphs[1].replay()
    graphs[0].replay()
    torch.cuda.synchronize()
    assert torch.equal(outs[0], want) and torch.equal(outs[1], want)
    o["x"].copy_(rand(tuple(o["x"].shape), 99).bfloat16())
    graphs[0].replay()
    torch.cuda.synchronize()
    near(outs[0], *plain_linear(o, "bias"))


def test_refusals():
    o = operands("bf16", 40, 64, 64)
    out = torch.empty(40, 64, dtype=torch.bfloat16, device=DEV)
    args = dict(A=o["x"], Wq=o["wq"], w_scale=o["ws"], bias=o["bias"], out=out)

    def call(epi="bias", **kw):
        a = dict(args)
        a.update({k: v for k, v in kw.items() if k in a})
        more = {k: v for k, v in kw.items() if k not in a}
        xb.op_linear_i8("bf16", EPI[epi], a["A"], a["Wq"], a["w_scale"], a["bias"], a["out"], **more)

    call()
    for bad in (dict(A=o["x"].float()), dict(A=o["x"].t()), dict(Wq=o["wq"].float()), dict(Wq=o["wq"][:, :48]),
                dict(w_scale=o["ws"].double()), dict(bias=o["bias"][:63]), dict(out=out.float()), dict(out=out.t()),
                dict(A=o["x"].cpu()), dict(out=out.cpu()), dict(resid=o["resid"].float()), dict(gate=o["gate"].double()),
                dict(a_scale=o["ws"][:40])):
        with pytest.raises(ValueError):
            call(**bad)
    for bad in (dict(epi="resid"), dict(workspace=torch.empty(16, dtype=torch.uint8, device=DEV))):
        with pytest.raises(xb.XCacheError) as e:
            call(**bad)
        assert e.value.status == xb.XC_EINVAL
    with pytest.raises(xb.XCacheError):
        call(A=torch.zeros(40, 40, dtype=torch.bfloat16, device=DEV), Wq=torch.zeros(64, 40, dtype=torch.int8, device=DEV))
    with pytest.raises(ValueError):
        xb.op_quantize_rows("f32", o["x"], torch.empty_like(o["x"], dtype=torch.int8), torch.empty(40, device=DEV))
