"""Operators around a layer's projections measured through the library's public entry points,
each beside its plain form in elementary torch operations: the residual's addition with the
RMS norm, the gated activation, the product in 8-bit floating point, and a whole MLP of them.

A case is a dict of plain values with an "op":
  norm    subspec_add_norm of M rows of K, bf16 out ("residual": with the addition)
  act     subspec_silu_mul of M rows of gate|up, I each, bf16 out
  linear  subspec_fp8_linear of M bf16 rows of K onto N columns of 8-bit weights
  mlp     add_norm into 8-bit rows, gate|up product, silu_mul into 8-bit rows, down product
"""
import math

import torch

own = False

DEV = "cuda"
EPS = 1e-6


def listed():
    return [
        # In front of a projection of a single-token step, 7B width: nothing but latency.
        dict(name="norm_7b_m1", op="norm", M=1, K=3584, residual=True),
        # A chain of 48 drafted tokens and the root, 32B width.
        dict(name="norm_32b_m49", op="norm", M=49, K=5120, residual=True),
        # A long prompt, 32B width.
        dict(name="norm_32b_m4096", op="norm", M=4096, K=5120, residual=True),
        # A draft pass of six leaves between gate|up and down, 7B.
        dict(name="act_7b_m6", op="act", M=6, I=18944),
        # A long prompt, 32B.
        dict(name="act_32b_m4096", op="act", M=4096, I=27648),
        # The output projection of a single-token step, 7B.
        dict(name="linear_7b_o_m1", op="linear", M=1, N=3584, K=3584),
        # The down projection over a short chain of drafted tokens, 32B.
        dict(name="linear_32b_down_m7", op="linear", M=7, N=5120, K=27648),
        # q|k|v in the verification of a tree of 48 levels of six and its root, 32B.
        dict(name="linear_32b_qkv_m289", op="linear", M=289, N=7168, K=5120),
        # gate|up over a ragged prompt, 7B.
        dict(name="linear_7b_gateup_m1000", op="linear", M=1000, N=37888, K=3584),
        # gate|up over a long prompt, 32B: bound by the matrix units.
        dict(name="linear_32b_gateup_m4096", op="linear", M=4096, N=55296, K=5120),
        # The MLP of a verification of a chain of 48 tokens, 7B.
        dict(name="mlp_7b_m49", op="mlp", M=49, K=3584, I=18944),
        # The MLP over a prompt, 32B.
        dict(name="mlp_32b_m2048", op="mlp", M=2048, K=5120, I=27648),
    ]


def _log_uniform(rng, lo, hi, step=1):
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(lo, min(hi, int(round(v / step)) * step))


def draw(rng):
    op = rng.choice(["norm", "act", "linear", "linear", "mlp"])
    M = _log_uniform(rng, 1, 4096)
    if op == "norm":
        return dict(op=op, M=M, K=_log_uniform(rng, 64, 16384, 8), residual=rng.random() < 0.8)
    if op == "act":
        return dict(op=op, M=M, I=_log_uniform(rng, 128, 27648, 8))
    most = 4096 * 55296 * 5120
    if op == "linear":
        K, N = _log_uniform(rng, 128, 27648, 128), _log_uniform(rng, 16, 55296, 16)
        return dict(op=op, M=max(1, min(M, most // (N * K))), N=N, K=K)
    K, I = _log_uniform(rng, 128, 8192, 128), _log_uniform(rng, 128, 27648, 128)
    return dict(op=op, M=max(1, min(M, most // (3 * K * I))), K=K, I=I)


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 1000003 + 31)
    return g


def _bf(g, *shape, scale=1.0):
    return torch.randn(shape, generator=g, device=DEV).mul_(scale).to(torch.bfloat16)


# --- 8-bit rows and weight tiles (include/subspec.h), written and read with torch ---------

def _power(e):
    """2^e in fp32 for whole e in -126 .. 127."""
    return ((e + 127) << 23).view(torch.float32)


def _quantize(x):
    """Codes (e4m3) and exponents (int32) of fp32 rows [R][K] with a scale for every 128."""
    b = x.view(x.shape[0], -1, 128)
    f, e = torch.frexp(b.abs().amax(-1, keepdim=True))  # largest = f 2^e, and 448 = 0.875 2^9
    e = (e - torch.where(f <= 0.875, 9, 8)).clamp_(min=-126).to(torch.int32)
    return (b * _power(-e)).to(torch.float8_e4m3fn).view(x.shape), e.squeeze(-1)


def _rounded(x):
    """The fp32 values that 8-bit rows of x stand for."""
    q, e = _quantize(x)
    return (q.view(x.shape[0], -1, 128).float() * _power(e)[..., None]).view(x.shape)


def _words(e):
    """Scale bytes [ceil(K / 512)][R][4] of exponents [R][K / 128]."""
    R, B = e.shape
    s = torch.full((R, (B + 3) // 4 * 4), 127, dtype=torch.uint8, device=DEV)
    s[:, :B] = (e + 127).to(torch.uint8)
    return s.view(R, -1, 4).permute(1, 0, 2).contiguous()


def _weights(g, N, K):
    """A projection [N][K] as weight tiles and scales; a few input channels are larger, as trained ones are."""
    w = torch.randn((N, K), generator=g, device=DEV).mul_(1.0 / math.sqrt(K))
    w[:, ::97] *= 4.0
    q, e = _quantize(w.to(torch.bfloat16).float())
    tiles = q.view(torch.uint8).view(N // 16, 16, K // 128, 2, 4, 16).permute(0, 2, 3, 4, 1, 5).contiguous()
    return tiles.view(-1), _words(e)


def _unpacked(tiles, words, N, K):
    """The fp32 values [N][K] of weight tiles."""
    q = tiles.view(N // 16, K // 128, 2, 4, 16, 16).permute(0, 4, 1, 2, 3, 5).contiguous()
    e = words.permute(1, 0, 2).reshape(N, -1)[:, :K // 128].int() - 127
    return (q.view(torch.float8_e4m3fn).view(N, K // 128, 128).float() * _power(e)[..., None]).view(N, K)


def prepare(case, seed):
    g, op, M = _gen(seed), case["op"], case["M"]
    e = lambda *shape, dtype=torch.bfloat16: torch.empty(shape, dtype=dtype, device=DEV)  # noqa: E731
    rows8 = lambda K: (e(M, K, dtype=torch.uint8), e((K + 511) // 512, M, dtype=torch.int32))  # noqa: E731
    if op == "act":
        return dict(case=case, gu=_bf(g, M, 2 * case["I"], scale=1.5), y=e(M, case["I"]))
    K = case["K"]
    x = _bf(g, M, K)
    if op == "linear":
        x[:, ::61] *= 8.0
        w, ws = _weights(g, case["N"], K)
        return dict(case=case, x=x, w=w, ws=ws, y=e(M, case["N"]))
    st = dict(case=case, x=x, res=None, sum=e(M, K), y=e(M, K),
              weight=(1.0 + 0.2 * torch.randn(K, generator=g, device=DEV)).to(torch.bfloat16))
    if op == "mlp" or case["residual"]:
        st["res"] = _bf(g, M, K, scale=4.0)  # a stream of many layers' sums, some channels far larger
        st["res"][:, ::113] *= 10.0
    if op == "mlp":
        I = case["I"]
        st["up"], st["up_s"] = _weights(g, 2 * I, K)
        st["down"], st["down_s"] = _weights(g, K, I)
        st["a"], st["a_s"] = rows8(K)
        st["h"], st["h_s"] = rows8(I)
        st["gu"] = e(M, 2 * I)
    return st


# --- one pass ----------------------------------------------------------------------------

def run(st):
    c = st["case"]
    op, M = c["op"], c["M"]
    if own:
        import paper_2509_18344_amd as ss
        if op == "norm":
            ss.subspec_add_norm(st["x"], st["res"], st["weight"], EPS, M, c["K"], st["sum"], st["y"], None, None)
            return dict(sum=st["sum"], y=st["y"])
        if op == "act":
            ss.subspec_silu_mul(st["gu"], M, c["I"], st["y"], None, None)
            return st["y"]
        if op == "linear":
            ss.subspec_fp8_linear(st["x"], None, st["w"], st["ws"], M, c["N"], c["K"], st["y"])
            return st["y"]
        K, I = c["K"], c["I"]
        ss.subspec_add_norm(st["x"], st["res"], st["weight"], EPS, M, K, st["sum"], None, st["a"], st["a_s"])
        ss.subspec_fp8_linear(st["a"], st["a_s"], st["up"], st["up_s"], M, 2 * I, K, st["gu"])
        ss.subspec_silu_mul(st["gu"], M, I, None, st["h"], st["h_s"])
        ss.subspec_fp8_linear(st["h"], st["h_s"], st["down"], st["down_s"], M, K, I, st["y"])
        return dict(sum=st["sum"], y=st["y"])
    if op == "norm":
        s, y = _plain_norm(st)
        return dict(sum=s.to(torch.bfloat16), y=y.to(torch.bfloat16))
    if op == "act":
        return _plain_act(st["gu"]).to(torch.bfloat16)
    if op == "linear":
        return _plain_product(st["x"].float(), st["w"], st["ws"], c["N"])
    s, y = _plain_norm(st)
    gu = _plain_product(y, st["up"], st["up_s"], 2 * c["I"])
    return dict(sum=s.to(torch.bfloat16), y=_plain_product(_plain_act(gu), st["down"], st["down_s"], c["K"]))


def _plain_norm(st):
    s = st["x"].float()
    if st["res"] is not None:
        s = s + st["res"].float()
    return s, s * torch.rsqrt((s * s).mean(-1, keepdim=True) + EPS) * st["weight"].float()


def _plain_act(gu):
    g, u = gu.float().chunk(2, -1)
    return g / (1.0 + (-g).exp()) * u


def _plain_product(x, tiles, words, N):
    w = _unpacked(tiles, words, N, x.shape[1])
    return torch.matmul(_rounded(x.contiguous()), w.t()).to(torch.bfloat16)


# --- what a pass cannot do without -------------------------------------------------------

def work(case):
    op, M = case["op"], case["M"]
    if op == "norm":
        n = M * case["K"]
        return dict(bytes=(8 if case["residual"] else 6) * n + 2 * case["K"], flops=6 * n)
    if op == "act":
        return dict(bytes=6 * M * case["I"], flops=6 * M * case["I"])
    weight = lambda N, K: N * K + 4 * N * ((K + 511) // 512)  # noqa: E731
    K = case["K"]
    if op == "linear":
        N = case["N"]
        return dict(bytes=2 * M * K + weight(N, K) + 2 * M * N, flops=2 * M * N * K)
    I = case["I"]
    # x, residual, sum and y of K; the rows between the products stay out: a pass could hold them on the chip
    return dict(bytes=8 * M * K + weight(2 * I, K) + weight(K, I), flops=6 * M * K * I)


# --- the definitions in 64 bits ----------------------------------------------------------

def _as_e4m3(x):
    """What 8-bit rows of fp64 x [R][K] stand for: each value on the grid of its binade."""
    b = x.reshape(x.shape[0], x.shape[1] // 128, 128)
    top = b.abs().max(2, keepdim=True).values
    scale = torch.exp2(torch.ceil(torch.log2(top / 448.0)).clamp(min=-126.0))
    v = b / scale
    step = torch.exp2(torch.floor(torch.log2(v.abs())).clamp(min=-6.0) - 3.0)
    return (torch.round(v / step) * step * scale).reshape(x.shape)


def _tile_values(tiles, words, N, K):
    """fp64 weights [N][K], each code and scale looked up at its place."""
    table = torch.arange(256, dtype=torch.uint8, device=DEV).view(torch.float8_e4m3fn).double()
    n, k = torch.arange(N, device=DEV)[:, None], torch.arange(K, device=DEV)[None, :]
    at = (n // 16) * (16 * K) + (n % 16) * 16 + (k // 128) * 2048 + (k % 128 // 64) * 1024 + (k % 64 // 16) * 256 + k % 16
    w = table[tiles[at].int()]
    e = words.reshape(-1)[(k // 512 * N + n) * 4 + k // 128 % 4].double() - 127.0
    return w * torch.exp2(e)


def exact(case, seed):
    st, op, M = prepare(case, seed), case["op"], case["M"]
    if op == "act":
        g, u = st["gu"][:, :case["I"]].double(), st["gu"][:, case["I"]:].double()
        return g * torch.sigmoid(g) * u
    if op == "linear":
        return _as_e4m3(st["x"].double()) @ _tile_values(st["w"], st["ws"], case["N"], case["K"]).T
    s = st["x"].double()
    if st["res"] is not None:
        s = s + st["res"].double()
    y = s / torch.sqrt(s.square().sum(1, keepdim=True) / case["K"] + EPS) * st["weight"].double()
    if op == "norm":
        return dict(sum=s, y=y)
    K, I = case["K"], case["I"]
    # the row between the two products is held in bf16
    gu = (_as_e4m3(y) @ _tile_values(st["up"], st["up_s"], 2 * I, K).T).to(torch.bfloat16).double()
    h = gu[:, :I] * torch.sigmoid(gu[:, :I]) * gu[:, I:]
    return dict(sum=s, y=_as_e4m3(h) @ _tile_values(st["down"], st["down_s"], K, I).T)
