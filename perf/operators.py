"""The 4-bit expert products and the router's balance loss, as cases to time and compare.

Four operators of a mixture-of-experts layer, called as a program that trains
or serves one calls them:

* ``quantize``: rows (of tokens, gathered into expert order, or of weights) to
  MX FP4 blocks of 32 values, and back to the values that they stand for;
* ``product``: y = a w^T over MX FP4 matrices, dense or one weight matrix per
  run of rows (an expert's rows);
* ``ffn``: the experts of a layer in MX FP4: gather and quantize the tokens,
  gate/up product with SwiGLU and 4-bit h, down product;
* ``balance``: the router's load-balance loss with per-expert counts, and its
  gradient in the logits.

The shapes are the repository's workloads: the mid-size layer, the
DeepSeek-V3-shaped expert share (even routing and Zipf-skewed routing) and the
share with hidden 2560 and 512 experts.

An MX FP4 matrix of R rows and K columns (K rounded up to a multiple of 256
with zeros) is held as the matrix cores read it: codes [ceil(R / 32), K / 32,
32 rows, 16 bytes] (value 2 i of a block of 32 in the low half of byte i), and
scales [ceil(R / 32), K / 256, 2, 32 rows, 4], where entry (b, h, r, s) is the
E8M0 scale of row r's block 8 b + 2 s + h.
"""

import functools
import math

import torch

own = False

# One GPU's share of a layer: expert pool, resident experts, top-k, hidden, expert width.
MID = dict(E=32, E_loc=32, k=4, H=2048, I=1024)
DSV3 = dict(E=256, E_loc=32, k=8, H=7168, I=2048)
WIDE_POOL = dict(E=512, E_loc=64, k=8, H=2560, I=768)


def _quantize(rows, cols, dtype, tokens=0, **name):
    """tokens: 0, or the rows are gathered from that many tokens."""
    return dict(**name, op="quantize", rows=rows, cols=cols, dtype=dtype, tokens=tokens)


def _product(rows, n, k, groups, out, zipf=0.0, **name):
    """groups: weight matrices, the rows shared among them (evenly on average, or by Zipf shares)."""
    return dict(**name, op="product", rows=rows, n=n, k=k, groups=groups, out=out, zipf=zipf)


def _ffn(shape, tokens, zipf=0.0, **name):
    """rows: of the tokens' k slots each, those that this share's experts take (three quarters of
    them where it owns the popular experts)."""
    share = 0.75 if zipf and shape["E"] > shape["E_loc"] else shape["E_loc"] / shape["E"]
    rows = max(1, round(tokens * shape["k"] * share))
    return dict(**name, op="ffn", tokens=tokens, rows=rows, zipf=zipf, **shape)


def _balance(tokens, E, k, seqs=1, dtype="f32", masked=False, train=True, **name):
    return dict(**name, op="balance", tokens=tokens, E=E, k=k, seqs=seqs, dtype=dtype, masked=masked, train=train)


def listed():
    return [
        # the hidden states of a decode batch, before a dense 4-bit product
        _quantize(64, 7168, "bf16", name="quantize-decode-64"),
        # a prefill batch's tokens gathered into the order of their experts
        _quantize(8243, 7168, "bf16", tokens=8192, name="quantize-gather-8192"),
        # a float32 master weight whose width is no multiple of a block
        _quantize(12289, 2559, "f32", name="quantize-weight-odd"),
        # one token through one matrix: a product that is all latency and weight stream
        _product(1, 7168, 2048, 1, "bf16", name="product-token"),
        # a decode batch's gate/up product over every expert of the share
        _product(131, 4096, 7168, 32, "f32", name="product-decode-dsv3"),
        # the down product of a ragged continuation prefill
        _product(3001, 2560, 768, 64, "bf16", name="product-prefill-pool512"),
        # the down product of the largest batch on the rank that owns the popular experts
        _product(96889, 7168, 2048, 32, "f32", zipf=1.2, name="product-prefill-dsv3-zipf"),
        # the end of a rollout: a few conversations left
        _ffn(WIDE_POOL, 37, name="ffn-decode-pool512-37"),
        # a long prefill batch
        _ffn(DSV3, 8192, name="ffn-prefill-dsv3-8192"),
        # watching the load of a small layer's router while it serves
        _balance(64, 8, 2, train=False, name="balance-watch-64"),
        # a training batch of packed sequences, padding masked, sequence by sequence
        _balance(12001, 512, 8, seqs=37, masked=True, name="balance-seqs-12001"),
        # one loss over a large training batch
        _balance(65536, 256, 8, name="balance-batch-65536"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["quantize", "quantize", "product", "product", "product", "ffn", "ffn", "balance", "balance"])
    if op == "quantize":
        cols = _log_int(rng, 33, 7168)
        rows = _log_int(rng, 1, min(65536, (1 << 26) // cols))
        tokens = _log_int(rng, max(1, rows // 8), rows) if rng.random() < 0.4 else 0
        return _quantize(rows, cols, rng.choice(["bf16", "bf16", "f32"]), tokens)
    if op == "product":
        shape = rng.choice([MID, WIDE_POOL, WIDE_POOL, DSV3, DSV3])
        n, k = rng.choice([(2 * shape["I"], shape["H"]), (shape["H"], shape["I"])])
        out = rng.choice(["f32", "bf16"])
        if rng.random() < 0.3:  # one matrix, odd widths among them
            n = _log_int(rng, 97, 8191)
            return _product(_log_int(rng, 1, 8192), n, k, 1, out)
        zipf = 1.2 if rng.random() < 0.25 else 0.0
        return _product(_log_int(rng, 1, 32768), n, k, shape["E_loc"], out, zipf)
    if op == "ffn":
        return _ffn(rng.choice([MID, WIDE_POOL, WIDE_POOL, DSV3]), _log_int(rng, 1, 8192),
                    1.2 if rng.random() < 0.25 else 0.0)
    E = _log_int(rng, 4, 1024)
    tokens = _log_int(rng, 1, min(65536, (1 << 24) // E))
    return _balance(tokens, E, rng.randint(1, min(8, E // 2)), seqs=_log_int(rng, 1, min(tokens, 128)),
                    dtype=rng.choice(["f32", "f32", "bf16"]), masked=tokens >= 32 and rng.random() < 0.5,
                    train=rng.random() < 0.75)


# ---- inputs -----------------------------------------------------------------

_DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 1000003 + 17)
    return g


def _up(v, m):
    return -(-v // m) * m


def _hold(codes, scales):
    """Row-major codes (one value a byte) and scales of whole blocks to the held form."""
    R, K = codes.shape
    Rp, Kp = _up(R, 32), _up(K, 256)
    codes = torch.nn.functional.pad(codes, (0, Kp - K, 0, Rp - R))
    scales = torch.nn.functional.pad(scales, (0, Kp // 32 - K // 32, 0, Rp - R))
    codes = codes[:, 0::2] | (codes[:, 1::2] << 4)
    return (codes.view(Rp // 32, 32, Kp // 32, 16).permute(0, 2, 1, 3).contiguous(),
            scales.view(Rp // 32, 32, Kp // 256, 4, 2).permute(0, 2, 4, 1, 3).contiguous())


def _random_mx4(g, R, K, std):
    """An MX FP4 matrix as quantizing normal values gives it, held as the products read it."""
    codes, scales = [], []
    step = _up(max(1, (1 << 26) // K), 32)  # whole 32-row blocks at a time
    for r in range(0, R, step):
        v = torch.randn((min(step, R - r), K), generator=g, device="cuda") * std
        b = v.view(v.shape[0], -1, 32)
        e = torch.frexp(b.abs().amax(dim=2))[1] - 3  # amax in [4, 8) 2^e
        q = b.abs() * torch.exp2(-e.to(torch.float32))[:, :, None]
        c = torch.bucketize(q, torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], device="cuda"))
        c = (c + 8 * (b < 0)).to(torch.uint8).view(v.shape)
        c, s = _hold(c, (e + 127).to(torch.uint8))
        codes.append(c)
        scales.append(s)
    return torch.cat(codes), torch.cat(scales)


def _shares(n, zipf):
    r = torch.arange(1, n + 1, dtype=torch.float64)
    p = r ** -zipf
    return p / p.sum()


def _counts(g, rows, groups, zipf):
    """Rows of each group, as routing deals them."""
    pick = torch.multinomial(_shares(groups, zipf).to("cuda"), rows, replacement=True, generator=g)
    return torch.bincount(pick, minlength=groups)


def _offsets(counts):
    return torch.nn.functional.pad(counts.cumsum(0), (1, 0)).to(torch.int32)


def _route(g, case):
    """(offsets, token of each row) of a batch: experts in order, an expert's tokens ascending."""
    R, T, G = case["rows"], case["tokens"], case["E_loc"]
    pick = torch.multinomial(_shares(G, case["zipf"]).to("cuda"), R, replacement=True, generator=g)
    key = (pick * T + torch.randint(0, T, (R,), generator=g, device="cuda")).sort().values
    return _offsets(torch.bincount(key // T, minlength=G)), (key % T).to(torch.int32)


def _activations(g, T, H):
    """Hidden states: normal, a few channels with larger values."""
    x = torch.randn((T, H), generator=g, device="cuda")
    loud = torch.rand((H,), generator=g, device="cuda") < 0.01
    return x * torch.where(loud, 8.0, 1.0)


class State:
    """What a program has in hand before the call."""


@functools.lru_cache(maxsize=None)
def _stream():
    """A program's stream, which it keeps."""
    return torch.cuda.Stream()


def _buffers(R, K):
    """Room for an MX FP4 matrix."""
    Rp, Kp = _up(max(R, 1), 32), _up(K, 256)
    return (torch.empty(Rp * Kp // 2, dtype=torch.uint8, device="cuda"),
            torch.empty(Rp * Kp // 32, dtype=torch.uint8, device="cuda"))


def prepare(case, seed):
    g = _generator(seed)
    s = State()
    s.case = case
    dev = dict(device="cuda")
    if case["op"] == "quantize":
        R, K = case["rows"], case["cols"]
        if case["tokens"]:
            s.x = _activations(g, case["tokens"], K).to(_DTYPES[case["dtype"]])
            s.index = torch.randint(0, case["tokens"], (R,), generator=g, dtype=torch.int32, **dev)
        else:
            s.x = _activations(g, R, K).to(_DTYPES[case["dtype"]])
            s.index = None
        s.q = _buffers(R, K)
        s.out = torch.empty((R, K), dtype=torch.bfloat16, **dev)
    elif case["op"] == "product":
        R, n, k, G = case["rows"], case["n"], case["k"], case["groups"]
        s.counts = [R]
        s.offsets = None
        if G > 1:
            counts = _counts(g, R, G, case["zipf"])
            s.counts = counts.tolist()
            s.offsets = _offsets(counts)
        s.a = _random_mx4(g, R, k, 1.0)
        s.w = _random_mx4(g, G * n, k, 1.0 / math.sqrt(k))
        s.out = torch.empty((R, n), dtype=_DTYPES[case["out"]], **dev)
    elif case["op"] == "ffn":
        H, I, G = case["H"], case["I"], case["E_loc"]
        s.offsets, s.token = _route(g, case)
        s.counts = (s.offsets[1:] - s.offsets[:-1]).tolist()
        s.x = _activations(g, case["tokens"], H).to(torch.bfloat16)
        s.gate_up = _random_mx4(g, G * 2 * I, H, 1.0 / math.sqrt(H))
        s.down = _random_mx4(g, G * H, I, 1.0 / math.sqrt(I))
        s.q, s.h = _buffers(case["rows"], H), _buffers(case["rows"], I)
        s.out = torch.empty((case["rows"], H), dtype=torch.bfloat16, **dev)
    else:
        T, E, S = case["tokens"], case["E"], case["seqs"]
        popular = torch.log(_shares(E, 0.6)).to("cuda", torch.float32)
        logits = torch.randn((T, E), generator=g, **dev) * 1.5 + popular[None, :]
        s.logits = logits.to(_DTYPES[case["dtype"]])
        s.idx = s.logits.to(torch.float32).topk(case["k"], dim=1).indices.to(torch.int32).contiguous()
        s.mask = (torch.rand((T,), generator=g, **dev) < 0.9).to(torch.uint8) if case["masked"] else None
        s.seq = None
        if S > 1:  # packed sequences of any length, empty ones among them
            cuts = torch.randint(0, T + 1, (S - 1,), generator=g, **dev).sort().values
            s.seq = torch.cat([torch.zeros(1, **dev), cuts, torch.full((1,), T, **dev)]).to(torch.int32)
        s.coef, s.grad = 0.01, torch.ones((1,), **dev)
        s.loss = torch.empty((1,), **dev)
        s.counts = torch.empty((S, E), dtype=torch.int32, **dev)
        s.live = torch.empty((S + 1,), dtype=torch.int32, **dev)
        s.dlogits = torch.empty_like(s.logits)
        # room for the sums of pieces of the batch, at the most that the loss asks for
        s.work = torch.empty(balance_workspace(T, E, S), dtype=torch.uint8, **dev)
    return s


def balance_workspace(T, E, S):
    return 8 * (S + 4096) * (E + 4) + 64


# ---- plain forms --------------------------------------------------------------

_MAGNITUDES = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def _values(m, R, K):
    """The float32 values of a held matrix."""
    Kp = _up(K, 256)
    codes = m[0].view(-1, Kp // 32, 32, 16).permute(0, 2, 1, 3).reshape(-1, Kp // 2)[:R]
    scales = m[1].view(-1, Kp // 256, 2, 32, 4).permute(0, 3, 1, 4, 2).reshape(-1, Kp // 32)[:R]
    codes = torch.stack([codes & 15, codes >> 4], dim=2).view(R, Kp)
    table = torch.tensor(_MAGNITUDES + [-v for v in _MAGNITUDES], device=codes.device)
    scale = torch.exp2(scales.to(torch.float32) - 127.0)
    return (table[codes.to(torch.int32)].view(R, Kp // 32, 32) * scale[:, :, None]).view(R, Kp)[:, :K]


def _rounded(v):
    """float32 rows to the values of their MX FP4 blocks."""
    K = v.shape[1]
    b = torch.nn.functional.pad(v, (0, _up(K, 32) - K)).view(v.shape[0], -1, 32)
    amax = b.abs().amax(dim=2, keepdim=True)
    e = torch.where(amax > 0, (torch.frexp(amax)[1] - 3).clamp(min=-127), -127).to(torch.float32)
    q = (b * torch.exp2(-e)).abs()
    code = (q > 0.25).to(torch.int32) + (q >= 0.75) + (q > 1.25) + (q >= 1.75) + (q > 2.5) + (q >= 3.5) + (q > 5.0)
    q = torch.tensor(_MAGNITUDES, device=v.device)[code] * torch.exp2(e)
    return torch.where(b < 0, -q, q).view(v.shape[0], -1)[:, :K]


def _grouped(a, w, counts):
    """Rows times the transposed matrix of their group."""
    w = w.view(len(counts), -1, w.shape[1])
    return torch.cat([x @ m.t() for x, m in zip(a.split(counts), w)])


def _plain(s):
    c = s.case
    if c["op"] == "quantize":
        x = s.x if s.index is None else s.x[s.index]
        return {"values": _rounded(x.to(torch.float32)).to(torch.bfloat16)}
    if c["op"] == "product":
        a, w = _values(s.a, c["rows"], c["k"]), _values(s.w, c["groups"] * c["n"], c["k"])
        return {"y": _grouped(a, w, s.counts).to(s.out.dtype)}
    if c["op"] == "ffn":
        H, I, G = c["H"], c["I"], c["E_loc"]
        a = _rounded(s.x[s.token].to(torch.float32))
        gu = _grouped(a, _values(s.gate_up, G * 2 * I, H), s.counts)
        gate, up = gu[:, :I], gu[:, I:]
        h = _rounded(gate / (1.0 + torch.exp(-gate)) * up)
        return {"y": _grouped(h, _values(s.down, G * H, I), s.counts).to(torch.bfloat16)}
    T, E, k, S = c["tokens"], c["E"], c["k"], c["seqs"]
    x = s.logits.to(torch.float32)
    p = torch.exp(x - x.amax(dim=1, keepdim=True))
    p = p / p.sum(dim=1, keepdim=True)
    live = torch.ones(T, device="cuda") if s.mask is None else (s.mask != 0).to(torch.float32)
    at = torch.arange(T, device="cuda", dtype=torch.int32)
    seq = torch.zeros_like(at) if s.seq is None else torch.searchsorted(s.seq[1:], at, right=True)
    member = (seq[None, :] == torch.arange(S, device="cuda")[:, None]).to(torch.float32) * live[None, :]
    slot = (seq[:, None] * E + s.idx).to(torch.int64)
    counts = torch.zeros(S * E, device="cuda", dtype=torch.int32)
    counts = counts.scatter_add_(0, slot.view(-1), live.to(torch.int32)[:, None].expand(T, k).reshape(-1)).view(S, E)
    tokens = member.sum(dim=1)
    seqs = (tokens > 0).sum()
    each = tokens.clamp(min=1.0)[:, None]
    f = counts.to(torch.float32) * (E / k) / each
    loss = s.coef * (f * (member @ p) / each).sum() / seqs.clamp(min=1)
    got = {"loss": loss.view(1), "counts": counts, "live": torch.cat([tokens, seqs.view(1)]).to(torch.int32)}
    if c["train"]:
        ft = f[seq]
        weight = s.grad * s.coef * live / (each[:, 0][seq] * seqs.clamp(min=1))
        got["dlogits"] = (weight[:, None] * p * (ft - (ft * p).sum(dim=1, keepdim=True))).to(s.logits.dtype)
    return got


# ---- the framework's operators --------------------------------------------------


def _own(s):
    from paper_2609_00993_amd import moepd as M

    c, st = s.case, _stream()
    types = {torch.float32: M.MOE_DTYPE_F32, torch.bfloat16: M.MOE_DTYPE_BF16}
    if c["op"] == "quantize":
        M.check(M.moe_mx4_quantize(s.x, types[s.x.dtype], s.x.stride(0), c["rows"], c["cols"], s.index, None, *s.q, st),
                "moe_mx4_quantize")
        M.check(M.moe_mx4_dequantize(*s.q, c["rows"], c["cols"], s.out, M.MOE_DTYPE_BF16, c["cols"], st),
                "moe_mx4_dequantize")
        return {"values": s.out}
    if c["op"] == "product":
        M.check(M.moe_mx4_gemm(*s.a, c["rows"], *s.w, c["groups"], s.offsets, c["n"], c["k"], s.out,
                               types[s.out.dtype], c["n"], st), "moe_mx4_gemm")
        return {"y": s.out}
    if c["op"] == "ffn":
        H, I, G = c["H"], c["I"], c["E_loc"]
        M.check(M.moe_mx4_quantize(s.x, M.MOE_DTYPE_BF16, H, c["rows"], H, s.token, s.offsets[G:], *s.q, st),
                "moe_mx4_quantize")
        M.check(M.moe_mx4_gemm_swiglu(*s.q, c["rows"], *s.gate_up, G, s.offsets, I, H, s.h[0], s.h[1], M.MOE_DTYPE_FP4, 0,
                                      st), "moe_mx4_gemm_swiglu")
        M.check(M.moe_mx4_gemm(*s.h, c["rows"], *s.down, G, s.offsets, H, I, s.out, M.MOE_DTYPE_BF16, H, st),
                "moe_mx4_gemm")
        return {"y": s.out}
    T, E, k, S = c["tokens"], c["E"], c["k"], c["seqs"]
    dt = types[s.logits.dtype]
    M.check(M.moe_balance_loss(s.logits, dt, E, s.idx, s.mask, s.seq, S, T, E, k, s.coef, s.loss, s.counts, s.live,
                               s.work, s.work.numel(), st), "moe_balance_loss")
    got = {"loss": s.loss, "counts": s.counts, "live": s.live}
    if c["train"]:
        M.check(M.moe_balance_loss_backward(s.logits, dt, E, s.mask, s.seq, S, T, E, k, s.coef, s.counts, s.live,
                                            s.grad, s.dlogits, E, False, st), "moe_balance_loss_backward")
        got["dlogits"] = s.dlogits
    return got


def run(s):
    return _own(s) if own else _plain(s)


# ---- what a pass cannot do without ---------------------------------------------


def _mx4_bytes(R, K):
    return R * K * (1 / 2 + 1 / 32)


def _touched(rows, groups, zipf):
    """Expected number of groups with a row."""
    return float((1 - (1 - _shares(groups, zipf)) ** rows).sum())


def work(case):
    if case["op"] == "quantize":
        R, K = case["rows"], case["cols"]
        read = min(R, case["tokens"] or R) * K * (4 if case["dtype"] == "f32" else 2)
        return {"bytes": read + _mx4_bytes(R, K) + R * K * 2, "flops": 0.0}
    if case["op"] == "product":
        R, n, k = case["rows"], case["n"], case["k"]
        touched = _touched(R, case["groups"], case["zipf"])
        return {"bytes": _mx4_bytes(R, k) + touched * _mx4_bytes(n, k) + R * n * (4 if case["out"] == "f32" else 2),
                "flops": 2.0 * R * n * k}
    if case["op"] == "ffn":
        T, R, H, I = case["tokens"], case["rows"], case["H"], case["I"]
        touched = _touched(R, case["E_loc"], case["zipf"])
        return {"bytes": T * H * 2 + touched * 3 * _mx4_bytes(I, H) + R * H * 2, "flops": 6.0 * R * H * I}
    T, E, k = case["tokens"], case["E"], case["k"]
    size = 4 if case["dtype"] == "f32" else 2
    return {"bytes": T * E * size * (2 if case["train"] else 1) + T * k * 4 + case["seqs"] * E * 4, "flops": 0.0}


# ---- the definitions in 64 bits --------------------------------------------------


def _exact_values(m, R, K):
    Kp = _up(K, 256)
    b = m[0].view(-1, Kp // 32, 32, 16)[:, :, :, :].transpose(1, 2).reshape(-1, Kp // 32, 16)[:R]
    nib = torch.cat([(b & 15)[..., None], (b >> 4)[..., None]], dim=-1).view(R, Kp).to(torch.int64)
    mag, sign = nib & 7, 1.0 - 2.0 * (nib >> 3)
    ex = mag >> 1  # E2M1: subnormal 0.5 m, else (1 + m / 2) 2^(ex - 1)
    v = torch.where(ex == 0, 0.5 * (mag & 1), (1.0 + 0.5 * (mag & 1)) * torch.exp2((ex - 1).to(torch.float64)))
    i = torch.arange(Kp // 32, device=b.device)
    s = m[1].view(-1, Kp // 256, 2, 32, 4)
    s = s[:, i // 8, i % 2, :, (i % 8) // 2]  # [block, row block, row]
    s = s.permute(1, 2, 0).reshape(-1, Kp // 32)[:R].to(torch.float64)
    return ((sign * v).view(R, -1, 32) * torch.exp2(s - 127.0)[:, :, None]).view(R, Kp)[:, :K]


def _exact_rounded(v):
    R, K = v.shape
    b = torch.nn.functional.pad(v, (0, _up(K, 32) - K)).view(R, -1, 32)
    amax = b.abs().amax(dim=2, keepdim=True)
    e = torch.floor(torch.log2(torch.where(amax > 0, amax, 1.0)))
    e = torch.where(torch.exp2(e) > amax, e - 1, e)  # a logarithm that rounded up to the next power
    e = torch.where(amax > 0, (e - 2).clamp(min=-127.0), torch.full_like(e, -127.0))
    q = b / torch.exp2(e)
    step = torch.where(q.abs() < 2, 0.5, torch.where(q.abs() < 4, 1.0, 2.0)).to(torch.float64)
    q = (torch.round(q / step) * step).clamp(-6.0, 6.0)  # ties to even
    return (q * torch.exp2(e)).view(R, -1)[:, :K]


def _exact_grouped(a, m, n, K, counts):
    """Group by group: the values of a held matrix [groups n, K] in 64 bits are large."""
    blocks, at, got = 0, 0, []
    for i, rows in enumerate(counts):
        first, last = i * n // 32, -(-(i + 1) * n // 32)
        part = (m[0][first:last], m[1][first:last])
        w = _exact_values(part, (last - first) * 32, K)[i * n - first * 32:][:n]
        got.append(a[at:at + rows] @ w.t())
        at += rows
    return torch.cat(got)


def exact(case, seed):
    s = prepare(case, seed)
    c = case
    if c["op"] == "quantize":
        x = s.x if s.index is None else s.x[s.index.to(torch.int64)]
        return {"values": _exact_rounded(x.to(torch.float64))}
    if c["op"] == "product":
        return {"y": _exact_grouped(_exact_values(s.a, c["rows"], c["k"]), s.w, c["n"], c["k"], s.counts)}
    if c["op"] == "ffn":
        H, I = c["H"], c["I"]
        a = _exact_rounded(s.x.to(torch.float64))[s.token.to(torch.int64)]
        gu = _exact_grouped(a, s.gate_up, 2 * I, H, s.counts)
        h = _exact_rounded(torch.sigmoid(gu[:, :I]) * gu[:, :I] * gu[:, I:])
        return {"y": _exact_grouped(h, s.down, H, I, s.counts)}
    T, E, k, S = c["tokens"], c["E"], c["k"], c["seqs"]
    p = torch.softmax(s.logits.to(torch.float64), dim=1)
    cuts = [0, T] if s.seq is None else s.seq.tolist()
    loss, seqs = 0.0, 0
    grad = torch.zeros_like(p)
    for a, b in zip(cuts[:-1], cuts[1:]):
        at = torch.arange(a, b, device="cuda")
        if s.mask is not None:
            at = at[s.mask[a:b] != 0]
        n = at.numel()
        if not n:
            continue
        seqs += 1
        f = torch.bincount(s.idx[at].reshape(-1).to(torch.int64), minlength=E).to(torch.float64) * E / (k * n)
        loss = loss + (f * p[at].mean(dim=0)).sum()
        grad[at] = p[at] * (f[None, :] - (p[at] @ f)[:, None]) / n
    seqs = max(seqs, 1)
    got = {"loss": torch.as_tensor(s.coef * loss / seqs, dtype=torch.float64).view(1).cpu(), "counts": None, "live": None}
    if c["train"]:
        got["dlogits"] = grad * (s.coef / seqs)
    return got
