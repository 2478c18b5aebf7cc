"""The training side of the expert layer, as cases to time and compare.

Three operators, called as a program that trains or serves a mixture of experts
calls them:

* ``ffn``: the gated feed-forward block over rows in expert order (one weight
  matrix per run of rows, or one for all): h = silu(x W1^T) * (x W3^T) and
  y = h W2^T, and its backward pass. h and the gradient of the two projections
  are results in bfloat16, and the operands of the products that follow them;
* ``rows``: tokens to rows in expert order and, weighted, back, with the
  gradients of both and of the gate;
* ``adamw``: one step over many tensors, with states in 32 bits or in 8; these
  are read out afterwards, as the values that they stand for.

The shapes are the repository's workloads: the mid-size layer, the
DeepSeek-V3-shaped expert share (even and Zipf-skewed routing) and the share
with hidden 2560 and 512 experts.

States in 8 bits are blocks of 32 values with one E8M0 scale byte S (a factor of
2^(S - 127)): m as E4M3 codes, and the square root of v as codes of five exponent
and three mantissa bits, (1 + f / 8) 2^(e - 30), or f / 8 2^-29 where e is 0. The
scale puts a block's largest magnitude into [128, 256) for m and into [1, 2) for
v. Codes are rounded at random, by the 16-bit halves of a word that the seed, the
step, the tensor's number and the element's place give; a v above 0 keeps at
least the smallest code.
"""

import functools
import math

import torch

own = False

# One GPU's share of a layer: expert pool, resident experts, top-k, hidden, expert width.
MID = dict(E=32, E_loc=32, k=4, H=2048, I=1024)
DSV3 = dict(E=256, E_loc=32, k=8, H=7168, I=2048)
WIDE_POOL = dict(E=512, E_loc=64, k=8, H=2560, I=768)


def _ffn(rows, H, I, groups, what, zipf=0.0, **name):
    """what: "serve" (h, y), "forward" (the projections too, for the backward pass), "backward"
    (every gradient), or "weights" (the gradient of the gate and up weights alone, added to float32 sums)."""
    return dict(**name, op="ffn", rows=rows, H=H, I=I, groups=groups, what=what, zipf=zipf)


def _rows(tokens, E, E_loc, k, H, train, dtype="bf16", **name):
    return dict(**name, op="rows", tokens=tokens, E=E, E_loc=E_loc, k=k, H=H, train=train, dtype=dtype)


def _adamw(tensors, elems, bits, param="bf16", master=True, grad="bf16", **name):
    """tensors of all sizes, elems elements in all."""
    return dict(**name, op="adamw", tensors=tensors, elems=elems, bits=bits, param=param, master=master, grad=grad)


def listed():
    return [
        # one token through an expert that all tokens share
        _ffn(1, 7168, 2048, 1, "serve", name="ffn-token"),
        # a decode batch over every expert of the share
        _ffn(61, 2560, 768, 64, "serve", name="ffn-decode-pool512"),
        # a training batch's forward pass, whose projections are kept
        _ffn(8243, 7168, 2048, 32, "forward", name="ffn-forward-dsv3"),
        # the backward pass of a small batch, some fifty rows to an expert
        _ffn(2999, 2560, 768, 64, "backward", name="ffn-backward-pool512"),
        # the backward pass of a training batch
        _ffn(8243, 7168, 2048, 32, "backward", name="ffn-backward-dsv3"),
        # weight gradients of skewed experts, added up over a step's batches
        _ffn(30001, 2048, 1024, 32, "weights", zipf=1.2, name="ffn-weights-mid-zipf"),
        # the end of a rollout: a few conversations left
        _rows(37, 512, 64, 8, 2560, False, name="rows-decode-37"),
        # every expert resident, float32 rows
        _rows(16383, 32, 32, 4, 2048, False, dtype="f32", name="rows-forward-mid"),
        # the way back of a training batch, the gate's gradient with it
        _rows(8192, 256, 32, 8, 7168, True, name="rows-backward-dsv3"),
        # a router's gate and biases, in float32
        _adamw(9, 600_011, 32, param="f32", master=False, grad="f32", name="adamw-router"),
        # the experts of the mid-size layer: bfloat16 weights beside float32 masters
        _adamw(5, 201_392_160, 32, name="adamw-experts"),
        # the same with states in 8 bits
        _adamw(5, 201_392_160, 8, name="adamw-experts-8bit"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["ffn", "ffn", "ffn", "ffn", "rows", "rows", "adamw", "adamw"])
    if op == "ffn":
        what = rng.choice(["serve", "forward", "backward", "backward", "weights"])
        if rng.random() < 0.4:  # one block for all rows, widths of any multiple of 8
            H, I, G = 8 * _log_int(rng, 8, 640), 8 * _log_int(rng, 8, 320), 1
        else:
            s = rng.choice([MID, WIDE_POOL, WIDE_POOL, DSV3])
            H, I, G = s["H"], s["I"], s["E_loc"]
        zipf = 1.2 if G > 1 and rng.random() < 0.25 else 0.0
        return _ffn(_log_int(rng, 1, min(32768, 8000 * 7168 * 2048 // (H * I))), H, I, G, what, zipf)
    if op == "rows":
        s = rng.choice([MID, WIDE_POOL, DSV3])
        H = rng.choice([s["H"], s["H"], _log_int(rng, 33, 8191)])
        return _rows(_log_int(rng, 1, 8192), s["E"], rng.choice([s["E_loc"], s["E"]]) if s is MID else s["E_loc"], s["k"], H,
                     rng.random() < 0.6, rng.choice(["bf16", "bf16", "f32"]))
    param = rng.choice(["bf16", "bf16", "f32"])
    return _adamw(_log_int(rng, 1, 200), _log_int(rng, 1000, 150_000_000), rng.choice([8, 8, 32]), param,
                  param == "bf16" and rng.random() < 0.8, rng.choice(["bf16", "f32"]))


# ---- inputs -----------------------------------------------------------------

_DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 1000003 + 29)
    return g


def _shares(n, zipf):
    r = torch.arange(1, n + 1, dtype=torch.float64)
    p = r ** -zipf
    return p / p.sum()


def _normal(g, shape, std=1.0, dtype=torch.bfloat16):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, std, generator=g)


class State:
    """What a program has in hand before the call."""


@functools.lru_cache(maxsize=None)
def _stream():
    """A program's stream, which it keeps."""
    return torch.cuda.Stream()


WORKSPACE = 1 << 27  # bytes, at the most that a weight gradient asks for

BETA1, BETA2, EPS, DECAY = 0.9, 0.95, 1e-8, 0.1


def sizes(case):
    """Elements of each tensor: of all sizes, the largest some 250 times the smallest."""
    w = [2.0 ** (8.0 * ((i * 0.6180339887) % 1.0)) for i in range(case["tensors"])]
    return [max(1, int(case["elems"] * v / sum(w))) for v in w]


def _pad32(v):
    return torch.nn.functional.pad(v, (0, -v.numel() % 32)).view(-1, 32)


def _encode_m(m):
    b = _pad32(m)
    top = b.abs().amax(dim=1, keepdim=True)
    S = torch.where(top > 0, torch.frexp(top)[1] + 119, 0).clamp(0, 254)
    q = b * torch.exp2(127.0 - S.to(torch.float32))
    return q.to(torch.float8_e4m3fn).view(torch.uint8).view(-1)[:m.numel()].contiguous(), S.to(torch.uint8).view(-1)


def _encode_v(v):
    b = _pad32(v).sqrt()
    top = b.amax(dim=1, keepdim=True)
    S = torch.where(top > 0, torch.frexp(top)[1] + 126, 0).clamp(0, 254)
    q = b * torch.exp2(127.0 - S.to(torch.float32))
    e = (torch.frexp(q)[1] + 29).clamp(min=1)  # of the binade, 1 for those below
    f = torch.round(q * torch.exp2(33.0 - e.to(torch.float32))).to(torch.int32)  # 8 + f, or f below
    code = (e - 1) * 8 + f
    return code.to(torch.uint8).view(-1)[:v.numel()].contiguous(), S.to(torch.uint8).view(-1)


def prepare(case, seed):
    g = _generator(seed)
    s = State()
    s.case = case
    dev = dict(device="cuda")
    if case["op"] == "ffn":
        R, H, I, G = case["rows"], case["H"], case["I"], case["groups"]
        s.counts, s.offsets = [R], None
        if G > 1:
            pick = torch.multinomial(_shares(G, case["zipf"]).to("cuda"), R, replacement=True, generator=g)
            counts = torch.bincount(pick, minlength=G)
            s.counts = counts.tolist()
            s.offsets = torch.nn.functional.pad(counts.cumsum(0), (1, 0)).to(torch.int32)
        empty = lambda *shape: torch.empty(shape, dtype=torch.bfloat16, **dev)  # noqa: E731
        loud = torch.where(torch.rand((H,), generator=g, **dev) < 0.01, 8.0, 1.0)  # a few channels have larger values
        s.x = (_normal(g, (R, H), dtype=torch.float32) * loud).to(torch.bfloat16)
        if case["what"] != "weights":
            s.w_gate_up = _normal(g, (G, 2 * I, H), 1.0 / math.sqrt(H))
            s.w_down = _normal(g, (G, H, I), 1.0 / math.sqrt(I))
        if case["what"] in ("serve", "forward"):
            s.gate_up = empty(R, 2 * I) if case["what"] == "forward" else None
            s.h, s.y = empty(R, I), empty(R, H)
        elif case["what"] == "backward":
            s.gate_up = _normal(g, (R, 2 * I), 1.2)
            s.dy = _normal(g, (R, H), 1e-3)
            s.dgate_up, s.h, s.dx = empty(R, 2 * I), empty(R, I), empty(R, H)
            s.dw_gate_up, s.dw_down = empty(G, 2 * I, H), empty(G, H, I)
        else:
            s.dgate_up = _normal(g, (R, 2 * I), 1e-3)
            s.dw_gate_up = _normal(g, (G, 2 * I, H), 1e-2, torch.float32)
        if case["what"] in ("backward", "weights"):
            s.work = torch.empty(WORKSPACE, dtype=torch.uint8, **dev)
    elif case["op"] == "rows":
        T, E, k, H, L = case["tokens"], case["E"], case["k"], case["H"], case["E_loc"]
        t = _DTYPES[case["dtype"]]
        logits = _normal(g, (T, E), 1.5, torch.float32)
        top = logits.topk(k, dim=1)
        s.idx = top.indices.to(torch.int32).contiguous()
        s.w = torch.softmax(top.values, dim=1).contiguous()
        # slots at the share's experts, in expert order, an expert's rows by token
        e = s.idx.view(-1).to(torch.int64)
        order = torch.where(e < L, e, E).argsort(stable=True)
        even = T * k * L / E
        s.rows = min(T * min(k, L), int(even + 5 * math.sqrt(even)) + 16)  # room for them; a slot past it gets no row
        s.count = min(s.rows, int((e < L).sum()))
        kept = order[:s.count]
        s.row = torch.full((T * k,), -1, dtype=torch.int32, **dev)
        s.row[kept] = torch.arange(s.count, dtype=torch.int32, **dev)
        s.row = s.row.view(T, k)
        s.token = torch.zeros(s.rows, dtype=torch.int32, **dev)
        s.token[:s.count] = (kept // k).to(torch.int32)
        s.y = _normal(g, (s.rows, H), 0.7, t)
        if case["train"]:
            s.dout = _normal(g, (T, H), 1e-3, t)
            s.dxr = _normal(g, (s.rows, H), 1e-3, t)
            s.dy = torch.zeros((s.rows, H), dtype=t, **dev)
            s.dw = torch.empty((T, k), **dev)
            s.dlogits = torch.empty((T, E), **dev)
            s.dx = torch.empty((T, H), dtype=t, **dev)
        else:
            s.x = _normal(g, (T, H), 1.0, t)
            s.xr = torch.zeros((s.rows, H), dtype=t, **dev)
            s.out = torch.empty((T, H), **dev)
    else:
        s.tensors = []
        for n in sizes(case):
            t = State()
            p = _normal(g, (n,), 0.02, torch.float32)
            t.param = p.to(_DTYPES[case["param"]])
            t.master = p if case["master"] else None
            # gradients of rows that differ in size, and a state that has seen a few of them
            size = torch.exp2(torch.randint(-6, 3, (-(-n // 512),), generator=g, **dev).to(torch.float32))
            size = size.repeat_interleave(512)[:n] * 1e-3
            t.grad = (_normal(g, (n,), dtype=torch.float32) * size).to(_DTYPES[case["grad"]])
            m = _normal(g, (n,), 0.3, torch.float32) * size
            v = size.square() * (0.05 + _normal(g, (n,), 1.0, torch.float32).square())
            t.m_scale = t.v_scale = None
            if case["bits"] == 8:
                t.m, t.m_scale = _encode_m(m)
                t.v, t.v_scale = _encode_v(v)
                t.m_out, t.root_v_out = (torch.empty(n, dtype=torch.bfloat16, **dev) for _ in range(2))
            else:
                t.m, t.v = m, v
            t.decay = DECAY if n >= 4096 else 0.0
            s.tensors.append(t)
        s.lr, s.scale = torch.full((1,), 3e-4, **dev), torch.full((1,), 0.5, **dev)
        s.step = torch.full((1,), 3 + int(seed) % 100, dtype=torch.int32, **dev)
        s.seed = (int(seed) * 2654435761 + 12345) & 0xFFFFFFFF
        s.handle = None
    return s


# ---- plain forms --------------------------------------------------------------


def _grouped(a, w, counts):
    """Rows times the transposed matrix of their group."""
    return torch.cat([x @ m.t() for x, m in zip(a.split(counts), w)])


def _outer(a, b, counts):
    """Each group's a^T b."""
    return torch.stack([x.t() @ y for x, y in zip(a.split(counts), b.split(counts))])


def _plain_ffn(s):
    c, f32, bf16 = s.case, torch.float32, torch.bfloat16
    I = c["I"]
    if c["what"] == "weights":
        s.dw_gate_up += _outer(s.dgate_up.to(f32), s.x.to(f32), s.counts)
        return {"dw_gate_up": s.dw_gate_up}
    if c["what"] != "backward":
        gu = _grouped(s.x.to(f32), s.w_gate_up.to(f32), s.counts)
        gate, up = gu[:, :I], gu[:, I:]
        h = (gate / (1.0 + torch.exp(-gate)) * up).to(bf16)
        y = _grouped(h.to(f32), s.w_down.to(f32), s.counts).to(bf16)
        return {"h": h, "y": y} if c["what"] == "serve" else {"gate_up": gu.to(bf16), "h": h, "y": y}
    dy = s.dy.to(f32)
    gate, up = s.gate_up[:, :I].to(f32), s.gate_up[:, I:].to(f32)
    sig = 1.0 / (1.0 + torch.exp(-gate))
    h = (gate * sig * up).to(bf16)
    dh = _grouped(dy, s.w_down.to(f32).transpose(1, 2), s.counts)
    d = torch.cat([dh * up * sig * (1.0 + gate * (1.0 - sig)), dh * gate * sig], dim=1).to(bf16)
    df = d.to(f32)
    return {"h": h, "dgate_up": d, "dx": _grouped(df, s.w_gate_up.to(f32).transpose(1, 2), s.counts).to(bf16),
            "dw_gate_up": _outer(df, s.x.to(f32), s.counts).to(bf16), "dw_down": _outer(dy, h.to(f32), s.counts).to(bf16)}


def _spread(rows, row, w):
    """Weighted sums of each token's rows; a slot without a row adds nothing."""
    got = rows[row.clamp(min=0).to(torch.int64)].to(torch.float32)
    return (got * torch.where(row >= 0, w, 0.0)[:, :, None]).sum(dim=1)


def _plain_rows(s):
    c, t = s.case, _DTYPES[s.case["dtype"]]
    if not c["train"]:
        s.xr[:s.count] = s.x[s.token[:s.count].to(torch.int64)]
        return {"rows": s.xr, "out": _spread(s.y, s.row, s.w)}
    T, k = s.row.shape
    dout = s.dout.to(torch.float32)
    slot = torch.nonzero(s.row.view(-1) >= 0)[:, 0]
    row, token = s.row.view(-1)[slot].to(torch.int64), slot // k
    s.dy[row] = (dout[token] * s.w.view(-1)[slot][:, None]).to(t)
    dw = torch.zeros(T * k, device="cuda")
    dw[slot] = (dout[token] * s.y[row].to(torch.float32)).sum(dim=1)
    dw = dw.view(T, k)
    mean = (s.w * dw).sum(dim=1, keepdim=True)
    dlogits = torch.zeros_like(s.dlogits).scatter_(1, s.idx.to(torch.int64), s.w * (dw - mean))
    return {"dy": s.dy, "dw": dw, "dlogits": dlogits, "dx": _spread(s.dxr, s.row, torch.ones_like(s.w)).to(t)}


_WORD = 0xFFFFFFFF


def _mix(x):
    x = x ^ (x >> 16)
    x = (x * 0x6A09E667) & _WORD
    x = x ^ (x >> 15)
    x = (x * 0xBB67AE85) & _WORD
    return x ^ (x >> 16)


def _words(s, number, n):
    """The rounding words of tensor `number`'s n elements."""
    key = _mix((_mix((_mix(s.seed) + s.step.to(torch.int64)) & _WORD) + number) & _WORD)
    return _mix(torch.arange(n, device="cuda") ^ key)


def _scale_of(S):
    return torch.exp2(S.to(torch.float32) - 127.0).repeat_interleave(32)


def _decode_m(code, S, dtype=torch.float32):
    return (code.view(torch.float8_e4m3fn).to(torch.float32) * _scale_of(S)[:code.numel()]).to(dtype)


def _decode_v(code, S, dtype=torch.float32):
    """The square root of v."""
    e, f = (code >> 3).to(torch.float32), (code & 7).to(torch.float32)
    r = torch.where(e > 0, (8.0 + f) * torch.exp2(e - 33.0), f * 2.0 ** -32)
    return (r * _scale_of(S)[:code.numel()]).to(dtype)


def _blocks(v, above, bottom, r):
    """Values to (multiples of a code's step under its block's scale, step's exponent, sign, S)."""
    b = _pad32(v)
    top = b.abs().amax(dim=1, keepdim=True)
    S = torch.where(top > 0, torch.frexp(top)[1] - 1 - above + 127, 0).clamp(0, 254)
    q = b.abs() * torch.exp2(127.0 - S.to(torch.float32))
    e = torch.where(q > 0, torch.frexp(q)[1] - 1, bottom).clamp(min=bottom) - 3
    n = torch.floor(q * torch.exp2(-e.to(torch.float32)) + _pad32(r.to(torch.float32)) / 65536.0)
    return n, e, S


def _plain_tensor(s, number, t):
    c = s.case
    n = t.param.numel()
    step = s.step.to(torch.float64)
    c1, c2 = ((1.0 - b ** step).to(torch.float32) for b in (BETA1, BETA2))
    small = c["bits"] == 8
    m = _decode_m(t.m, t.m_scale) if small else t.m
    v = _decode_v(t.v, t.v_scale).square() if small else t.v
    g = t.grad.to(torch.float32) * s.scale
    m = BETA1 * m + (1.0 - BETA1) * g
    v = BETA2 * v + (1.0 - BETA2) * g * g
    p = t.param.to(torch.float32) if t.master is None else t.master
    p = p - s.lr * (m / c1 / (torch.sqrt(v / c2) + EPS) + t.decay * p)
    got = {}
    if t.master is not None:
        got["master"] = t.master.copy_(p)
    got["param"] = t.param.copy_(p)
    if not small:
        return dict(got, m=t.m.copy_(m), v=t.v.copy_(v))
    word = _words(s, number, n)
    k, e, S = _blocks(m, 7, -6, word >> 16)
    q = (k * torch.exp2(e.to(torch.float32))).view(-1)[:n]
    t.m.copy_(torch.where(m < 0, -q, q).to(torch.float8_e4m3fn).view(torch.uint8))
    t.m_scale.copy_(S.view(-1))
    k, e, S = _blocks(torch.sqrt(v), 0, -29, word & 0xFFFF)
    k = torch.where((k == 0) & (_pad32(v) > 0), 1.0, k)
    t.v.copy_(((e + 32) * 8 + k.to(torch.int32)).to(torch.uint8).view(-1)[:n])
    t.v_scale.copy_(S.view(-1))
    # the values that the codes stand for, which are exact in bfloat16
    return dict(got, m=_decode_m(t.m, t.m_scale, torch.bfloat16), root_v=_decode_v(t.v, t.v_scale, torch.bfloat16))


def _largest(s, got):
    """The results of up to 12 tensors, the largest ones and the smallest."""
    order = sorted(range(len(got)), key=lambda i: -s.tensors[i].param.numel())
    return [got[i] for i in (order if len(order) <= 12 else order[:4] + order[-8:])]


def _plain(s):
    if s.case["op"] == "ffn":
        return _plain_ffn(s)
    if s.case["op"] == "rows":
        return _plain_rows(s)
    return _largest(s, [_plain_tensor(s, i, t) for i, t in enumerate(s.tensors)])


# ---- the framework's operators --------------------------------------------------


def _own_ffn(s):
    from paper_2609_00993_amd import moepd as M

    c, st = s.case, _stream()
    R, H, I, G = c["rows"], c["H"], c["I"], c["groups"]
    bf16, f32 = M.MOE_DTYPE_BF16, M.MOE_DTYPE_F32
    if c["what"] == "weights":
        M.check(M.moe_ffn_weight_grad(s.dgate_up, 0, s.x, 0, R, G, s.offsets, 2 * I, H, bf16, s.dw_gate_up, f32, True, s.work,
                                      WORKSPACE, st), "moe_ffn_weight_grad")
        return {"dw_gate_up": s.dw_gate_up}
    if c["what"] != "backward":
        M.check(M.moe_ffn_gate_up(s.x, 0, R, s.w_gate_up, G, s.offsets, H, I, bf16, s.gate_up, s.h, st), "moe_ffn_gate_up")
        M.check(M.moe_ffn_down(s.h, R, s.w_down, G, s.offsets, H, I, bf16, s.y, bf16, 0, st), "moe_ffn_down")
        return {"h": s.h, "y": s.y} if c["what"] == "serve" else {"gate_up": s.gate_up, "h": s.h, "y": s.y}
    M.check(M.moe_ffn_down_backward(s.dy, 0, R, s.w_down, s.gate_up, G, s.offsets, H, I, bf16, s.dgate_up, s.h, st),
            "moe_ffn_down_backward")
    M.check(M.moe_ffn_gate_up_backward(s.dgate_up, R, s.w_gate_up, G, s.offsets, H, I, bf16, s.dx, bf16, 0, st),
            "moe_ffn_gate_up_backward")
    M.check(M.moe_ffn_weight_grad(s.dgate_up, 0, s.x, 0, R, G, s.offsets, 2 * I, H, bf16, s.dw_gate_up, bf16, False, s.work,
                                  WORKSPACE, st), "moe_ffn_weight_grad")
    M.check(M.moe_ffn_weight_grad(s.dy, 0, s.h, 0, R, G, s.offsets, H, I, bf16, s.dw_down, bf16, False, s.work, WORKSPACE, st),
            "moe_ffn_weight_grad")
    return {"h": s.h, "dgate_up": s.dgate_up, "dx": s.dx, "dw_gate_up": s.dw_gate_up, "dw_down": s.dw_down}


def _own_rows(s):
    from paper_2609_00993_amd import moepd as M

    c, st = s.case, _stream()
    T, E, k, H = c["tokens"], c["E"], c["k"], c["H"]
    dt = M.MOE_DTYPE_F32 if c["dtype"] == "f32" else M.MOE_DTYPE_BF16
    f32 = M.MOE_DTYPE_F32
    if not c["train"]:
        M.check(M.moe_rows_gather(s.x, dt, 0, T, s.token, None, s.count, H, s.xr, 0, st), "moe_rows_gather")
        M.check(M.moe_rows_combine(s.y, dt, 0, s.count, s.w, s.row, T, k, H, s.out, f32, 0, st), "moe_rows_combine")
        return {"rows": s.xr, "out": s.out}
    M.check(M.moe_rows_combine_backward(s.dout, dt, 0, s.y, dt, 0, s.count, s.w, s.row, T, k, H, s.dy, dt, 0, s.dw, st),
            "moe_rows_combine_backward")
    M.check(M.moe_gate_backward(s.idx, s.w, s.dw, T, E, k, s.dlogits, f32, 0, False, st), "moe_gate_backward")
    M.check(M.moe_rows_combine(s.dxr, dt, 0, s.count, None, s.row, T, k, H, s.dx, dt, 0, st), "moe_rows_combine")
    return {"dy": s.dy, "dw": s.dw, "dlogits": s.dlogits, "dx": s.dx}


class _Optimizer:
    """The library's table of a program's tensors, for as long as the program keeps them."""

    def __init__(self, s):
        from paper_2609_00993_amd import moepd as M

        code = {torch.float32: M.MOE_DTYPE_F32, torch.bfloat16: M.MOE_DTYPE_BF16}
        self.M = M
        table = [M.adamw_tensor(t.param, code[t.param.dtype], t.master, t.grad, code[t.grad.dtype], t.m, t.v, t.m_scale,
                                t.v_scale, t.param.numel(), t.decay) for t in s.tensors]
        st, self.handle = M.moe_adamw_create(table, s.case["bits"])
        M.check(st, "moe_adamw_create")

    def __del__(self):
        self.M.moe_adamw_destroy(self.handle)


def _own_adamw(s):
    from paper_2609_00993_amd import moepd as M

    if s.handle is None:
        s.handle = _Optimizer(s)
    M.check(M.moe_adamw_step(s.handle.handle, BETA1, BETA2, EPS, s.lr, s.step, s.scale, s.seed, _stream()), "moe_adamw_step")
    got = []
    for i, t in _largest(s, list(enumerate(s.tensors))):
        d = {"param": t.param}
        if t.master is not None:
            d["master"] = t.master
        if s.case["bits"] == 8:
            M.check(M.moe_adamw_read(s.handle.handle, i, t.m_out, t.root_v_out, M.MOE_DTYPE_BF16, _stream()), "moe_adamw_read")
            got.append(dict(d, m=t.m_out, root_v=t.root_v_out))
        else:
            got.append(dict(d, m=t.m, v=t.v))
    return got


def _own(s):
    return {"ffn": _own_ffn, "rows": _own_rows, "adamw": _own_adamw}[s.case["op"]](s)


def run(s):
    return _own(s) if own else _plain(s)


# ---- what a pass cannot do without ---------------------------------------------


def _touched(rows, groups, zipf):
    """Expected number of groups with a row."""
    return float((1 - (1 - _shares(groups, zipf)) ** rows).sum())


def work(case):
    if case["op"] == "ffn":
        R, H, I, G = case["rows"], case["H"], case["I"], case["groups"]
        weights = 3.0 * H * I * _touched(R, G, case["zipf"])
        if case["what"] == "weights":
            return {"bytes": 2.0 * R * (2 * I + H) + 8.0 * 2 * H * I * _touched(R, G, case["zipf"]), "flops": 4.0 * R * H * I}
        if case["what"] == "backward":  # dy, gate_up, x; the weights; dgate_up, h, dx; the weights' gradients
            return {"bytes": 2.0 * (R * (H + 2 * I + H) + weights + R * (2 * I + I + H) + 3.0 * H * I * G),
                    "flops": 12.0 * R * H * I}
        kept = 2 * I if case["what"] == "forward" else 0
        return {"bytes": 2.0 * (R * H + weights + R * (I + kept + H)), "flops": 6.0 * R * H * I}
    if case["op"] == "rows":
        T, k, H, E = case["tokens"], case["k"], case["H"], case["E"]
        size = 4 if case["dtype"] == "f32" else 2
        rows = T * k * case["E_loc"] / E
        if case["train"]:  # dout, y, rows' gradients; dy, dx, the gate
            return {"bytes": size * H * (T + rows + rows + rows + T) + T * k * 16.0 + T * E * 4.0, "flops": 0.0}
        return {"bytes": size * H * (min(T, rows) + rows + rows) + 4.0 * T * H + T * k * 8.0, "flops": 0.0}
    n = sum(sizes(case))
    p, g = (4 if case[x] == "f32" else 2 for x in ("param", "grad"))
    states = 16.0 if case["bits"] == 32 else 8.0 + 4.0 / 32  # with 8 bits, and their values written
    held = 2.0 * p if not case["master"] else p + 8.0
    return {"bytes": n * (held + g + states), "flops": 0.0}


# ---- the definitions in 64 bits --------------------------------------------------


def _exact_ffn(s):
    c, f64 = s.case, torch.float64
    I, got, at = c["I"], {}, 0
    bf = lambda v: v.to(torch.bfloat16).to(f64)  # noqa: E731  what is held in bfloat16 between products
    parts = []
    for e, n in enumerate(s.counts):
        x = s.x[at:at + n].to(f64)
        if c["what"] == "weights":
            parts.append({"dw_gate_up": s.dw_gate_up[e].to(f64) + s.dgate_up[at:at + n].to(f64).t() @ x})
        elif c["what"] == "backward":
            gate, up = s.gate_up[at:at + n].to(f64).split(I, dim=1)
            sig = torch.sigmoid(gate)
            dy = s.dy[at:at + n].to(f64)
            dh = dy @ s.w_down[e].to(f64)
            d = torch.cat([dh * up * (sig + gate * sig * torch.sigmoid(-gate)), dh * gate * sig], dim=1)
            h = gate * sig * up
            parts.append({"h": h, "dgate_up": d, "dx": bf(d) @ s.w_gate_up[e].to(f64), "dw_gate_up": bf(d).t() @ x,
                          "dw_down": dy.t() @ bf(h)})
        else:
            gate, up = (x @ s.w_gate_up[e].to(f64).t()).split(I, dim=1)
            h = torch.sigmoid(gate) * gate * up
            p = {"h": h, "y": bf(h) @ s.w_down[e].to(f64).t()}
            if c["what"] == "forward":
                p["gate_up"] = torch.cat([gate, up], dim=1)
            parts.append(p)
        at += n
    for name in parts[0]:
        got[name] = (torch.stack if name.startswith("dw") else torch.cat)([p[name] for p in parts])
    return got


def _exact_rows(s):
    c, f64 = s.case, torch.float64
    T, k = s.row.shape
    if not c["train"]:
        out = torch.zeros((T, c["H"]), dtype=f64, device="cuda")
        for j in range(k):
            at = torch.nonzero(s.row[:, j] >= 0)[:, 0]
            out[at] += s.w[at, j].to(f64)[:, None] * s.y[s.row[at, j].to(torch.int64)].to(f64)
        rows = torch.zeros((s.rows, c["H"]), dtype=f64, device="cuda")
        rows[:s.count] = s.x.to(f64)[s.token[:s.count].to(torch.int64)]
        return {"rows": rows, "out": out}
    dy = torch.zeros((s.rows, c["H"]), dtype=f64, device="cuda")
    dx = torch.zeros((T, c["H"]), dtype=f64, device="cuda")
    dw = torch.zeros((T, k), dtype=f64, device="cuda")
    for j in range(k):
        at = torch.nonzero(s.row[:, j] >= 0)[:, 0]
        r = s.row[at, j].to(torch.int64)
        d = s.dout[at].to(f64)
        dy[r] = s.w[at, j].to(f64)[:, None] * d
        dw[at, j] = torch.einsum("ij,ij->i", d, s.y[r].to(f64))
        dx[at] += s.dxr[r].to(f64)
    w = s.w.to(f64)
    dl = torch.zeros((T, c["E"]), dtype=f64, device="cuda")
    dl.scatter_(1, s.idx.to(torch.int64), w * dw - w * torch.einsum("ij,ij->i", w, dw)[:, None])
    return {"dy": dy, "dw": dw, "dlogits": dl, "dx": dx}


def _exact_root(code, S):
    """The square roots that codes stand for."""
    table = [f / 8 * 2.0 ** -29 for f in range(8)] + [(1 + f / 8) * 2.0 ** (e - 30) for e in range(1, 32) for f in range(8)]
    t = torch.tensor(table, dtype=torch.float64, device=code.device)
    return t[code.to(torch.int64)] * torch.exp2(S.to(torch.float64) - 127)[torch.arange(code.numel(), device=code.device) // 32]


def _exact_round(v, r, above, lowest):
    """Rounded at random to three mantissa bits under a block's scale, down to steps of 2^lowest."""
    n = v.numel()
    b = torch.nn.functional.pad(v, (0, -n % 32)).view(-1, 32)
    top = b.abs().amax(dim=1)
    X = torch.floor(torch.log2(torch.where(top > 0, top, 1.0)))
    X = torch.where(torch.exp2(X) > top, X - 1, X) - above  # a logarithm that rounded up
    X = torch.where(top > 0, X.clamp(-127, 127), torch.full_like(X, -127.0))
    one = torch.exp2(X).repeat_interleave(32)[:n]
    q = v.abs() / one
    e = torch.floor(torch.log2(torch.where(q > 0, q, 1.0)))
    e = torch.where(torch.exp2(e) > q, e - 1, e) - 3
    unit = torch.exp2(torch.where(q > 0, e, torch.full_like(e, float(lowest))).clamp(min=lowest))
    return torch.sign(v) * torch.floor(q / unit + r.to(torch.float64) / 65536) * unit * one, unit * one


def _exact_tensor(s, number, t):
    c, f64 = s.case, torch.float64
    n, step = t.param.numel(), int(s.step)
    if c["bits"] == 8:
        at = torch.arange(n, device="cuda") // 32
        m = t.m.view(torch.float8_e4m3fn).to(f64) * torch.exp2(t.m_scale.to(f64) - 127)[at]
        v = _exact_root(t.v, t.v_scale) ** 2
    else:
        m, v = t.m.to(f64), t.v.to(f64)
    g = t.grad.to(f64) * float(s.scale)
    m = m + (1 - BETA1) * (g - m)
    v = v + (1 - BETA2) * (g * g - v)
    p = (t.param if t.master is None else t.master).to(f64)
    lr = float(s.lr)
    p = p * (1 - lr * t.decay) - lr * (m / (1 - BETA1 ** step)) / ((v / (1 - BETA2 ** step)).sqrt() + EPS)
    got = {"param": p}
    if t.master is not None:
        got["master"] = p
    if c["bits"] == 32:
        return dict(got, m=m, v=v)

    def mixed(x):
        for shift, by in ((16, 0x6A09E667), (15, 0xBB67AE85)):
            x = ((x ^ (x >> shift)) * by) & 0xFFFFFFFF
        return x ^ (x >> 16)

    key = mixed((mixed((mixed(s.seed) + step) % 2 ** 32) + number) % 2 ** 32)
    word = mixed(torch.arange(n, device="cuda") ^ key)
    root = v.sqrt()
    qm, _ = _exact_round(m, word // 65536, 7, -9)
    qv, unit = _exact_round(root, word % 65536, 0, -32)
    return dict(got, m=qm, root_v=torch.where((v > 0) & (qv == 0), unit, qv))


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "ffn":
        return _exact_ffn(s)
    if case["op"] == "rows":
        return _exact_rows(s)
    order = sorted(range(len(s.tensors)), key=lambda i: -s.tensors[i].param.numel())
    return [_exact_tensor(s, i, s.tensors[i]) for i in (order if len(order) <= 12 else order[:4] + order[-8:])]
