"""What a layer does around its product, as measured cases: the forward pass of a linear
layer with bias, activation, dropout and residual in one call, the gradients that its
backward pass needs, and dropout on its own.

Four operators; `rows` are tokens, g(i) the number of row-major element i:

  linear        z = x W^T + b;  y = residual + drop(act(z));  z is returned too where the
                backward pass is to follow (`train`).
  grad          g_z = drop(g_y) act'(z): what reaches the product in the backward pass.
  project_grad  p(g_z): the same, projected block by block onto the r lowest Walsh-Hadamard
                bases (Eq. 3 and 6 of arXiv 2309.15275), which is what Algorithm 1 reads.
  dropout       y = residual + drop(x).

  drop(v)_i = v_i 65536 / (65536 - t) where u_i >= t, else 0, with t = round(65536 p) and u_i
  the 16-bit number i of a counter-based generator: half i % 2 (0: low) of word (i % 8) / 2 of
  Philox4x32-10 (Salmon et al. 2011) at counter (lo(i/8), hi(i/8), lo(o), hi(o) + 2^31) under
  the key (lo(s), hi(s)) of seed s and offset o.  No mask is stored.
  act: none, relu, gelu (erf), gelu_tanh, silu.
"""
import math

import torch

own = False

# --------------------------------------------------------------------- cases ----


def listed():
    lin = lambda name, rows, cin, cout, act, p=0.0, residual=False, train=False, dtype="bf16": dict(  # noqa: E731
        name=name, op="linear", rows=rows, cin=cin, cout=cout, act=act, p=p, residual=residual, train=train, dtype=dtype)
    ele = lambda name, op, rows, c, act, p, residual, dtype: dict(  # noqa: E731
        name=name, op=op, rows=rows, c=c, act=act, p=p, residual=residual, dtype=dtype)
    pro = lambda name, B, H, W, c, k, rank, act, p, dtype: dict(  # noqa: E731
        name=name, op="project_grad", B=B, H=H, W=W, c=c, k=k, rank=rank, act=act, p=p, dtype=dtype)
    return [
        # answering with one token in hand: ViT-B fc1, weights from memory and latency decide
        lin("linear_one_token", 1, 768, 3072, "gelu"),
        # a handful of tokens through fc2 and back onto the residual stream
        lin("linear_few_tokens", 7, 3072, 768, "none", residual=True),
        # training, ViT-B MLP at the benchmark's batch: fc1 with GELU and dropout, z kept
        lin("linear_fc1_train", 32768, 768, 3072, "gelu", p=0.1, train=True),
        # and fc2 with dropout onto the residual stream
        lin("linear_fc2_train", 32768, 3072, 768, "none", p=0.1, residual=True, train=True),
        # an early stage: few channels, many tokens, memory decides
        lin("linear_early_stage", 200704, 48, 192, "gelu", train=True),
        # fp32 training of the last linear layers of a small network on 7 x 7 maps
        lin("linear_last_fp32", 3136, 448, 1792, "gelu", p=0.1, train=True, dtype="fp32"),
        # backward pass of fc1's epilogue at the benchmark's batch
        ele("grad_fc1", "grad", 32768, 3072, "gelu", 0.1, False, "bf16"),
        # the same of a small fp32 layer, an odd number of tokens
        ele("grad_small_fp32", "grad", 49, 1792, "silu", 0.0, False, "fp32"),
        # backward pass of fc1 up to the coefficients that Algorithm 1 reads
        pro("project_grad_fc1", 128, 16, 16, 3072, 8, 8, "gelu", 0.1, "bf16"),
        # the same on 7 x 7 maps, which the blocks hang over, at the rank of LP_L1-4
        pro("project_grad_last_fp32", 64, 7, 7, 1792, 8, 10, "gelu", 0.1, "fp32"),
        # dropout of token sequences with a class token, onto the residual stream
        ele("dropout_sequence", "dropout", 128 * 197, 768, "none", 0.1, True, "bf16"),
        # dropout of one small map in fp32: latency
        ele("dropout_small_fp32", "dropout", 49, 448, "none", 0.5, False, "fp32"),
    ]


ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")


def _log(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def _channels(rng, lo, hi):
    """Mostly multiples of 64 as in real networks, some of 8 only."""
    step = 8 if rng.random() < 0.3 else 64 if hi > 64 else 16
    return max(step, int(round(_log(rng, lo, hi) / step)) * step)


def draw(rng):
    op = rng.choice(["linear", "linear", "linear", "grad", "project_grad", "dropout"])
    dtype = "fp32" if rng.random() < 0.25 else "bf16"
    p = rng.choice([0.0, 0.1, round(rng.uniform(0.02, 0.6), 3)])
    case = {"op": op, "dtype": dtype, "act": rng.choice(ACTS if op != "dropout" else ("none",)), "p": p}
    if op == "linear":
        a, b = _channels(rng, 48, 1024), rng.choice([1, 1, 3, 4])
        case["cin"], case["cout"] = (a, a * b) if rng.random() < 0.6 else (a * b, a)
        # one token, some, or up to the work of the largest listed case
        most = 1.5e11 / (2.0 * case["cin"] * case["cout"])
        most = min(most, 200704.0, 2.4e8 / (case["cin"] + 2 * case["cout"]))
        case["rows"] = 1 if rng.random() < 0.1 else max(1, int(_log(rng, 1.0, most)))
        case["residual"] = rng.random() < 0.5
        case["train"] = rng.random() < 0.6
    elif op == "project_grad":
        case["c"] = _channels(rng, 48, 4096)
        case["H"] = rng.choice([7, 14, 16, 28, 32, int(_log(rng, 5, 64))])
        case["W"] = case["H"] if rng.random() < 0.7 else max(4, int(case["H"] * rng.uniform(0.6, 1.6)))
        case["k"] = rng.choice([4, 8, 8, 16])
        most = min(case["k"] ** 2 - 1, 36)
        case["rank"] = max(1, min(most, int(round(_log(rng, 1, most)))))
        case["B"] = max(1, int(_log(rng, 1.0, max(1.01, 1.0e8 / (case["H"] * case["W"] * case["c"])))))
    else:
        case["c"] = _channels(rng, 48, 4096)
        case["rows"] = max(1, int(_log(rng, 1.0, min(200704.0, 1.0e8 / case["c"]))))
        case["residual"] = op == "dropout" and rng.random() < 0.5
    return case


def work(case):
    es = 4 if case["dtype"] == "fp32" else 2
    if case["op"] == "linear":
        m, a, b = case["rows"], case["cin"], case["cout"]
        outs = 1 + (1 if case["residual"] else 0) + (1 if _keeps_z(case) else 0)
        return {"bytes": es * (m * a + a * b + b + outs * m * b), "flops": 2.0 * m * a * b}
    if case["op"] == "project_grad":
        n, c, k = case["B"] * case["H"] * case["W"], case["c"], case["k"]
        blocks = case["B"] * -(-case["H"] // k) * -(-case["W"] // k)
        ins = 1 if case["act"] == "none" else 2
        return {"bytes": es * c * (ins * n + blocks * case["rank"]), "flops": 2.0 * n * c * case["rank"]}
    n = case["rows"] * case["c"]
    tensors = 2 + (1 if case["op"] == "grad" and case["act"] != "none" else 0) + (1 if case["residual"] else 0)
    return {"bytes": es * n * tensors, "flops": float(n)}


# -------------------------------------------------------------------- inputs ----


def _dtype(case):
    return torch.float32 if case["dtype"] == "fp32" else torch.bfloat16


def _keeps_z(case):
    return bool(case["train"]) and case["act"] != "none"


def _walsh(k):
    """Rows of +-1 by number of sign changes."""
    h = torch.ones(1, 1, dtype=torch.float64)
    while h.shape[0] < k:
        h = torch.cat([torch.cat([h, h], 1), torch.cat([h, -h], 1)], 0)
    changes = (h[:, 1:] != h[:, :-1]).sum(1)
    return h[torch.argsort(changes)]


def _bases(k, rank):
    """The `rank` lowest pairs in the order (i + j, max(i, j), i)."""
    pairs = sorted(((i, j) for i in range(k) for j in range(k)), key=lambda q: (q[0] + q[1], max(q), q[0]))
    return pairs[:rank]


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dt = _dtype(case)
    normal = lambda shape, std=1.0: torch.randn(shape, generator=g, device="cuda").mul_(std).to(dt)  # noqa: E731
    s = dict(case, seed=(seed * 0x9E3779B97F4A7C15 + 0x1234567) % 2 ** 63, offset=4 * (seed % 1000003))
    if case["op"] == "linear":
        s["x"] = normal((case["rows"], case["cin"]))
        s["W"] = normal((case["cout"], case["cin"]), case["cin"] ** -0.5)
        s["b"] = normal((case["cout"],), 0.1)
        s["res"] = normal((case["rows"], case["cout"])) if case["residual"] else None
    elif case["op"] == "dropout":
        s["x"] = normal((case["rows"], case["c"]))
        s["res"] = normal((case["rows"], case["c"])) if case["residual"] else None
    else:
        shape = ((case["rows"], case["c"]) if case["op"] == "grad"
                 else (case["B"], case["H"], case["W"], case["c"]))
        s["gy"] = normal(shape, 0.01)
        s["z"] = normal(shape) if case["act"] != "none" else None
        if case["op"] == "project_grad":
            s["bases"] = _bases(case["k"], case["rank"])
            walsh = _walsh(case["k"])
            s["matrix"] = torch.stack([torch.outer(walsh[i], walsh[j]) / case["k"]
                                       for i, j in s["bases"]]).float().cuda()   # (r, k, k)
    return s


# --------------------------------------------------------------- plain form ----


def _mul32(a, b):
    """High and low word of the product of 32-bit numbers (held in int64; the product wraps)."""
    full = a * b
    return (full >> 32) & 0xFFFFFFFF, full & 0xFFFFFFFF


def _u16(n, seed, offset, device):
    """The first n 16-bit numbers of the generator."""
    i = torch.arange((n + 7) // 8, dtype=torch.int64, device=device)
    c0, c1 = i & 0xFFFFFFFF, i >> 32
    c2 = torch.full_like(i, offset & 0xFFFFFFFF)
    c3 = torch.full_like(i, ((offset >> 32) + 0x80000000) & 0xFFFFFFFF)
    k0, k1 = seed & 0xFFFFFFFF, (seed >> 32) & 0xFFFFFFFF
    for _ in range(10):
        h0, l0 = _mul32(c0, 0xD2511F53)
        h1, l1 = _mul32(c2, 0xCD9E8D57)
        c0, c1, c2, c3 = h1 ^ c1 ^ k0, l1, h0 ^ c3 ^ k1, l0
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    words = torch.stack([c0, c1, c2, c3], 1)
    return torch.stack([words & 0xFFFF, words >> 16], 2).reshape(-1)[:n]


def _drop(v, s):
    t = int(round(65536 * s["p"]))
    if t == 0:
        return v
    keep = _u16(v.numel(), s["seed"], s["offset"], v.device).reshape(v.shape) >= t
    return torch.where(keep, v * (65536.0 / (65536 - t)), torch.zeros_like(v))


_ROOT_HALF = math.sqrt(0.5)
_TANH_A, _TANH_B = math.sqrt(2.0 / math.pi), 0.044715


def _act(z, act):
    if act == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if act == "gelu":
        return 0.5 * z * torch.erfc(-z * _ROOT_HALF)
    if act == "gelu_tanh":
        return 0.5 * z * (1.0 + torch.tanh(_TANH_A * (z + _TANH_B * z * z * z)))
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    return z


def _dact(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        return 0.5 * torch.erfc(-z * _ROOT_HALF) + z * torch.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    if act == "gelu_tanh":
        t = torch.tanh(_TANH_A * (z + _TANH_B * z * z * z))
        return 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * _TANH_A * (1.0 + 3.0 * _TANH_B * z * z)
    if act == "silu":
        e = 1.0 / (1.0 + torch.exp(-z))
        return e * (1.0 + z * (1.0 - e))
    return torch.ones_like(z)


def _grad(s):
    v = _drop(s["gy"].float(), s)
    return v if s["z"] is None else v * _dact(s["z"].float(), s["act"])


def _blocks(t, k):
    """(B, H, W, C) -> (B, Hb, k, Wb, k, C), zero tokens past the high end."""
    B, H, W, C = t.shape
    hb, wb = -(-H // k), -(-W // k)
    full = t.new_zeros((B, hb * k, wb * k, C))
    full[:, :H, :W] = t
    return full.reshape(B, hb, k, wb, k, C)


def _plain(s):
    dt = _dtype(s)
    if s["op"] == "linear":
        z = s["x"].float() @ s["W"].float().t() + s["b"].float()
        y = _drop(_act(z, s["act"]), s)
        if s["res"] is not None:
            y = s["res"].float() + y
        return [y.to(dt), z.to(dt)] if _keeps_z(s) else [y.to(dt)]
    if s["op"] == "dropout":
        y = _drop(s["x"].float(), s)
        return [(y if s["res"] is None else s["res"].float() + y).to(dt)]
    if s["op"] == "grad":
        return [_grad(s).to(dt)]
    t = _blocks(_grad(s), s["k"])
    return [torch.einsum("quv,bhuwvc->bhwqc", s["matrix"], t).to(dt)]


def run(state):
    s = state
    if not own:
        return _plain(s)
    import paper_2309_15275_b200 as lbp
    more = {"p": s["p"], "seed": s["seed"], "offset": s["offset"]}
    if s["op"] == "linear":
        got = lbp.lbp_linear(s["x"], s["W"], s["b"], activation=s["act"], residual=s["res"],
                             save_z=_keeps_z(s), **more)
        return list(got) if _keeps_z(s) else [got]
    if s["op"] == "dropout":
        return [lbp.lbp_dropout(s["x"], residual=s["res"], **more)]
    if s["op"] == "grad":
        return [lbp.lbp_linear_grad(s["gy"], s["z"], activation=s["act"], **more)]
    return [lbp.lbp_project_grad(s["gy"], s["z"], s["k"], s["bases"], activation=s["act"], **more)]


# ---------------------------------------------------------------- definition ----


def _keep_exact(n, seed, offset, t):
    """Which of n numbers are at least t, element by element from the definition."""
    e = torch.arange(n, dtype=torch.int64, device="cuda")
    mask = 2 ** 32 - 1
    ctr = [(e // 8) % 2 ** 32, (e // 8) // 2 ** 32,
           torch.zeros_like(e) + offset % 2 ** 32, torch.zeros_like(e) + (offset // 2 ** 32 + 2 ** 31) % 2 ** 32]
    key = [seed % 2 ** 32, seed // 2 ** 32 % 2 ** 32]

    def hi_lo(a, m):   # in 16-bit halves, so that nothing wraps
        p0, p1 = (a & 0xFFFF) * m, (a >> 16) * m
        mid = (p0 >> 16) + (p1 & 0xFFFFFFFF)
        return (p1 >> 32 << 16) + (mid >> 16), ((mid & 0xFFFF) << 16) | (p0 & 0xFFFF)

    for r in range(10):
        (ah, al), (bh, bl) = hi_lo(ctr[0], 0xD2511F53), hi_lo(ctr[2], 0xCD9E8D57)
        ka, kb = (key[0] + r * 0x9E3779B9) & mask, (key[1] + r * 0xBB67AE85) & mask
        ctr = [bh ^ ctr[1] ^ ka, bl, ah ^ ctr[3] ^ kb, al]
    w = e % 8 // 2
    word = torch.where(w == 0, ctr[0], torch.where(w == 1, ctr[1], torch.where(w == 2, ctr[2], ctr[3])))
    return ((word >> (16 * (e % 2))) & 0xFFFF) >= t


def exact(case, seed):
    s = prepare(case, seed)
    d = lambda v: v.double()  # noqa: E731
    t = math.floor(65536 * s["p"] + 0.5)

    def dropped(v):
        if t == 0:
            return v
        keep = _keep_exact(v.numel(), s["seed"], s["offset"], t).view(v.shape)
        return v.mul(65536).div(65536 - t).masked_fill(~keep, 0.0)

    def phi(v):   # of the normal distribution
        return torch.special.ndtr(v)

    def inner(v):
        return math.sqrt(2 / math.pi) * (v + 0.044715 * v ** 3)

    act = s["act"]
    f = {"none": lambda v: v, "relu": lambda v: v.clamp(min=0), "gelu": lambda v: v * phi(v),
         "gelu_tanh": lambda v: v * torch.sigmoid(2 * inner(v)), "silu": lambda v: v * torch.sigmoid(v)}[act]

    def slope(v):
        if act == "none":
            return torch.ones_like(v)
        if act == "relu":
            return (v > 0).double()
        if act == "gelu":
            return phi(v) + v * torch.exp(-v * v / 2) / math.sqrt(2 * math.pi)
        if act == "silu":
            return torch.sigmoid(v) * (1 + v * torch.sigmoid(-v))
        u = 2 * inner(v)
        return torch.sigmoid(u) + v * torch.sigmoid(u) * torch.sigmoid(-u) * 2 * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * v * v)

    if s["op"] == "linear":
        z = torch.nn.functional.linear(d(s["x"]), d(s["W"]), d(s["b"]))
        y = dropped(f(z))
        y = y if s["res"] is None else y + d(s["res"])
        return [y, z] if _keeps_z(s) else [y]
    if s["op"] == "dropout":
        y = dropped(d(s["x"]))
        return [y if s["res"] is None else y + d(s["res"])]
    g = dropped(d(s["gy"]))
    g = g if s["z"] is None else g * slope(d(s["z"]))
    if s["op"] == "grad":
        return [g]
    k = s["k"]
    g = torch.nn.functional.pad(g, (0, 0, 0, -g.shape[2] % k, 0, -g.shape[1] % k))
    w = _walsh(k).cuda() / math.sqrt(k)
    # both sides of every block at once, then the chosen pairs
    B, H, W, C = g.shape
    g = g.view(B, H // k, k, W // k, k, C)
    rows = torch.einsum("iu,bhuwvc->bhwivc", w, g)
    both = torch.einsum("jv,bhwivc->bhwijc", w, rows)
    return [torch.stack([both[:, :, :, i, j] for i, j in s["bases"]], 3)]
