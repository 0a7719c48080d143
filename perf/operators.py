"""Performance cases of the operators that a batched MLA decode with quantised weights and a quantised cache uses.

Four kinds of case (the field ``kind``):

* ``w4``         nmm_gemv_w4, y = x . W^T with W [N, K] in 4 bits and a scale per group of K: integers with
                 16-bit scales (optionally zero points), or e2m1 values with a power of two per 32
* ``write``      nmm_latent_cache_write and nmm_latent_cache_read: RMSNorm, RoPE and the 8-bit cache rows of many
                 tokens at once, read back as bf16
* ``read``       nmm_latent_cache_read alone, a context's rows out of the 8-bit cache
* ``attention``  nmm_latent_attention_batch over a paged latent cache (bf16 or 8-bit rows) whose sequences
                 share a prefix

With ``own`` false every case is computed in its plain form, elementary torch operations in 32 bits.
"""
import math

import torch

own = False

# DeepSeek-V3's MLA dimensions
HIDDEN, Q_LORA, KV_LORA, ROPE, NOPE = 7168, 1536, 512, 64, 128
D = KV_LORA + ROPE
SCALE = 1.0 / math.sqrt(NOPE + ROPE)
EPS, THETA = 1e-6, 10000.0
BLOCK = 32                          # latent values that share a scale in an 8-bit cache row
ROW_BYTES = KV_LORA + 16 + 2 * ROPE
E_MIN = -117                        # the lowest scale exponent of a row: what it stands for stays a normal bf16 number
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
MAX_WEIGHT = 16384 * 7168
MAX_PAIRS = 2048 * 10240            # (sequence, head) rows x positions of the largest attention


def listed():
    return [
        # the smallest call: a 512 x 512 projection of one token, all launch latency
        {"name": "w4_512", "kind": "w4", "M": 1, "K": 512, "N": 512, "fp16": False, "format": "int", "group": 128,
         "zeros": False},
        # the output projection of one token, the largest weight of a layer
        {"name": "w4_w_o", "kind": "w4", "M": 1, "K": 16384, "N": HIDDEN, "fp16": False, "format": "int", "group": 128,
         "zeros": False},
        # W_UQ for eight tokens in the power-of-two format
        {"name": "w4_w_uq_8", "kind": "w4", "M": 8, "K": Q_LORA, "N": 24576, "fp16": False, "format": "mx", "group": 32,
         "zeros": False},
        # no size a multiple of a tile, the last group cut short, zero points, fp16
        {"name": "w4_ragged_5", "kind": "w4", "M": 5, "K": 4099, "N": 5003, "fp16": True, "format": "int", "group": 64,
         "zeros": True},
        # the output projection of a batch of 32
        {"name": "w4_w_o_32", "kind": "w4", "M": 32, "K": 16384, "N": HIDDEN, "fp16": False, "format": "int",
         "group": 128, "zeros": False},
        # the cache rows of one step of a decode batch
        {"name": "write_64", "kind": "write", "tokens": 64, "rows": 65536},
        # the cache rows of a prefill chunk
        {"name": "write_8192", "kind": "write", "tokens": 8192, "rows": 65536},
        # a long context's rows as bf16, for a prefill over it
        {"name": "read_40001", "kind": "read", "tokens": 40001, "rows": 65536},
        # one sequence of few tokens on a tensor-parallel shard of 16 heads, all launch latency
        {"name": "attention_1x16x200", "kind": "attention", "B": 1, "T": 1, "H": 16, "prefix": 0, "own": 200,
         "page": 64, "fp8": True},
        # a batch on such a shard without a shared prefix, long ragged sequences: the cache's bytes
        {"name": "attention_64x16x4097", "kind": "attention", "B": 64, "T": 1, "H": 16, "prefix": 0, "own": 4097,
         "page": 64, "fp8": True},
        # a batch of 32 on such a shard behind one system prompt, two tokens a sequence (speculative decode)
        {"name": "attention_32x2x16_prefix", "kind": "attention", "B": 32, "T": 2, "H": 16, "prefix": 16000,
         "own": 301, "page": 32, "fp8": True},
        # all heads, a batch of 16 behind one prompt, bf16 rows: the matrix cores' work
        {"name": "attention_16x128_prefix", "kind": "attention", "B": 16, "T": 1, "H": 128, "prefix": 8192,
         "own": 1024, "page": 64, "fp8": False},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """A size between lo and hi over its logarithm: half of them any number, half a multiple of 64."""
    v = _log(rng, lo, hi)
    return v if rng.random() < 0.5 else max(lo, v // 64 * 64)


def draw(rng):
    kind = rng.choice(["w4", "w4", "w4", "write", "read", "attention", "attention", "attention"])
    if kind == "w4":
        M = 1 if rng.random() < 0.3 else _log(rng, 1, 32)
        K = _size(rng, 512, 16384)
        N = _size(rng, 512, min(24576, MAX_WEIGHT // K))
        mx = rng.random() < 0.4
        return {"kind": kind, "M": M, "K": K, "N": N, "fp16": rng.random() < 0.3, "format": "mx" if mx else "int",
                "group": 32 if mx else rng.choice([32, 64, 128]), "zeros": not mx and rng.random() < 0.5}
    if kind in ("write", "read"):
        return {"kind": kind, "tokens": _log(rng, 1, 8192 if kind == "write" else 40001), "rows": 65536}
    H = rng.choice([8, 16, 32, 64, 128]) if rng.random() < 0.7 else _log(rng, 8, 128)
    B, T = _log(rng, 1, 64), rng.choice([1, 1, 1, 2])
    most = max(64, min(40000, MAX_PAIRS // (B * T * H)))
    prefix = 0 if rng.random() < 0.3 else _size(rng, 64, max(65, most * 3 // 4))
    return {"kind": kind, "B": B, "T": T, "H": H, "prefix": prefix,
            "own": _size(rng, 1 + T, max(2 + T, min(4097, most // 4))), "page": rng.choice([16, 32, 64, 128]),
            "fp8": rng.random() < 0.6}


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed) * 7919 + 29)


def _normal(g, shape, sigma=1.0):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32) * sigma


def _lens(case):
    """The sequences' own lengths: ragged, between the longest and half of it."""
    B, longest = case["B"], case["own"]
    return [longest - (b * longest) // (2 * B) for b in range(B)]


def _quantise_w4(w, case):
    """A weight [N, K] in the case's 4-bit format: packed codes, scales and zero points."""
    N, K = w.shape
    G = case["group"]
    n_groups = (K + G - 1) // G
    wg = torch.nn.functional.pad(w, (0, n_groups * G - K)).view(N, n_groups, G)
    zeros = None
    if case["format"] == "mx":
        amax = wg.abs().amax(-1, keepdim=True).clamp(min=2.0 ** -100)
        e = torch.floor(torch.log2(amax)) - 2
        mag = (wg * torch.exp2(-e)).abs()
        grid = torch.tensor(E2M1, device=w.device)
        code = torch.bucketize(mag, (grid[1:] + grid[:-1]) / 2).to(torch.uint8)
        code = code | ((wg < 0).to(torch.uint8) << 3)
        scales = (e[..., 0] + 127).to(torch.uint8)
    elif case["zeros"]:
        lo, hi = wg.amin(-1, keepdim=True).clamp(max=0), wg.amax(-1, keepdim=True).clamp(min=0)
        s = ((hi - lo) / 15).clamp(min=2.0 ** -24)
        z = torch.round(-lo / s).clamp(0, 15)
        code = (torch.round(wg / s) + z).clamp(0, 15).to(torch.uint8)
        zeros, scales = z[..., 0].to(torch.uint8).contiguous(), s[..., 0]
    else:
        s = (wg.abs().amax(-1, keepdim=True) / 7).clamp(min=2.0 ** -24)
        code = (torch.round(wg / s) + 8).clamp(0, 15).to(torch.uint8)
        scales = s[..., 0]
    if case["format"] != "mx":
        scales = scales.to(torch.float16 if case["fp16"] else torch.bfloat16)
    code = torch.nn.functional.pad(code.view(N, n_groups * G)[:, :K], (0, -K % 32))
    return (code[:, 0::2] | (code[:, 1::2] << 4)).contiguous(), scales.contiguous(), zeros


def _pack(rows):
    """bf16 cache rows [n, 576] as 8-bit rows [n, 656]: codes, scale bytes, the RoPE part as it is."""
    v = rows[:, :KV_LORA].float().view(-1, KV_LORA // BLOCK, BLOCK)
    amax = v.abs().amax(-1, keepdim=True)
    m, x = torch.frexp(amax)                      # amax = m 2^x, m in [0.5, 1): 448 = 0.875 2^9
    e = (x - 9 + (m > 0.875)).clamp(min=E_MIN)
    code = (v * torch.exp2(-e.float())).to(torch.float8_e4m3fn).view(torch.uint8).view(-1, KV_LORA)
    return torch.cat((code, (e[..., 0] + 127).to(torch.uint8), rows[:, KV_LORA:].contiguous().view(torch.uint8)), 1)


def _unpack(rows):
    """What 8-bit cache rows [n, 656] stand for, in fp32."""
    code = rows[:, :KV_LORA].contiguous().view(torch.float8_e4m3fn).float().view(-1, KV_LORA // BLOCK, BLOCK)
    scale = torch.exp2(rows[:, KV_LORA:KV_LORA + 16].float() - 127.0)
    rope = rows[:, KV_LORA + 16:].contiguous().view(torch.bfloat16).float()
    return torch.cat(((code * scale[..., None]).view(-1, KV_LORA), rope), 1)


def prepare(case, seed):
    g = _gen(seed)
    s = {"case": case}
    kind = case["kind"]
    if kind == "w4":
        M, K, N = case["M"], case["K"], case["N"]
        dt = torch.float16 if case["fp16"] else torch.bfloat16
        s["x"] = _normal(g, (M, (K + 7) // 8 * 8)).to(dt)
        s["Wq"], s["scales"], s["zeros"] = _quantise_w4(_normal(g, (N, K), K ** -0.5), case)
        s["y"] = torch.zeros((M, N), device="cuda")
        return s
    if kind in ("write", "read"):
        T = case["tokens"]
        s["slots"] = torch.randperm(case["rows"], generator=g, device="cuda")[:T].contiguous()
        if kind == "write":
            s["mm"] = _normal(g, (T, D))
            s["gamma"] = (1.0 + 0.1 * _normal(g, (KV_LORA,))).to(torch.bfloat16)
            s["positions"] = torch.randint(0, 131072, (T,), generator=g, device="cuda")
            s["cache"] = torch.zeros((case["rows"], ROW_BYTES), dtype=torch.uint8, device="cuda")
        else:
            s["cache"] = _pack(_normal(g, (case["rows"], D)).to(torch.bfloat16))
        s["out"] = torch.zeros((T, D), dtype=torch.bfloat16, device="cuda")
        return s
    B, T, H, page = case["B"], case["T"], case["H"], case["page"]
    pages_of = lambda n: (n + page - 1) // page
    n_own, n_pre = pages_of(case["own"]), pages_of(case["prefix"])
    n_pages = n_pre + B * n_own + 3
    order = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    rows = _normal(g, (n_pages * page, D)).to(torch.bfloat16)
    s["cache"] = _pack(rows) if case["fp8"] else rows
    s["prefix_pages"] = order[:n_pre].contiguous()
    s["pages"] = order[n_pre:n_pre + B * n_own].view(B, n_own).contiguous()
    s["lens"] = torch.tensor(_lens(case), dtype=torch.int32, device="cuda")
    s["q"] = _normal(g, (B, T, H, D)).to(torch.bfloat16)
    s["out"] = torch.zeros((B, T, H, KV_LORA), dtype=torch.bfloat16, device="cuda")
    return s


def _w4_plain(s):
    case = s["case"]
    N, K, G = case["N"], case["K"], case["group"]
    q = s["Wq"]
    code = torch.stack((q & 15, q >> 4), -1).view(N, -1)[:, :K]
    if case["format"] == "mx":
        w = torch.tensor(E2M1 + tuple(-v for v in E2M1), device=q.device)[code.int()]
        scale = torch.exp2(s["scales"].float() - 127.0)
    else:
        zero = s["zeros"].float().repeat_interleave(G, 1)[:, :K] if case["zeros"] else 8.0
        w = code.float() - zero
        scale = s["scales"].float()
    w = w * scale.repeat_interleave(G, 1)[:, :K]
    return s["x"][:, :K].float() @ w.T


def _rope(k, positions):
    """RoPE of adjacent pairs; the angles in 64 bits."""
    i = torch.arange(ROPE // 2, dtype=torch.float64, device=k.device)
    a = positions.double()[:, None] * THETA ** (-2.0 * i / ROPE)
    c, s = torch.cos(a).to(k.dtype), torch.sin(a).to(k.dtype)
    k0, k1 = k[:, 0::2], k[:, 1::2]
    return torch.stack((k0 * c - k1 * s, k0 * s + k1 * c), -1).reshape(k.shape)


def _gather(cache, pages, page):
    """The rows of the pages in `pages` [..., n], as fp32 [..., n * page, 576]."""
    at = pages.long()[..., None] * page + torch.arange(page, device=pages.device)
    rows = cache[at.reshape(-1)]
    rows = _unpack(rows) if cache.dtype == torch.uint8 else rows.float()
    return rows.view(*pages.shape[:-1], -1, D)


def _attention_plain(s):
    case = s["case"]
    B, T, H, P = case["B"], case["T"], case["H"], case["prefix"]
    q = s["q"].float().view(B, T * H, D) * SCALE
    kv = _gather(s["cache"], s["pages"], case["page"])
    at = torch.arange(kv.shape[1], device=kv.device)
    limit = s["lens"][:, None] - (T - 1) + torch.arange(T, device=kv.device)
    seen = (at < limit[..., None]).repeat_interleave(H, 1)            # [B, T * H, positions]
    kv = torch.where((at < s["lens"][:, None])[..., None], kv, 0.0)
    score = torch.where(seen, q @ kv.transpose(1, 2).contiguous(), -math.inf)
    if P:
        pre = _gather(s["cache"], s["prefix_pages"], case["page"])[:P]
        score_p = (q.view(-1, D) @ pre.T).view(B, T * H, P)
        top = torch.maximum(score.amax(-1, keepdim=True), score_p.amax(-1, keepdim=True))
    else:
        top = score.amax(-1, keepdim=True)
    p = torch.exp(score - top)
    total, out = p.sum(-1, keepdim=True), p @ kv[..., :KV_LORA].contiguous()
    if P:
        p = torch.exp(score_p - top)
        total = total + p.sum(-1, keepdim=True)
        out = out + (p.view(-1, P) @ pre[:, :KV_LORA]).view(B, T * H, KV_LORA)
    return (out / total).to(torch.bfloat16).view(B, T, H, KV_LORA)


def run(s):
    case = s["case"]
    kind = case["kind"]
    if own:
        import paper_2609_16009_amd as nmm

        if kind == "w4":
            return nmm.nmm_gemv_w4(s["x"], s["Wq"], s["scales"], s["y"], group=case["group"], zeros=s["zeros"],
                                   K=case["K"])
        if kind == "attention":
            return nmm.nmm_latent_attention_batch(s["q"], s["cache"], s["out"], SCALE, kv_lora=KV_LORA, rope=ROPE,
                                                  page_size=case["page"], pages=s["pages"], lens=s["lens"],
                                                  max_len=case["own"], prefix_pages=s["prefix_pages"],
                                                  prefix_len=case["prefix"])
        if kind == "write":
            nmm.nmm_latent_cache_write(s["mm"], s["slots"], s["cache"], kv_lora=KV_LORA, rope=ROPE, gamma=s["gamma"],
                                       eps=EPS, positions=s["positions"], theta=THETA)
        return nmm.nmm_latent_cache_read(s["cache"], s["slots"], s["out"], kv_lora=KV_LORA, rope=ROPE)
    if kind == "w4":
        return _w4_plain(s)
    if kind == "attention":
        return _attention_plain(s)
    if kind == "write":
        c = s["mm"][:, :KV_LORA]
        c = c * torch.rsqrt((c * c).mean(-1, keepdim=True) + EPS) * s["gamma"].float()
        entry = torch.cat((c, _rope(s["mm"][:, KV_LORA:], s["positions"])), 1).to(torch.bfloat16)
        s["cache"][s["slots"]] = _pack(entry)
    return _unpack(s["cache"][s["slots"]]).to(torch.bfloat16)


def work(case):
    kind = case["kind"]
    if kind == "w4":
        M, K, N = case["M"], case["K"], case["N"]
        groups = (K + case["group"] - 1) // case["group"]
        per_group = 1 if case["format"] == "mx" else 3 if case["zeros"] else 2
        return {"bytes": N * ((K + 1) // 2 + groups * per_group) + M * K * 2 + M * N * 4, "flops": 2 * M * N * K}
    if kind in ("write", "read"):
        T = case["tokens"]
        read = T * (8 + ROW_BYTES + 2 * D)
        if kind == "read":
            return {"bytes": read, "flops": T * KV_LORA}
        return {"bytes": read + T * (4 * D + 8 + ROW_BYTES) + 2 * KV_LORA, "flops": T * (8 * KV_LORA + 8 * ROPE)}
    B, T, H, P = case["B"], case["T"], case["H"], case["prefix"]
    lens = _lens(case)
    row = ROW_BYTES if case["fp8"] else 2 * D
    pairs = sum(T * H * (P + n) for n in lens)
    return {"bytes": (P + sum(lens)) * row + B * T * H * 2 * (D + KV_LORA), "flops": 2 * pairs * (D + KV_LORA)}


def _w4_exact(s):
    case = s["case"]
    M, K, N, G = case["M"], case["K"], case["N"], case["group"]
    y = torch.zeros((M, N), dtype=torch.float64, device="cuda")
    x = s["x"].double()
    for k0 in range(0, K, G):
        k1 = min(K, k0 + G)
        byte = s["Wq"][:, k0 // 2:(k1 + 1) // 2].long()
        code = torch.empty((N, 2 * byte.shape[1]), dtype=torch.long, device="cuda")
        code[:, 0::2], code[:, 1::2] = byte % 16, byte // 16
        code = code[:, :k1 - k0]
        scale = s["scales"][:, k0 // G]
        if case["format"] == "mx":
            mag, sign = code % 8, 1.0 - 2.0 * (code // 8).double()
            # e2m1: two exponent bits, one of mantissa; exponent 0 holds 0 and 1/2
            ex, man = mag // 2, (mag % 2).double()
            val = torch.where(ex == 0, 0.5 * man, (1.0 + 0.5 * man) * 2.0 ** (ex.double() - 1.0)) * sign
            scale = torch.ldexp(torch.ones(N, dtype=torch.float64, device="cuda"), scale.int() - 127)
        else:
            val = code.double() - (s["zeros"][:, k0 // G].double()[:, None] if case["zeros"] else 8.0)
            scale = scale.double()
        y += (x[:, k0:k1] @ val.T.contiguous()) * scale
    return y


def _entry_exact(s):
    """The cache entries in 64 bits, rounded to bf16 and their latent part to 8 bits as the cache holds them."""
    mm = s["mm"].double()
    c = mm[:, :KV_LORA]
    c = c / torch.sqrt((c ** 2).sum(1, keepdim=True) / KV_LORA + EPS) * s["gamma"].double()
    z = torch.view_as_complex(mm[:, KV_LORA:].reshape(-1, ROPE // 2, 2).contiguous())
    freq = torch.pow(torch.tensor(THETA, dtype=torch.float64, device="cuda"),
                     -torch.arange(0, ROPE, 2, dtype=torch.float64, device="cuda") / ROPE)
    angle = torch.outer(s["positions"].double(), freq)
    k = torch.view_as_real(z * torch.polar(torch.ones_like(angle), angle)).reshape(-1, ROPE)
    c, k = c.to(torch.bfloat16).double(), k.to(torch.bfloat16).double()
    blocks = c.view(-1, KV_LORA // BLOCK, BLOCK)
    e = torch.ceil(torch.log2(blocks.abs().amax(-1, keepdim=True).clamp(min=2.0 ** -140) / 448)).clamp(min=E_MIN)
    v = blocks * torch.exp2(-e)
    # e4m3: steps of 2^(exponent - 3), at least 2^-9
    step = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -20))).clamp(min=-6) - 3)
    return torch.cat(((torch.round(v / step) * step * torch.exp2(e)).view(-1, KV_LORA), k), 1)


def _rows_exact(rows):
    """8-bit cache rows in 64 bits, from the bits of their codes."""
    code = rows[:, :KV_LORA].long()
    sign, ex, man = 1.0 - 2.0 * (code // 128).double(), (code // 8) % 16, (code % 8).double()
    v = sign * torch.where(ex == 0, man / 8 * 2.0 ** -6, (1 + man / 8) * torch.exp2(ex.double() - 7))
    v = v.view(-1, KV_LORA // BLOCK, BLOCK) * torch.exp2(rows[:, KV_LORA:KV_LORA + 16].double() - 127)[..., None]
    return torch.cat((v.view(-1, KV_LORA), rows[:, KV_LORA + 16:].contiguous().view(torch.bfloat16).double()), 1)


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "w4":
        return _w4_exact(s)
    if kind == "write":
        return _entry_exact(s)
    if kind == "read":
        return _rows_exact(s["cache"][s["slots"]])
    B, T, H, P, page = case["B"], case["T"], case["H"], case["prefix"], case["page"]
    out = torch.empty((B, T, H, KV_LORA), dtype=torch.float64, device="cuda")

    def rows_of(pages, n):
        at = (pages.long()[:, None] * page + torch.arange(page, device="cuda")).reshape(-1)[:n]
        rows = s["cache"][at]
        return _rows_exact(rows) if case["fp8"] else rows.double()

    shared = rows_of(s["prefix_pages"], P)
    for b, n in enumerate(_lens(case)):
        mine = torch.cat((shared, rows_of(s["pages"][b], n)))
        for t in range(T):
            ctx = mine[:P + n - (T - 1 - t)]
            p = torch.softmax(SCALE * (s["q"][b, t].double() @ ctx.T.contiguous()), dim=-1)
            out[b, t] = p @ ctx[:, :KV_LORA].contiguous()
    return out
