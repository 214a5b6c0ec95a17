"""The 4-bit operators and the token log-probabilities of the library, as cases that can be timed and compared.

Four kinds of case; each is what a program that serves a masked-diffusion model does around its forwards:

  quantize   rows to microscaled 4-bit floating point (E2M1 codes, a scale byte per 16 or 32 channels), with the
             values that the codes stand for, as a program that calibrates or stores activations and weights wants them
  matmul     a projection with 4-bit weights: activation rows are quantised and multiplied with weights that were
             quantised and laid out when the model was loaded
  kv4        a cache of keys and values in 4 bits: new rows are written at their positions ("append"), query rows attend
             over the cache ("attend"), or both as in a denoising step ("step")
  logprobs   log-probability of a given token, entropy and the most likely alternatives of every logits row

Sizes are those of `inputs.config` and of the benchmark (d_model 4096 / 3584, 32 / 32, 28 / 4 and 4 / 4 heads, vocabularies
126464 / 152064, blocks of 32, sequences of 512 to 65536 positions) or generic odd ones around them.

Definitions (`x` rows of `d` channels, groups of g = 16 ("nv") or 32 ("mx") channels, t = a positive factor of the tensor):

  nv  s = E4M3(amax / 6 t), nearest even, saturating at 448
  mx  s = 2^clamp(floor(log2(amax / t)) - 2, -127, 127)
  code = the value of {0, .5, 1, 1.5, 2, 3, 4, 6} nearest to |x| / (s t), ties to the even code, saturating, with x's sign
  stored value = code s t;  a group with an infinity or NaN has the scale NaN;  a group whose s is 0 is 0
"""
import math

import torch

own = False

GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
HEADS = {"llada": (32, 32, 128), "dream": (28, 4, 128), "tiny": (4, 4, 64)}
SCALE_TYPES = {"nv": torch.float8_e4m3fn, "mx": torch.float8_e8m0fnu}
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ------------------------------------------------------------------------------------------
# cases
# ------------------------------------------------------------------------------------------

def listed():
    return [
        # one block of activations (32 rows of d_model 4096): the smallest call, latency
        dict(name="quantize-block", kind="quantize", rows=32, d=4096, dtype="bf16", fmt="nv"),
        # the gate/up weights of a layer when a model is loaded, fp32 masters: bound by HBM
        dict(name="quantize-weights", kind="quantize", rows=24576, d=4096, dtype="f32", fmt="mx"),
        # QKV projection of a denoising step (one block of 32 rows): bound by the weight stream
        dict(name="matmul-block", kind="matmul", rows=32, n=12288, k=4096, out="bf16", fmt="nv"),
        # gate/up projection of the Dream widths at an odd number of rows (a ragged refresh step of a batch)
        dict(name="matmul-odd", kind="matmul", rows=997, n=37888, k=3584, out="f32", fmt="mx"),
        # the same kind of projection in a block entry over eight long prompts: bound by the tensor cores
        dict(name="matmul-entry", kind="matmul", rows=8192, n=24576, k=4096, out="bf16", fmt="nv"),
        # a denoising step of the benchmark's workload in one layer: 32 rows written, 32 rows attend over 512 positions
        dict(name="kv4-step", kind="kv4", op="step", heads="llada", batch=1, rows=32, cap=512, dtype="bf16"),
        # the fp32 model with 64-wide heads, an odd block in a ragged batch
        dict(name="kv4-step-f32", kind="kv4", op="step", heads="tiny", batch=3, rows=29, cap=1021, dtype="f32"),
        # single tokens over long ragged prompts, grouped heads: bound by the cache's bytes
        dict(name="kv4-token", kind="kv4", op="attend", heads="dream", batch=8, rows=1, cap=32768, dtype="bf16"),
        # window and block of a refresh step over the longest sequence the library takes
        dict(name="kv4-refresh-long", kind="kv4", op="attend", heads="dream", batch=1, rows=128, cap=65536, dtype="bf16"),
        # the rows of a block entry over long prompts go into the cache
        dict(name="kv4-append-entry", kind="kv4", op="append", heads="llada", batch=8, rows=1984, cap=2048, dtype="bf16"),
        # log-probabilities of one block, alternatives as a sampler or a client asks for them
        dict(name="logprobs-block", kind="logprobs", rows=32, vocab=126464, dtype="f32", top=8),
        # scoring of whole sequences, 16-bit logits
        dict(name="logprobs-score", kind="logprobs", rows=1024, vocab=152064, dtype="bf16", top=20),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["quantize", "matmul", "matmul", "kv4", "kv4", "kv4", "logprobs"])
    if kind == "quantize":
        d = 32 * _log_int(rng, 2, 592)
        return dict(kind=kind, rows=min(_log_int(rng, 1, 24576), 100663296 // d), d=d, dtype=rng.choice(["bf16", "f32"]), fmt=rng.choice(["nv", "mx"]))
    if kind == "matmul":
        k, n = 64 * _log_int(rng, 4, 192), _log_int(rng, 200, 37888)
        return dict(kind=kind, rows=min(_log_int(rng, 1, 8192), 824633720832 // (k * n)), n=n, k=k, out=rng.choice(["bf16", "bf16", "f32"]), fmt=rng.choice(["nv", "nv", "mx"]))
    if kind == "kv4":
        heads = rng.choice(["llada", "dream", "dream", "tiny"])
        nh, nkv, dh = HEADS[heads]
        batch, cap = rng.choice([1, 1, 2, 3, 5, 8]), _log_int(rng, 40, 65536)
        most = max(1, int(1.5e10 / (batch * cap * nh * dh)))                 # rows: no more products than the largest listed case ...
        cap = min(cap, 2 ** 29 // (batch * nkv * dh * 2))                     # ... and no larger a cache
        rows = rng.choice([1, _log_int(rng, 1, 256), _log_int(rng, 1, min(cap, 2048))])
        return dict(kind=kind, op=rng.choice(["step", "attend", "attend", "append"]), heads=heads, batch=batch, rows=max(1, min(rows, most, cap)), cap=cap,
                    dtype="f32" if heads == "tiny" else rng.choice(["bf16", "bf16", "bf16", "f32"]))
    return dict(kind=kind, rows=_log_int(rng, 1, 1024), vocab=_log_int(rng, 500, 152064), dtype=rng.choice(["bf16", "f32"]), top=rng.choice([0, 1, 2, 5, 8, 20, 32]))


# ------------------------------------------------------------------------------------------
# the formats in elementary operations
# ------------------------------------------------------------------------------------------

def _group(fmt):
    return 16 if fmt == "nv" else 32


def _code_of(y):
    """|x| / scale -> index on the grid: nearest value, ties to the even index."""
    return ((y > 0.25).to(torch.uint8) + (y >= 0.75) + (y > 1.25) + (y >= 1.75) + (y > 2.5) + (y >= 3.5) + (y > 5.0)).to(torch.uint8)


def _quantize(x, fmt, t):
    """x [..., d] fp32, t one fp32 on the GPU -> codes [..., d] (bit 3: sign), scale values [..., d / g] fp32."""
    g = x.unflatten(-1, (-1, _group(fmt)))
    a = g.abs().amax(-1)
    if fmt == "nv":
        s = torch.clamp(a / (t * 6.0), max=448.0).to(torch.float8_e4m3fn).float()
    else:
        e = torch.frexp(torch.where(torch.isfinite(a), a / t, torch.ones_like(a)))[1] - 3        # 2^(e + 2) <= a / t < 2^(e + 3)
        e = torch.where(a > 0, e, -127).clamp(-127, 127)
        s = torch.ldexp(torch.ones_like(a, dtype=torch.float64), e).float()
    s = torch.where(torch.isfinite(a), s, float("nan"))
    y = g.abs() / (s * t).unsqueeze(-1)
    c = torch.where((s > 0).unsqueeze(-1), _code_of(y) | ((g < 0).to(torch.uint8) << 3), 0)
    return c.flatten(-2), s


def _value(codes, scales, fmt, t):
    """codes [..., d] of four bits, scale values -> the values they stand for, fp32."""
    grid = torch.tensor(GRID, device=codes.device)
    v = grid[(codes & 7).long()]
    v = torch.where(codes >= 8, -v, v).unflatten(-1, (-1, _group(fmt))) * scales.unsqueeze(-1)
    return (v * t).flatten(-2)


def _pack(codes):
    return codes[..., 0::2] | (codes[..., 1::2] << 4)


def _unpack(b):
    return torch.stack((b & 15, b >> 4), -1).flatten(-2)


def _scale_bytes(s, fmt):
    if fmt == "nv":
        return s.to(torch.float8_e4m3fn).view(torch.uint8)
    return torch.where(torch.isnan(s), 255, torch.frexp(s)[1] + 126).to(torch.uint8)


def _scale_values(b, fmt):
    if fmt == "nv":
        return b.view(torch.float8_e4m3fn).float()
    s = torch.ldexp(torch.ones(b.shape, dtype=torch.float64, device=b.device), b.int() - 127).float()
    return torch.where(b == 255, float("nan"), s)


def _tile_scales(b):
    """Scale bytes [rows, groups] -> blocks of 128 rows x 4 groups: byte (r % 32) * 16 + (r % 128 / 32) * 4 + group % 4 of
    block (r / 128, group / 4), zeros where there is no row or group."""
    r, n = b.shape
    b = torch.nn.functional.pad(b, (0, -n % 4, 0, -r % 128))
    return b.view(-1, 4, 32, b.shape[1] // 4, 4).permute(0, 3, 2, 1, 4).contiguous()


# ------------------------------------------------------------------------------------------
# inputs
# ------------------------------------------------------------------------------------------

def _rows(gen, shape, spread, dtype):
    """Activations as models have them: channels of different size, a few large ones."""
    x = torch.randn(shape, generator=gen, device="cuda")
    x *= torch.exp(spread * torch.randn(shape[-1], generator=gen, device="cuda"))
    return x.to(dtype)


def _kv_lens(c, gen):
    """Keys of every sequence of a ragged batch: the first fills the cache, the others at least a quarter of it."""
    u = torch.rand(c["batch"], generator=gen, device="cuda")
    lens = (c["cap"] * (0.25 + 0.75 * u)).int().clamp(1, c["cap"])
    lens[0] = c["cap"]
    return torch.maximum(lens, torch.tensor(c["rows"] if c["op"] != "attend" else 1, device="cuda", dtype=torch.int32))


def prepare(case, seed):
    c = dict(case)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = {"c": c}
    if c["kind"] == "quantize":
        s["x"] = _rows(gen, (c["rows"], c["d"]), 0.5, DTYPES[c["dtype"]])
        s["t"] = torch.tensor([0.0123], device="cuda")
        s["codes"] = torch.empty((c["rows"], c["d"] // 2), dtype=torch.uint8, device="cuda")
        s["scales"] = torch.empty((c["rows"], c["d"] // _group(c["fmt"])), dtype=torch.uint8, device="cuda")
        s["deq"] = torch.empty_like(s["x"])
    elif c["kind"] == "matmul":
        fmt, m, n, k = c["fmt"], c["rows"], c["n"], c["k"]
        s["x"] = _rows(gen, (m, k), 0.3, torch.bfloat16)
        s["tx"], s["tw"] = torch.tensor([0.0123], device="cuda"), torch.tensor([0.00021], device="cuda")
        s["wc"] = torch.empty((n, k // 2), dtype=torch.uint8, device="cuda")
        sb = torch.empty((n, k // _group(fmt)), dtype=torch.uint8, device="cuda")
        for r in range(0, n, 8192):                      # weights of a trained model's size, quantised when it was loaded
            w = torch.randn((min(8192, n - r), k), generator=gen, device="cuda") * 0.02
            codes, sv = _quantize(w, fmt, s["tw"])
            s["wc"][r:r + 8192], sb[r:r + 8192] = _pack(codes), _scale_bytes(sv, fmt)
        s["ws"], s["wsb"] = _tile_scales(sb), sb
        s["xc"] = torch.empty((m, k // 2), dtype=torch.uint8, device="cuda")
        s["xs"] = torch.empty((-(-m // 128), -(-(k // _group(fmt)) // 4), 32, 4, 4), dtype=torch.uint8, device="cuda")
        s["out"] = torch.empty((m, n), dtype=DTYPES[c["out"]], device="cuda")
    elif c["kind"] == "kv4":
        nh, nkv, dh = HEADS[c["heads"]]
        b, r, cap, dt = c["batch"], c["rows"], c["cap"], DTYPES[c["dtype"]]
        s["tk"], s["tv"] = torch.tensor([0.0173], device="cuda"), torch.tensor([0.0031], device="cuda")
        s["lens"] = _kv_lens(c, gen)
        for name, spread, t in (("k", 0.6, s["tk"]), ("v", 0.2, s["tv"])):
            codes = torch.empty((b, cap, nkv, dh // 2), dtype=torch.uint8, device="cuda")
            scales = torch.empty((b, cap, nkv, dh // 16), dtype=torch.uint8, device="cuda")
            for i in range(b):
                for p in range(0, cap, 8192):
                    n = min(8192, cap - p)
                    x = _rows(gen, (n, nkv, dh), spread, torch.bfloat16).float()
                    q, sv = _quantize(x, "nv", t)
                    codes[i, p:p + n], scales[i, p:p + n] = _pack(q), _scale_bytes(sv, "nv")
            s[name + "c"], s[name + "s"] = codes, scales
        if c["op"] != "attend":
            s["k"], s["v"] = _rows(gen, (b, r, nkv * dh), 0.6, dt), _rows(gen, (b, r, nkv * dh), 0.2, dt)
            # positions in a sequence, ascending, as a selection of stale rows leaves them; the last sequences list fewer
            idx = torch.full((b, r), -1, dtype=torch.int32, device="cuda")
            counts = torch.full((b,), r, dtype=torch.int32, device="cuda")
            for i in range(b):
                n = r if i == 0 else max(1, r - i)
                counts[i] = n
                idx[i, :n] = torch.sort(torch.randperm(cap, generator=gen, device="cuda")[:n])[0].int()
            s["idx"], s["counts"] = idx, counts
            s["kd"], s["vd"] = torch.zeros_like(s["k"]), torch.zeros_like(s["v"])
        if c["op"] != "append":
            s["q"] = _rows(gen, (b, r, nh * dh), 0.3, dt)
            s["out"] = torch.empty_like(s["q"])
            s["lse"] = torch.empty((b, r, nh), device="cuda")
    else:
        r, v = c["rows"], c["vocab"]
        x = 2.0 * torch.randn((r, v), generator=gen, device="cuda")
        hot = torch.randint(0, v, (r, 4), generator=gen, device="cuda")          # rows from undecided to nearly certain
        x.scatter_add_(1, hot, 14.0 * torch.rand((r, 4), generator=gen, device="cuda"))
        x[:, 1::97] = float("-inf")                                              # tokens that the sampler has ruled out
        s["x"] = x.to(DTYPES[c["dtype"]])
        target = torch.where(torch.rand(r, generator=gen, device="cuda") < 0.5, hot[:, 0], torch.randint(0, v, (r,), generator=gen, device="cuda"))
        s["target"] = torch.where(target % 97 == 1, target - 1, target).int()
        s["lp"], s["h"] = torch.empty(r, device="cuda"), torch.empty(r, device="cuda")
        s["ids"] = torch.empty((r, c["top"]), dtype=torch.int32, device="cuda")
        s["tops"] = torch.empty((r, c["top"]), device="cuda")
    return s


# ------------------------------------------------------------------------------------------
# one pass
# ------------------------------------------------------------------------------------------

def _attend(q, k, v, lens):
    """q [b, r, n_heads, dh], k / v [b, cap, n_kv, dh] in one floating type; keys behind a sequence's length take no part."""
    b, r, nh, dh = q.shape
    cap, nkv = k.shape[1], k.shape[2]
    qg = q.view(b, r, nkv, nh // nkv, dh).permute(0, 2, 3, 1, 4).reshape(b, nkv, -1, dh)
    sc = qg @ k.permute(0, 2, 3, 1) / math.sqrt(dh)
    gone = torch.arange(cap, device=q.device)[None, :] >= lens[:, None]
    sc = sc.masked_fill_(gone[:, None, None, :], float("-inf"))
    m = sc.amax(-1, keepdim=True)
    p = torch.exp_(sc.sub_(m))
    total = p.sum(-1, keepdim=True)
    back = lambda x: x.view(b, nkv, nh // nkv, r, -1).permute(0, 3, 1, 2, 4).reshape(b, r, nh, -1)  # noqa: E731
    return back(p @ v.permute(0, 2, 1, 3) / total), back(m + torch.log(total)).squeeze(-1)


def _write(s, name, t):
    """The new rows of one of the caches, in place; returns the values stored, zeros where a sequence lists fewer rows."""
    x, idx, codes, scales = s[name], s["idx"].long(), s[name + "c"], s[name + "s"]
    b, r, _ = x.shape
    live = torch.arange(r, device="cuda")[None, :] < s["counts"][:, None]
    q, sv = _quantize(x.float().view(b, r, *codes.shape[2:3], -1), "nv", t)
    at, seq = idx[live], torch.arange(b, device="cuda")[:, None].expand(b, r)[live]
    codes[seq, at], scales[seq, at] = _pack(q)[live], _scale_bytes(sv, "nv")[live]
    return torch.where(live[:, :, None], _value(q, sv, "nv", t).flatten(2), 0.0).to(x.dtype)


def _plain(s):
    c = s["c"]
    if c["kind"] == "quantize":
        codes, sv = _quantize(s["x"].float(), c["fmt"], s["t"])
        return {"values": _value(codes, sv, c["fmt"], s["t"]).to(s["x"].dtype), "scales": sv.to(SCALE_TYPES[c["fmt"]])}
    if c["kind"] == "matmul":
        x = _value(*_quantize(s["x"].float(), c["fmt"], s["tx"]), c["fmt"], s["tx"])
        w = _value(_unpack(s["wc"]), _scale_values(s["wsb"], c["fmt"]), c["fmt"], s["tw"])
        return {"out": (x @ w.t()).to(s["out"].dtype)}
    if c["kind"] == "kv4":
        got = {}
        if c["op"] != "attend":
            got["k"], got["v"] = _write(s, "k", s["tk"]), _write(s, "v", s["tv"])
        if c["op"] != "append":
            k = _value(_unpack(s["kc"]), _scale_values(s["ks"], "nv"), "nv", s["tk"])
            v = _value(_unpack(s["vc"]), _scale_values(s["vs"], "nv"), "nv", s["tv"])
            q = s["q"].float().view(*s["q"].shape[:2], -1, k.shape[-1])
            out, got["lse"] = _attend(q, k, v, s["lens"])
            got["out"] = out.flatten(2).to(s["q"].dtype)
        return got
    x = s["x"].double()                                    # long sums, and entropies next to zero
    m = x.amax(-1, keepdim=True)
    z = x - m
    e = torch.exp(z)
    total = e.sum(-1, keepdim=True)
    lse = m + torch.log(total)
    h = torch.log(total) - torch.where(e > 0, e * z, 0.0).sum(-1, keepdim=True) / total
    lp = x.gather(1, s["target"].long()[:, None]) - lse
    # (the mask token, the last of the vocabulary, is no alternative)
    tops, ids = torch.sort(s["x"].float().masked_fill(torch.arange(c["vocab"], device="cuda") == c["vocab"] - 1, float("-inf")), dim=-1, descending=True, stable=True)
    ids, tops = ids[:, :c["top"]].int(), tops[:, :c["top"]].double() - lse
    return {"logprob": lp[:, 0].float(), "entropy": h[:, 0].float(), "ids": ids, "tops": tops.float()}


def run(s):
    if not own:
        return _plain(s)
    from paper_2607_14107_b200 import binding as Bd
    c = s["c"]
    if c["kind"] == "quantize":
        fmt = Bd.FP4_NV if c["fmt"] == "nv" else Bd.FP4_MX
        Bd.polestar_k_fp4_quantize(s["x"], s["codes"], s["scales"], fmt, Bd.SCALES_ROWS, tensor_scale=s["t"], deq=s["deq"])
        return {"values": s["deq"], "scales": s["scales"].view(SCALE_TYPES[c["fmt"]])}
    if c["kind"] == "matmul":
        fmt = Bd.FP4_NV if c["fmt"] == "nv" else Bd.FP4_MX
        Bd.polestar_k_fp4_quantize(s["x"], s["xc"], s["xs"], fmt, Bd.SCALES_TILED, tensor_scale=s["tx"])
        Bd.polestar_k_fp4_matmul(s["xc"], s["xs"], s["wc"], s["ws"], s["out"], fmt, a_tensor_scale=s["tx"], b_tensor_scale=s["tw"])
        return {"out": s["out"]}
    if c["kind"] == "kv4":
        got = {}
        if c["op"] != "attend":
            Bd.polestar_k_kv4_append(s["k"], s["v"], s["idx"], s["counts"], s["kc"], s["ks"], s["vc"], s["vs"], s["tk"], s["tv"], k_deq=s["kd"], v_deq=s["vd"])
            got["k"], got["v"] = s["kd"], s["vd"]
        if c["op"] != "append":
            if "scratch" not in s:                         # a program keeps one for all its calls
                n = Bd.polestar_k_kv4_scratch_bytes(*s["q"].shape[:2], s["kc"].shape[1], s["lse"].shape[2], s["kc"].shape[2], 2 * s["kc"].shape[3])
                s["scratch"] = torch.empty(n, dtype=torch.uint8, device="cuda")
            Bd.polestar_k_kv4_attention(s["q"], s["kc"], s["ks"], s["vc"], s["vs"], s["tk"], s["tv"], s["lens"], s["out"], s["lse"], s["scratch"])
            got["lse"], got["out"] = s["lse"], s["out"]
        return got
    Bd.polestar_k_token_logprobs(s["x"], s["target"], c["vocab"] - 1, s["lp"], s["h"], s["ids"], s["tops"])
    return {"logprob": s["lp"], "entropy": s["h"], "ids": s["ids"], "tops": s["tops"]}


# ------------------------------------------------------------------------------------------
# the definition in 64 bits
# ------------------------------------------------------------------------------------------

def _exact_quantize(x, fmt, t):
    """The values that x [..., d] (64 bits) is stored as, and the scales: nearest values found by distance."""
    g = x.unflatten(-1, (-1, 16 if fmt == "nv" else 32))
    top = g.abs().amax(-1)
    if fmt == "nv":
        want = torch.clamp(top / 6 / t, max=448.0)
        step = torch.exp2(torch.clamp(torch.floor(torch.log2(want.clamp(min=1e-300))), min=-6.0) - 3)      # three bits behind the first
        s = torch.round(want / step) * step
    else:
        s = torch.exp2(torch.clamp(torch.floor(torch.log2((top / t).clamp(min=1e-300))) - 2, -127, 127))
    grid = torch.tensor(GRID, dtype=torch.float64, device=x.device)
    unit = (s * t).unsqueeze(-1)
    y = torch.where(unit > 0, g.abs() / unit, torch.zeros_like(g)).clamp(max=6.0)
    middle = (grid[1:] + grid[:-1]) / 2
    low = torch.bucketize(y, middle)                       # number of middles below y: a tie stays at the lower value ...
    tie = (low < 7) & (y == middle[low.clamp(max=6)]) & (low % 2 == 1)
    near = grid[low + tie.long()]                          # ... or goes to the upper one, whichever code is even
    return (torch.sign(g) * near * unit).flatten(-2), s


def _exact_rows(x, fmt, t, at_once=4096):
    return torch.cat([_exact_quantize(x[i:i + at_once].double(), fmt, t)[0] for i in range(0, x.shape[0], at_once)])


def _exact_stored(codes, scales, t):
    """Values of a 4-bit matrix as stored: low nibble first."""
    c = torch.stack((codes % 16, codes // 16), -1).flatten(-2)
    v = torch.tensor(GRID + tuple(-g for g in GRID), dtype=torch.float64, device=codes.device)[c.long()]
    return (v.unflatten(-1, (scales.shape[-1], -1)) * scales.double().unsqueeze(-1)).flatten(-2) * t


def exact(case, seed):
    c, s = dict(case), prepare(case, seed)
    if c["kind"] == "quantize":
        v, sc = _exact_quantize(s["x"].double(), c["fmt"], s["t"].double())
        return {"values": v, "scales": sc}
    if c["kind"] == "matmul":
        x = _exact_rows(s["x"], c["fmt"], s["tx"].double())
        out = torch.empty((c["rows"], c["n"]), dtype=torch.float64, device="cuda")
        for r in range(0, c["n"], 4096):
            w = _exact_stored(s["wc"][r:r + 4096], _scale_values(s["wsb"][r:r + 4096], c["fmt"]), s["tw"].double())
            out[:, r:r + 4096] = x @ w.t()
        return {"out": out}
    if c["kind"] == "kv4":
        got, nh = {}, HEADS[c["heads"]][0]
        nkv, dh = HEADS[c["heads"]][1:]
        tk, tv = s["tk"].double(), s["tv"].double()
        new = {}
        if c["op"] != "attend":
            live = torch.arange(c["rows"], device="cuda")[None, :] < s["counts"][:, None]
            for name, t in (("k", tk), ("v", tv)):
                new[name] = torch.stack([_exact_quantize(x.double(), "nv", t)[0] for x in s[name]])
                got[name] = torch.where(live[:, :, None], new[name], 0.0)
        if c["op"] != "append":
            out = torch.zeros((c["batch"], c["rows"], nh, dh), dtype=torch.float64, device="cuda")
            lse = torch.zeros((c["batch"], c["rows"], nh), dtype=torch.float64, device="cuda")
            for i in range(c["batch"]):
                n = int(s["lens"][i])
                for h in range(nkv):
                    at = {}
                    for name, t in (("k", tk), ("v", tv)):
                        x = _exact_stored(s[name + "c"][i, :, h], s[name + "s"][i, :, h].view(torch.float8_e4m3fn).float(), t)
                        if new:
                            m = int(s["counts"][i])
                            x[s["idx"][i, :m].long()] = new[name][i, :m, h * dh:(h + 1) * dh]
                        at[name] = x[:n]
                    for hq in range(h * (nh // nkv), (h + 1) * (nh // nkv)):
                        sc = s["q"][i, :, hq * dh:(hq + 1) * dh].double() @ at["k"].t() / math.sqrt(dh)
                        lse[i, :, hq] = torch.logsumexp(sc, -1)
                        out[i, :, hq] = torch.softmax(sc, -1) @ at["v"]
            got["lse"], got["out"] = lse, out.flatten(2)
        return got
    x = s["x"].double()
    lp = torch.log_softmax(x, -1)
    h = -torch.where(lp > -math.inf, lp.exp() * lp, torch.zeros_like(lp)).sum(-1)
    rows = torch.arange(c["rows"], device="cuda")
    lp_t = lp[rows, s["target"].long()]
    lp[:, -1] = -math.inf
    return {"logprob": lp_t, "entropy": h, "ids": None, "tops": torch.topk(lp, c["top"], dim=-1).values}


# ------------------------------------------------------------------------------------------
# what a pass cannot do without
# ------------------------------------------------------------------------------------------

def work(case):
    c = dict(case)
    size = {"bf16": 2, "f32": 4}
    if c["kind"] == "quantize":
        n = c["rows"] * c["d"]
        return {"bytes": n * (2 * size[c["dtype"]] + 0.5 + 1 / _group(c["fmt"])), "flops": 4 * n}
    if c["kind"] == "matmul":
        m, n, k = c["rows"], c["n"], c["k"]
        return {"bytes": m * k * 2 + n * k * (0.5 + 1 / _group(c["fmt"])) + m * n * size[c["out"]], "flops": 2 * m * n * k}
    if c["kind"] == "kv4":
        nh, nkv, dh = HEADS[c["heads"]]
        b, r, es = c["batch"], c["rows"], size[c["dtype"]]
        keys = c["cap"] + (b - 1) * c["cap"] * 0.625                          # on average
        got = {"bytes": 0, "flops": 0}
        if c["op"] != "attend":
            got["bytes"] += 2 * b * r * nkv * dh * (2 * es + 0.5625)
        if c["op"] != "append":
            got["bytes"] += 2 * keys * nkv * dh * 0.5625 + 2 * b * r * nh * dh * es
            got["flops"] += 4 * keys * r * nh * dh
        return got
    n = c["rows"] * c["vocab"]
    return {"bytes": n * size[c["dtype"]] + c["rows"] * (12 + 8 * c["top"]), "flops": 6 * n}
