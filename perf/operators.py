"""Performance cases of the operators for quantized language models: microscaled 4-bit tensors (the (4, 1) type in
blocks of 32 values with a power-of-two scale each), products of them, root-mean-square norms that end in 8 or 4 bits,
and quantized caches.

Four kinds of work:

  codec   a tensor to 4-bit codes and scales and back to values: `qmx_quantize`, `qmx_dequantize`
  linear  activations times weights, both in microscaled 4 bits: `QMXLinear.run` on a handle that is kept
  norm    residual addition, root-mean-square norm, output in 8 bits or in microscaled 4 bits: `qrmsnorm`
  cache   new keys and values quantized into their slots, the sequences' keys and values read back: `QCache`

`own` says which side `run` takes: the library's calls, or the same in elementary torch operations.  Inputs are made
from the seed alone; sizes are generic.
"""
import math

import torch

own = False

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_BLOCK = 32
_VALUES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)            # magnitudes of the 4-bit type


def _codec(name, rows, K, dtype, layout, rule):
    case = dict(kind="codec", rows=rows, K=K, dtype=dtype, layout=layout, rule=rule)
    return dict(case, name=name) if name else case


def _linear(name, M, N, K, dtype, bias=False, relu=False):
    case = dict(kind="linear", M=M, N=N, K=K, dtype=dtype, bias=bias, relu=relu)
    return dict(case, name=name) if name else case


def _norm(name, rows, C, dtype, residual, out):
    case = dict(kind="norm", rows=rows, C=C, dtype=dtype, residual=residual, out=out)
    return dict(case, name=name) if name else case


def _cache(name, fmt, seqs, new, length, heads, D, dtype):
    case = dict(kind="cache", fmt=fmt, seqs=seqs, new=new, length=length, heads=heads, D=D, dtype=dtype)
    return dict(case, name=name) if name else case


def listed():
    return [
        # the activations of sixteen sequences that decode together, on their way into a product
        _codec("codec 16 rows", 16, 4096, "bf16", "tiles", "cover"),
        # a weight matrix of odd width, converted once and read back to see what the conversion did to it
        _codec("codec weights", 8192, 5000, "f32", "rows", "floor"),
        # one token against one weight matrix: a decoding step of a single sequence
        _linear("linear one token", 1, 4096, 4096, "bf16"),
        # a decoding step of a batch against a wide layer: bound by the weights' bytes
        _linear("linear 48 tokens", 48, 16384, 8192, "f16", bias=True),
        # a short ragged prompt, no size a multiple of a tile, output kept in 32 bits
        _linear("linear ragged", 1000, 5000, 2000, "f32", bias=True, relu=True),
        # a long prompt: bound by the tensor cores
        _linear("linear prompt", 8192, 8192, 8192, "bf16"),
        # the norm before an int8 layer with a calibrated scale, one token
        _norm("norm one token", 1, 4096, "bf16", True, "i8"),
        # rows of odd length with a scale for each
        _norm("norm odd rows", 3000, 1155, "f32", True, "i8_rows"),
        # a long prompt's norm into 4 bits
        _norm("norm prompt", 16384, 8192, "bf16", True, "mx"),
        # one decoding step of eight short sequences
        _cache("cache step", "i8", 8, 1, 1024, 8, 128, "bf16"),
        # a prompt written into a 4-bit cache and read back, heads of an odd size
        _cache("cache prompt", "mx", 2, 1500, 2000, 8, 80, "f16"),
        # one decoding step of many long sequences
        _cache("cache long", "i8", 32, 1, 8192, 8, 128, "bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    dtype = rng.choice(["f32", "bf16", "f16"])
    kind = rng.choice(["codec", "linear", "linear", "norm", "cache"])
    if kind == "codec":
        rows, K = _log(rng, 1, 8192), _log(rng, 32, 8192)
        return _codec(None, rows, min(K, max(32, 40_000_000 // rows)), dtype, rng.choice(["tiles", "rows"]), rng.choice(["cover", "floor"]))
    if kind == "linear":
        M, N, K = _log(rng, 1, 8192), _log(rng, 64, 16384), _log(rng, 64, 8192)
        if rng.random() < 0.5:                             # layers are mostly multiples of 64 wide
            N, K = max(64, N // 64 * 64), max(64, K // 64 * 64)
        return _linear(None, min(M, max(1, 8192 * 8192 // N)), N, K, dtype, rng.random() < 0.5, rng.random() < 0.3)
    if kind == "norm":
        rows, C = _log(rng, 1, 16384), _log(rng, 16, 8192)
        if rng.random() < 0.5:
            C = max(16, C // 16 * 16)
        return _norm(None, rows, C, dtype, rng.random() < 0.6, rng.choice(["i8", "i8_rows", "mx"]))
    seqs, length = _log(rng, 1, 32), _log(rng, 1, 8192)
    heads, D = rng.choice([1, 2, 4, 8]), rng.choice([64, 80, 96, 112, 128])
    return _cache(None, rng.choice(["i8", "mx"]), seqs, rng.randint(1, length) if rng.random() < 0.3 else 1, length, heads, D, dtype)


# ------------------------------------------------------------------------------------------------ plain forms
def _power(e):
    """2^e for whole e in [-126, 127], from its bit pattern."""
    return ((e + 127) << 23).to(torch.int32).view(torch.float32)


def _largest(x):
    """The largest finite magnitude along the last axis."""
    a = x.abs()
    return torch.where(torch.isfinite(a), a, torch.zeros((), device=x.device)).amax(-1)


def _plain_blocks(x):
    """[..., K] -> [..., blocks, 32] in 32 bits, the last block filled up with zeros."""
    K = x.shape[-1]
    return torch.nn.functional.pad(x.float(), (0, -K % _BLOCK)).unflatten(-1, (-1, _BLOCK))


def _plain_mx_encode(x, rule):
    """[..., K] -> codes [..., blocks * 16], two to a byte, and scale bytes [..., blocks]."""
    x = _plain_blocks(x)
    top = _largest(x)
    bits = top.view(torch.int32)
    s = ((bits + (0x3FFFFF if rule == "cover" else 0)) >> 23) - 2      # 6 * 2^e covers the block, or 4 * 2^e is in its binade
    s = torch.where(top > 0, s.clamp(min=0), 127)
    a = x.abs() * _power(127 - s).unsqueeze(-1)
    code = (a > 0.25).byte() + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5)
    code = code | (((x < 0) & (code > 0)).byte() << 3)
    return (code[..., 0::2] | (code[..., 1::2] << 4)).flatten(-2), s.byte()


def _plain_mx_decode(codes, scales, K):
    """Codes [..., blocks * 16] and scales [..., blocks] -> values [..., K] in 32 bits."""
    values = torch.tensor(_VALUES + tuple(-v for v in _VALUES), device=codes.device)
    code = torch.stack((codes & 15, codes >> 4), -1).flatten(-2)
    half = scales.int() >> 1                                 # 2^(s - 127) in two factors: it may be below the smallest normal number
    y = values[code.long()].unflatten(-1, (-1, _BLOCK)) * _power(half - 63).unsqueeze(-1) * _power(scales.int() - half - 64).unsqueeze(-1)
    return y.flatten(-2)[..., :K]


def _to_tiles(s):
    """Scales [rows, blocks] -> the order of the tensor cores: 128 rows x 4 blocks a tile, padding bytes 127."""
    rows, blocks = s.shape
    s = torch.nn.functional.pad(s, (0, -blocks % 4, 0, -rows % 128), value=127)
    s = s.view(s.shape[0] // 128, 4, 32, s.shape[1] // 4, 4)
    return s.permute(0, 3, 2, 1, 4).reshape(-1)


def _from_tiles(t, rows, blocks):
    t = t.view(-(-rows // 128), -(-blocks // 4), 32, 4, 4).permute(0, 3, 2, 1, 4)
    return t.reshape(t.shape[0] * 128, -1)[:rows, :blocks]


def _plain_i8(y):
    """Rows -> int8 and a scale byte for each: the smallest e with 127 * 2^e >= the row's largest magnitude."""
    top = _largest(y)
    s = torch.where(top > 0, (((top.view(torch.int32) + 0x1FFFF) >> 23) - 6).clamp(min=1), 127)
    return _plain_round(y * _power(127 - s).unsqueeze(-1)), s.byte()


def _plain_round(y):
    return torch.nan_to_num(y.round(), nan=0.0).clamp(-127, 127).to(torch.int8)


def _plain_codec(st):
    codes, scales = _plain_mx_encode(st["x"], st["rule"])
    values = _plain_mx_decode(codes, scales, st["x"].shape[1]).to(st["x"].dtype)
    return dict(codes=codes, scales=_to_tiles(scales) if st["layout"] == "tiles" else scales, values=values)


def _plain_linear(st):
    K, blocks = st["K"], -(-st["K"] // _BLOCK)
    x = _plain_mx_decode(st["x_codes"], _from_tiles(st["x_scales"], st["M"], blocks), K)
    w = _plain_mx_decode(st["w_codes"], _from_tiles(st["w_scales"], st["N"], blocks), K)
    y = x @ w.T
    if st["bias"] is not None:
        y = y + st["bias"]
    return (y.relu() if st["relu"] else y).to(st["y"].dtype)


def _plain_norm(st):
    x, out = st["x"], {}
    if st["residual"] is not None:
        x = out["sum"] = (x.float() + st["residual"].float()).to(x.dtype)
    r = (1.0 / torch.sqrt(x.double().square().mean(-1) + _EPS)).float()      # long sums
    y = x.float() * r[:, None] * st["gain"].float()
    if st["out"] == "i8":
        return dict(out, codes=_plain_round(y * 2.0**-st["e"]))
    if st["out"] == "i8_rows":
        codes, scales = _plain_i8(y)
        return dict(out, codes=codes, scales=scales)
    codes, scales = _plain_mx_encode(y, "cover")
    return dict(out, values=_plain_mx_decode(codes, scales, y.shape[1]).to(x.dtype))


def _plain_cache(st):
    out = {}
    for name in ("k", "v"):
        codes, scales = st[name + "_codes"], st[name + "_scales"]
        kept = st["new_slots"] >= 0
        new = st[name][kept].float()
        c, s = _plain_i8(new) if st["fmt"] == "i8" else _plain_mx_encode(new, "cover")
        codes[st["new_slots"][kept]] = c.view(torch.uint8)
        scales[st["new_slots"][kept]] = s.unsqueeze(-1) if st["fmt"] == "i8" else s
        c, s = codes[st["slots"]], scales[st["slots"]]
        y = c.view(torch.int8).float() * _power(s.int() - 127) if st["fmt"] == "i8" else _plain_mx_decode(c, s, st["D"])
        out.update({name: y.to(st[name].dtype), name + "_codes": codes, name + "_scales": scales})
    return out


# ------------------------------------------------------------------------------------------------ inputs
_EPS = 1e-6
_NORM_E = -4                                               # calibrated exponent of a norm's int8 output


def _activations(gen, shape, dtype):
    """Normal values, some channels of them far larger, as activations of language models have them."""
    x = torch.randn(shape, generator=gen, device="cuda")
    loud = torch.rand(shape[-1:], generator=gen, device="cuda") < 0.01
    return (x * torch.where(loud, 20.0, 1.0)).to(dtype)


def _lengths(case):
    """Lengths of the sequences, the same for every seed: the first has the whole length, the others less."""
    return [case["length"]] + [1 + (case["length"] * (7 * i % 16)) // 16 for i in range(1, case["seqs"])]


def _prepare_codec(case, gen):
    x = _activations(gen, (case["rows"], case["K"]), _TYPES[case["dtype"]])
    blocks = -(-case["K"] // _BLOCK)
    scales = (-(-case["rows"] // 128) * -(-blocks // 4) * 512,) if case["layout"] == "tiles" else (case["rows"], blocks)
    return dict(case, x=x, codes=torch.empty((case["rows"], blocks * 16), dtype=torch.uint8, device="cuda"),
                scales=torch.empty(scales, dtype=torch.uint8, device="cuda"), values=torch.empty_like(x))


def _prepare_linear(case, gen):
    M, N, K = case["M"], case["N"], case["K"]
    st = dict(case, y=torch.empty((M, N), dtype=_TYPES[case["dtype"]], device="cuda"))
    for name, t in (("x", _activations(gen, (M, K), torch.float32)), ("w", torch.randn((N, K), generator=gen, device="cuda") * K**-0.5)):
        codes, scales = _plain_mx_encode(t, "cover")
        st[name + "_codes"], st[name + "_scales"] = codes, _to_tiles(scales)
    st["bias"] = torch.randn((N,), generator=gen, device="cuda") if case["bias"] else None
    if own:                                                # the handle that a program keeps beside its weights
        from paper_1805_07941_b200 import binding
        st["linear"] = binding.QMXLinear(st["w_codes"], st["w_scales"], N=N, K=K, bias=st["bias"], relu=int(case["relu"]),
                                         dtype=st["y"].dtype)
    return st


def _prepare_norm(case, gen):
    rows, C, dtype = case["rows"], case["C"], _TYPES[case["dtype"]]
    x = _activations(gen, (rows, C), dtype)
    blocks = -(-C // _BLOCK)
    if case["out"] == "mx":
        codes, scales = (rows, blocks * 16), (-(-rows // 128) * -(-blocks // 4) * 512,)
    else:
        codes, scales = (rows, C), (rows,)
    return dict(case, x=x, residual=_activations(gen, (rows, C), dtype) if case["residual"] else None, e=_NORM_E,
                gain=(1 + 0.2 * torch.randn((C,), generator=gen, device="cuda")).to(dtype), sum=torch.empty_like(x),
                codes=torch.empty(codes, dtype=torch.uint8 if case["out"] == "mx" else torch.int8, device="cuda"),
                scales=torch.empty(scales, dtype=torch.uint8, device="cuda"),
                values=torch.empty_like(x) if case["out"] == "mx" else None)


def _prepare_cache(case, gen):
    heads, D, dtype, page = case["heads"], case["D"], _TYPES[case["dtype"]], 16
    lengths = _lengths(case)
    pages = [-(-n // page) for n in lengths]
    total = sum(pages) + 4
    order = torch.randperm(total, generator=gen, device="cuda")
    first = 0
    slots, new = [], []
    for n, p in zip(lengths, pages):
        at = torch.arange(n, device="cuda")
        s = order[first + at // page] * page + at % page
        first += p
        slots.append(s)
        fresh = s[-min(case["new"], n):]
        new.append(torch.nn.functional.pad(fresh, (0, case["new"] - fresh.numel()), value=-1))     # a padded batch
    st = dict(case, slots=torch.cat(slots), new_slots=torch.cat(new))
    blocks = -(-D // _BLOCK)
    for name in ("k", "v"):
        st[name] = _activations(gen, (st["new_slots"].numel(), heads, D), dtype)
        if case["fmt"] == "i8":
            codes = torch.randint(-127, 128, (total * page, heads, D), generator=gen, device="cuda", dtype=torch.int8).view(torch.uint8)
            scales = torch.randint(118, 124, (total * page, heads, 1), generator=gen, device="cuda", dtype=torch.uint8)
        else:
            old = torch.randint(1, 8, (total * page, heads, blocks * 16), generator=gen, device="cuda", dtype=torch.uint8)
            codes = old * 17
            scales = torch.randint(124, 128, (total * page, heads, blocks), generator=gen, device="cuda", dtype=torch.uint8)
        st[name + "_codes"], st[name + "_scales"] = codes, scales
        st[name + "_out"] = torch.empty((st["slots"].numel(), heads, D), dtype=dtype, device="cuda")
    if own:                                                # the object that a program keeps beside its cache
        from paper_1805_07941_b200 import binding
        st["cache"] = binding.QCache(st["k_codes"], st["k_scales"], st["v_codes"], st["v_scales"], D=D,
                                     fmt=binding.CACHE_I8 if case["fmt"] == "i8" else binding.CACHE_MX)
    return st


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    return {"codec": _prepare_codec, "linear": _prepare_linear, "norm": _prepare_norm, "cache": _prepare_cache}[case["kind"]](case, gen)


# ------------------------------------------------------------------------------------------------ running
def _own_codec(st):
    from paper_1805_07941_b200 import binding
    rule = binding.MX_COVER if st["rule"] == "cover" else binding.MX_FLOOR
    layout = binding.MX_TILES if st["layout"] == "tiles" else binding.MX_ROWS
    binding.qmx_quantize(st["x"], rule=rule, layout=layout, codes=st["codes"], scales=st["scales"])
    binding.qmx_dequantize(st["codes"], st["scales"], st["K"], layout=layout, out=st["values"])
    return dict(codes=st["codes"], scales=st["scales"], values=st["values"])


def _own_norm(st):
    from paper_1805_07941_b200 import binding
    out = dict(sum=st["sum"]) if st["residual"] is not None else {}
    kw = dict(residual=st["residual"], sum_out=st["sum"] if out else None, codes=st["codes"])
    if st["out"] == "i8":
        binding.qrmsnorm(st["x"], st["gain"], _EPS, out=binding.NORM_I8, e=st["e"], **kw)
        return dict(out, codes=st["codes"])
    if st["out"] == "i8_rows":
        binding.qrmsnorm(st["x"], st["gain"], _EPS, out=binding.NORM_I8_ROWS, scales=st["scales"], **kw)
        return dict(out, codes=st["codes"], scales=st["scales"])
    binding.qrmsnorm(st["x"], st["gain"], _EPS, out=binding.NORM_MX, scales=st["scales"], **kw)
    binding.qmx_dequantize(st["codes"], st["scales"], st["C"], out=st["values"])
    return dict(out, values=st["values"])


def _own_cache(st):
    cache = st["cache"]
    cache.write(st["new_slots"], st["k"], st["v"])
    cache.read(st["slots"], st["k_out"], st["v_out"])
    return dict(k=st["k_out"], k_codes=st["k_codes"], k_scales=st["k_scales"], v=st["v_out"], v_codes=st["v_codes"], v_scales=st["v_scales"])


def run(state):
    kind = state["kind"]
    if own:
        if kind == "linear":
            return state["linear"].run(state["x_codes"], state["x_scales"], state["y"])
        return {"codec": _own_codec, "norm": _own_norm, "cache": _own_cache}[kind](state)
    return {"codec": _plain_codec, "linear": _plain_linear, "norm": _plain_norm, "cache": _plain_cache}[kind](state)


# ------------------------------------------------------------------------------------------------ definition in 64 bits
def _exact_power_scale(top, largest):
    """The smallest whole e with largest * 2^e >= top (0 where top is 0), as 2^e in 64 bits."""
    m, e = torch.frexp(top / largest)                      # top / largest = m 2^e, m in [0.5, 1)
    e = torch.where(m == 0.5, e - 1, e)
    return torch.where(top > 0, torch.ldexp(torch.ones_like(top), e), torch.ones_like(top))


def _exact_nearest(a):
    """Magnitudes -> the nearest of the type's values, ties to the even place."""
    grid = torch.tensor(_VALUES, dtype=torch.float64, device=a.device)
    hi = torch.searchsorted(grid, a.clamp(max=6.0).contiguous()).clamp(1, 7)
    lo = hi - 1
    a = a.clamp(max=6.0)
    up, down = grid[hi] - a, a - grid[lo]
    return torch.where((up < down) | ((up == down) & (hi % 2 == 0)), grid[hi], grid[lo])


def _exact_mx(x, rule="cover"):
    K = x.shape[-1]
    b = torch.nn.functional.pad(x.double(), (0, -K % _BLOCK)).unflatten(-1, (-1, _BLOCK))
    top = b.abs().amax(-1)
    if rule == "cover":
        scale = _exact_power_scale(top, 6.0)
    else:
        scale = torch.where(top > 0, torch.ldexp(torch.ones_like(top), torch.frexp(top)[1] - 3), torch.ones_like(top))
    y = _exact_nearest(b.abs() / scale.unsqueeze(-1)) * scale.unsqueeze(-1) * b.sign()
    return y.flatten(-2)[..., :K]


def _exact_i8(x):
    scale = _exact_power_scale(x.abs().amax(-1), 127.0).unsqueeze(-1)
    return (x / scale).round().clamp(-127, 127) * scale


def _exact_operand(codes, scales, rows, K):
    """Values in 64 bits of codes whose scales lie in tiles: byte (r % 32) * 16 + (r % 128 // 32) * 4 + b % 4 of tile (r // 128, b // 4)."""
    r = torch.arange(rows, device=codes.device)[:, None]
    b = torch.arange(-(-K // _BLOCK), device=codes.device)[None]
    at = ((r // 128) * -(-b.shape[1] // 4) + b // 4) * 512 + (r % 32) * 16 + (r % 128 // 32) * 4 + b % 4
    scale = torch.ldexp(torch.ones((), dtype=torch.float64, device=codes.device), scales[at].int() - 127)
    grid = torch.tensor(_VALUES, dtype=torch.float64, device=codes.device)
    k = torch.arange(K, device=codes.device)
    code = (codes[:, k // 2] >> (4 * (k % 2)).byte()) & 15
    return torch.where(code > 7, -1.0, 1.0) * grid[(code & 7).long()] * scale[:, k // _BLOCK]


def exact(case, seed):
    st = prepare(case, seed)
    kind = case["kind"]
    if kind == "codec":
        return dict(codes=None, scales=None, values=_exact_mx(st["x"], case["rule"]))
    if kind == "linear":
        x = _exact_operand(st["x_codes"], st["x_scales"], case["M"], case["K"])
        y = x @ _exact_operand(st["w_codes"], st["w_scales"], case["N"], case["K"]).T
        y = y if st["bias"] is None else y + st["bias"].double()
        return y.clamp(min=0) if case["relu"] else y
    if kind == "norm":
        out, x = {}, st["x"].double()
        if st["residual"] is not None:
            out["sum"] = x + st["residual"].double()
            x = out["sum"].to(st["x"].dtype).double()       # what is normalised is the sum as it is kept
        y = x / torch.sqrt((x * x).sum(-1, keepdim=True) / x.shape[1] + _EPS) * st["gain"].double()
        if case["out"] == "mx":
            return dict(out, values=_exact_mx(y))
        return dict(out, codes=None) if case["out"] == "i8" else dict(out, codes=None, scales=None)
    out = {}
    for name in ("k", "v"):
        new = st[name].double()
        new = _exact_i8(new) if case["fmt"] == "i8" else _exact_mx(new)
        codes, scales = st[name + "_codes"][st["slots"]], st[name + "_scales"][st["slots"]]
        power = torch.ldexp(torch.ones((), dtype=torch.float64, device="cuda"), scales.int() - 127)
        if case["fmt"] == "i8":
            y = codes.view(torch.int8).double() * power
        else:
            grid = torch.tensor(_VALUES, dtype=torch.float64, device="cuda")
            k = torch.arange(case["D"], device="cuda")
            code = (codes[..., k // 2] >> (4 * (k % 2)).byte()) & 15
            y = torch.where(code > 7, -1.0, 1.0) * grid[(code & 7).long()] * power[..., k // _BLOCK]
        place = torch.full((st["k_codes"].shape[0],), -1, dtype=torch.int64, device="cuda")
        kept = st["new_slots"] >= 0
        place[st["new_slots"][kept]] = torch.arange(kept.numel(), device="cuda")[kept]
        from_new = place[st["slots"]]
        y[from_new >= 0] = new[from_new[from_new >= 0]]
        out.update({name: y, name + "_codes": None, name + "_scales": None})
    return out


# ------------------------------------------------------------------------------------------------ accounting
def work(case):
    """Bytes and operations of one pass: every input read once, every output written once."""
    kind = case["kind"]
    size = {"f32": 4, "bf16": 2, "f16": 2}[case["dtype"]]
    if kind == "codec":
        n = case["rows"] * case["K"]
        return dict(bytes=n * (2 * size + 17 / 32), flops=4 * n)
    if kind == "linear":
        M, N, K = case["M"], case["N"], case["K"]
        return dict(bytes=(M + N) * K * 17 / 32 + M * N * size + (4 * N if case["bias"] else 0), flops=2 * M * N * K)
    if kind == "norm":
        n = case["rows"] * case["C"]
        moved = n * size * (3 if case["residual"] else 1) + case["C"] * size
        return dict(bytes=moved + n * (size if case["out"] == "mx" else 1), flops=6 * n)
    per_row = case["heads"] * case["D"] * 2
    code = 1.0 if case["fmt"] == "i8" else 17 / 32
    rows, new = sum(_lengths(case)), case["seqs"] * case["new"]
    return dict(bytes=per_row * (new * (size + code) + rows * (code + size)) + 8 * (rows + new), flops=2 * per_row * (rows + new))
