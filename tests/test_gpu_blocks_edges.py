"""Calls around a block's linears at the edges of what they accept, on the GPU, against the float64 oracle.  Bounds as in
test_gpu_blocks.py: n roundings of float32 leave n 2^-24 of the magnitudes behind a value, an output in bf16 another 2^-8 of itself."""
import pytest
import torch

from oracle import block_ops as ref
from paper_2503_06564_amd import trdq

pytestmark = pytest.mark.gpu


def dev():
    return torch.device("cuda:0")


def rand(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed))


@pytest.mark.parametrize("params", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("c", [1, 771, 4608])
def test_no_rows_have_zero_gradients(c, params):
    """Every parameter's gradient of a call without rows is written, also where a captured graph replays it."""
    none = torch.empty(0, c, dtype=torch.bfloat16, device=dev())
    vec, mods = torch.full((c,), float("nan"), dtype=params, device=dev()), torch.ones(3, 3 * c, dtype=params, device=dev())
    off = torch.zeros(4, dtype=torch.int32, device=dev())
    grads = {k: torch.empty(c, device=dev()) for k in ("dpre_weight", "dpre_bias", "dpost_weight", "dpost_bias")}
    grads.update({k: torch.empty(3, c, device=dev()) for k in ("dscale", "dshift", "dgate")})

    def call():
        trdq.block_norm_bwd(none, none, none, none, Y=none, pre_weight=vec, pre_bias=vec, post="layer", post_weight=vec, post_bias=vec,
                            shift=mods[:, :c], scale=mods[:, c:2 * c], gate=mods[:, 2 * c:], seg_off=off, **grads)

    def check():
        torch.cuda.synchronize()
        for k, g in grads.items():
            assert bool((g == 0).all()), k
            g.fill_(9.0)

    for g in grads.values():
        g.fill_(9.0)
    call()
    check()
    dgate = torch.full((c,), 9.0, device=dev())
    trdq.block_norm_bwd(none, none, none, none, Y=none, gate=vec, dgate=dgate, seg_len=7)
    torch.cuda.synchronize()
    assert bool((dgate == 0).all())
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        call()
    for _ in range(3):
        graph.replay()
        check()


@pytest.mark.parametrize("off", [[0, 0, 9, 9, 20, 20], [0, 20, 20], [0, 0, 20]])
@pytest.mark.parametrize("c,post", [(96, None), (771, "layer"), (2304, "rms")])
def test_parameters_of_empty_segments_reach_nothing(off, c, post):
    """NaN and Inf in the scale, shift and gate of a segment without rows: the same outputs and gradients as with zeros there, zeros as
    its own gradients, also where a weight is not finite."""
    rows, segs = off[-1], len(off) - 1
    empty = torch.tensor([off[i] == off[i + 1] for i in range(segs)])
    seg_off = torch.tensor(off, dtype=torch.int32, device=dev())
    x, y, dxo, dh = ((rand(i, rows, c)).to(dev()).to(torch.bfloat16) for i in range(4))
    vec = {"pre_weight": rand(5, c), "pre_bias": rand(6, c)}
    if post:
        vec.update(post_weight=rand(7, c), post_bias=rand(8, c))
    vec["pre_weight"][3] = float("inf")
    vec = {k: v.to(dev()) for k, v in vec.items()}

    def run(mods):
        p = dict(vec, shift=mods[:, :c], scale=mods[:, c:2 * c], gate=mods[:, 2 * c:])
        xo, h, dx, dy = (torch.empty_like(x) for _ in range(4))
        grads = {"d" + k: torch.full(v.shape, 9.0, device=dev()) for k, v in p.items()}
        kw = dict(post=post, seg_off=seg_off, **p)
        trdq.block_norm(x, xo, h, Y=y, **kw)
        ws = torch.empty(trdq.block_norm_bwd_ws_nbytes(rows, c, segs), dtype=torch.uint8, device=dev())
        trdq.block_norm_bwd(dx, dy, xo, dh, Y=y, dXout=dxo, ws=ws, **grads, **kw)
        torch.cuda.synchronize()
        return dict(grads, xo=xo, h=h, dx=dx, dy=dy)

    mods = rand(9, segs, 3 * c) * 0.3
    mods[empty] = 0.0
    clean = run(mods.to(dev()))
    for bad in (float("nan"), float("inf")):
        mods[empty] = bad
        got = run(mods.to(dev()))
        for k in clean:
            assert torch.equal(got[k].nan_to_num(), clean[k].nan_to_num()) and torch.equal(got[k].isnan(), clean[k].isnan()), k
        for k in ("dscale", "dshift", "dgate"):
            assert bool((got[k].cpu()[empty] == 0).all()), k
        assert bool(got["dpre_bias"].isfinite().all())


# A dispatch counts its threads in 32 bits: calls of more rows are several.  Their rows are checked on both sides of that.

def test_norm_of_more_rows_than_a_launch_takes():
    """8 channels (four rows a workgroup of 256 threads: 2^26 - 4 rows a launch), modulated by segments of 2^25 rows."""
    rows, c, seg_len = 2 ** 26 + 37, 8, 2 ** 25
    at = torch.tensor([0, 1, 2 ** 25 - 1, 2 ** 25, 2 ** 26 - 5, 2 ** 26 - 4, 2 ** 26 - 3, 2 ** 26 - 1, 2 ** 26, rows - 1])
    mods = (rand(1, 3, 2 * c) * 0.3).to(dev())
    X, H = (torch.zeros(rows, c, dtype=torch.bfloat16, device=dev()) for _ in range(2))
    X[at.to(dev())] = rand(2, len(at), c).to(dev()).to(torch.bfloat16)
    H.fill_(7.0)
    trdq.block_norm(X, None, H, shift=mods[:, :c], scale=mods[:, c:], seg_len=seg_len)
    torch.cuda.synchronize()
    o = ref.BlockNorm({"shift": mods[:, :c].cpu().double(), "scale": mods[:, c:].cpu().double()}, at // seg_len, "layer", None, 1e-6)
    x, got = X[at.to(dev())].cpu().double(), H[at.to(dev())].cpu().double()
    assert bool(((got - o.out(x)).abs() <= 128 * 2.0 ** -24 * o.out_size(x) + 2.0 ** -8 * 1.01 * o.out(x).abs()).all())
    # every other row is zeros in, its segment's shift out
    for s in range(3):
        part = H[s * seg_len:(s + 1) * seg_len]
        same = (part == mods[s, :c].to(torch.bfloat16)).all(1)
        assert int((~same).sum()) <= len(at)


def test_norm_of_more_wide_rows_than_a_launch_takes():
    """1032 channels (a workgroup of 192 threads a row: 22369621 rows a launch), to bf16 and to codes of another row count."""
    c, at_once = 1032, 2 ** 32 // 192
    rows = at_once + 9
    X = torch.empty(rows, c, dtype=torch.bfloat16, device=dev())
    x = rand(3, 12, c).to(torch.bfloat16)
    X[-12:].copy_(x)
    H = torch.empty(rows, c, dtype=torch.bfloat16, device=dev())
    trdq.block_norm(X, None, H, pre="rms")
    few, fewer = torch.empty(12, c, dtype=torch.bfloat16, device=dev()), X[-12:].clone()
    trdq.block_norm(fewer, None, few, pre="rms")
    torch.cuda.synchronize()
    assert torch.equal(H[-12:], few)
    del H
    Q = torch.empty(rows, 1152, dtype=torch.uint8, device=dev()).view(torch.float8_e4m3fn)
    S = torch.empty(9, rows, device=dev())
    trdq.block_norm(X, None, None, codes=Q, code_scales=S, pre="rms")
    Q2, S2 = torch.empty(12, 1152, dtype=torch.uint8, device=dev()).view(torch.float8_e4m3fn), torch.empty(9, 12, device=dev())
    trdq.block_norm(fewer, None, None, codes=Q2, code_scales=S2, pre="rms")
    torch.cuda.synchronize()
    assert torch.equal(Q[-12:].view(torch.uint8), Q2.view(torch.uint8)) and torch.equal(S[:, -12:], S2)
    del X, Q, S
    torch.cuda.empty_cache()


def test_codes_of_more_rows_than_a_launch_takes():
    """One channel (32 rows a workgroup of 256 threads: 2^29 - 32 rows a launch)."""
    rows = 2 ** 29 + 75
    X = torch.ones(rows, 1, dtype=torch.bfloat16, device=dev())
    tail = rand(4, 200, 1).to(torch.bfloat16)
    X[-200:].copy_(tail)
    Q = torch.empty(rows, 128, dtype=torch.uint8, device=dev()).view(torch.float8_e4m3fn)
    S = torch.empty(1, rows, device=dev())
    trdq.fp8_quant(X, Q, S)
    torch.cuda.synchronize()
    want, s, _ = ref.quant(tail, "rows", "e4m3", False)
    assert torch.equal(Q[-200:].cpu().float().double(), want) and torch.equal(S[:, -200:].cpu().double(), s.float().double())
    one = torch.tensor(1.0) / 448.0
    assert bool((S[:, :-200] == one.item()).all()) and bool((Q[:-200, 0].view(torch.uint8) == 0x7E).all())
    del X, Q, S
    torch.cuda.empty_cache()


FORMATS = {"e4m3": (torch.float8_e4m3fn, 448.0), "e5m2": (torch.float8_e5m2, 57344.0)}


def next_to_borders(fmt, top, dtype):
    """[128, 128]: the values of one block (its rows', its columns', the tile's largest magnitude is top) that lie nearest to a border
    between two codes, and the float32 values beside them."""
    kind, most = FORMATS[fmt]
    codes = torch.arange(0, 128 if fmt == "e4m3" else 124, dtype=torch.uint8).view(kind).float().double()
    codes = codes[codes.isfinite()]
    near = ((codes[1:] + codes[:-1]) / 2 * top / most).to(dtype)
    if dtype == torch.float32:
        near = torch.cat([near, torch.nextafter(near, torch.zeros(())), torch.nextafter(near, torch.full((), 3e38))])
    v = near[torch.arange(128 * 128) % len(near)].reshape(128, 128)
    v = torch.where(torch.arange(128 * 128).reshape(128, 128) % 5 < 2, -v, v)
    v[0, :] = v[:, 0] = top
    return v


def codes_like_the_oracle(x, blocks, fmt, pow2):
    rows, c = x.shape
    r, k = (c, ref.up(rows)) if blocks in ("cols", "tiles_t") else (rows, ref.up(c))
    n = -(-r // 128) if blocks.startswith("tiles") else r
    Q = torch.full((r, k), 0x55, dtype=torch.uint8, device=dev()).view(FORMATS[fmt][0])
    S = torch.empty(k // 128, n, dtype=torch.uint8 if pow2 else torch.float32, device=dev())
    trdq.fp8_quant(x.to(dev()), Q, S, blocks=blocks)
    torch.cuda.synchronize()
    want, s, _ = ref.quant(x, blocks, fmt, pow2)
    got = S.cpu().double() if not pow2 else torch.pow(2.0, S.cpu().double() - 127)
    assert torch.equal(got, s.float().double()), (blocks, fmt, pow2)
    bad = Q.cpu().float().double() != want
    assert not bool(bad.any()), (blocks, fmt, pow2, int(bad.sum()))


@pytest.mark.parametrize("blocks", ["rows", "cols", "tiles", "tiles_t"])
@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_codes_next_to_borders(blocks, fmt, dtype):
    """Every code is the nearest to the exact quotient: float32 values within a rounding of a border, and bf16 ones on it (the largest
    value is 7 times a power of two), in blocks from the smallest scale to the largest."""
    g = torch.Generator().manual_seed(11)
    tiles = []
    for e in (-100, -99, -95, -90, -85, -80, -60, -20, 0, 3, 40, 100, 126, 127):
        if dtype == torch.float32:
            mantissa = 1.0 + torch.randint(0, 2 ** 23, (), generator=g).item() * 2.0 ** -23
        else:
            mantissa = 1.75
        tiles.append(next_to_borders(fmt, mantissa * 2.0 ** e, dtype))
    x = torch.cat(tiles, 1)
    for pow2 in (False, True):
        codes_like_the_oracle(x, blocks, fmt, pow2)


@pytest.mark.parametrize("blocks", ["rows", "cols", "tiles", "tiles_t"])
def test_codes_of_any_float32(blocks):
    """Every code of ordinary float32 values, at a ragged size."""
    x = rand(21, 1000, 1411) * torch.exp2(rand(22, 1000, 1411).mul(6).round())
    for fmt in FORMATS:
        for pow2 in (False, True):
            codes_like_the_oracle(x, blocks, fmt, pow2)


@pytest.mark.parametrize("m,k,n", [(16, 8192, 512), (100, 4096, 300), (512, 1152, 3456), (1000, 8192, 1152), (2100, 4100, 2200)])
@pytest.mark.parametrize("a_fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("pow2", [False, True])
@pytest.mark.parametrize("hot", [False, True])
def test_products_as_a_whole(m, k, n, a_fmt, pow2, hot):
    """The norm of a product's error beside the norm of the product.  Outputs in bf16: rounding is even over half a step, at most 2^-8 / sqrt 3 =
    2.26e-3.  The instruction cuts seven of eight products by up to 2^-13 of the largest, which is three to four times their root mean
    square: sqrt(7 / 3 / 8) 2^-13 4 = 2.6e-4 without a common sign, the two together 2.27e-3 (a common sign would add up over K: 2e-2 at
    8192).  Outputs in float32: 16 roundings in a block and one a block, of sums no larger than the last on the whole,
    sqrt(16 + 64) 2^-24 = 5.3e-7 and twice that for sums cut in place of rounded."""
    x, w = rand(31, m, k), rand(32, n, k) * 0.02
    if hot:
        x[:, ::128] *= 20.0
    qa, sa, _ = ref.quant(x.to(torch.bfloat16), "rows", a_fmt, pow2)
    qb, sb, _ = ref.quant(w, "tiles", "e4m3", pow2)
    A, B = qa.float().to(dev()).to(FORMATS[a_fmt][0]), qb.float().to(dev()).to(FORMATS["e4m3"][0])
    put = lambda s: torch.log2(s).add(127).to(torch.uint8).to(dev()) if pow2 else s.to(dev())  # noqa: E731
    sa, sb = sa.float(), sb.float()
    need = trdq.fp8_gemm_ws_nbytes(m, n, A.shape[1])
    ws = torch.empty(need, dtype=torch.uint8, device=dev()) if need else None
    want = (qa * ref.wide(sa, *qa.shape)).to(dev()) @ (qb * ref.wide(sb, *qb.shape)).to(dev()).t()
    for dtype, bound in ((torch.bfloat16, 2.3e-3), (torch.float32, 1.1e-6)):
        Y = torch.empty(m, n, dtype=dtype, device=dev())
        trdq.fp8_gemm(A, put(sa), B, put(sb), Y, ws=ws)
        torch.cuda.synchronize()
        err = float((Y.double() - want).norm() / want.norm())
        print(f"{m} x {k} x {n} {a_fmt} pow2={pow2} hot={hot} {dtype}: {err:.3e}", flush=True)
        assert err <= bound, (dtype, err)
