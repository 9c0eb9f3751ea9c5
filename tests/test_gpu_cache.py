"""The 8-bit paged cache on the GPU against its plain definition in 64 bits (oracle/cache.py)."""
import math

import numpy as np
import pytest

from oracle import cache as oc

pytestmark = pytest.mark.gpu
PLACE = [4 * ((t % 8) // 2) + 2 * (t // 8) + t % 2 for t in range(16)]


@pytest.fixture(scope="module")
def torch():
    t = pytest.importorskip("torch")
    if not t.cuda.is_available():
        pytest.skip("needs a CUDA device")
    return t


def _bytes(x, fmt):
    """Codes as numbers -> bytes."""
    if fmt == "int8":
        return x.astype(np.int8).view(np.uint8)
    return (np.searchsorted(oc.e4m3_values(), np.abs(x)) | np.where(np.signbit(x), 0x80, 0)).astype(np.uint8)


def _pool(c):
    """The oracle's codes in the order of the pool."""
    b = _bytes(c.codes, c.fmt)
    L, kv, P, _, T, D = b.shape
    out = np.empty((L, kv, P, 2, T * D), np.uint8)
    out[..., 0, :] = b[..., 0, :, :].reshape(L, kv, P, 2, 8, D // 16, 16).swapaxes(-2, -3).reshape(L, kv, P, -1)
    v = np.empty((L, kv, P, D, T), np.uint8)
    v[..., PLACE] = b[..., 1, :, :].swapaxes(-1, -2)
    out[..., 1, :] = v.reshape(L, kv, P, -1)
    return out


def _upload(torch, c):
    from paper_2503_14153_b200 import SpecCache
    ints = lambda a: torch.from_numpy(np.ascontiguousarray(a).astype(np.int32)).cuda()  # noqa: E731
    return SpecCache.from_tensors(torch.from_numpy(_pool(c)).cuda(), torch.from_numpy(c.scales.astype(np.float32)).cuda(), ints(c.table), ints(c.refs), ints(c.lens), fmt=c.fmt)


def _ints(torch, v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _filled(rng, layers, kv, D, lens, fmt, width=None, spare=2):
    """An oracle cache whose sequences hold random rows on scattered pages; float32 scales."""
    need = [-(-n // 16) for n in lens]
    c = oc.Cache(layers, kv, D, sum(need) + spare, len(lens), max(need + [1]) + 1 if width is None else width, fmt)
    order = list(rng.permutation(len(c.refs)))
    for b, n in enumerate(lens):
        for i in range(need[b]):
            c.table[b, i] = order.pop()
            c.refs[c.table[b, i]] = 1
        c.lens[b] = n
    x = rng.standard_normal((layers, kv, len(c.refs), 2, 16, D)) * np.exp(0.4 * rng.standard_normal((layers, kv, len(c.refs), 2, 1, 1)))
    c.scales[:] = (np.abs(x).max(axis=(-1, -2)) / oc.CODE_MAX[fmt]).astype(np.float32)
    c.codes[:] = oc.nearest_code(x / c.scales[..., None, None], fmt)
    return c


def _tree(rng, nodes):
    sees = np.zeros((nodes, nodes), bool)
    for i in range(nodes):
        if i:
            sees[i] = sees[rng.integers(max(0, i - 9), i)]
        sees[i, i] = True
    return sees


def _words(torch, sees_list, words):
    rows = []
    for s in sees_list:
        for r in s:
            bits = np.zeros(32 * words, bool)
            bits[:len(r)] = r
            rows.append(np.packbits(bits, bitorder="little").view(np.int32))
    return torch.from_numpy(np.stack(rows).copy()).cuda()


def _check_attention(torch, rng, D, kv, G, lens, rows, fmt, dtype, mask="tree", peak=1.0, spoil=None, seqs=None, cache=None, strided=False, scale=None):
    """rows: the groups' numbers of rows (an int: the same for all). Compares out and lse with the oracle."""
    B, H = len(lens), kv * G
    counts = [rows] * B if isinstance(rows, int) else rows
    c = _filled(rng, 2, kv, D, lens, fmt)
    dev = _upload(torch, c)
    R = sum(counts)
    offs = np.concatenate([[0], np.cumsum(counts)])
    dt = getattr(torch, dtype)
    wide = torch.from_numpy(rng.standard_normal((max(R, 1), H + 2 * kv, D)).astype(np.float32)).cuda()[:R]
    wide[:, :H] *= peak
    wide = wide.to(dt)
    q, k, v = wide[:, :H], wide[:, H:H + kv], wide[:, H + kv:]
    if not strided:
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    sees = [np.tril(np.ones((n, n), bool)) if mask == "causal" else np.zeros((n, n), bool) if mask == "nothing" else _tree(rng, n) for n in counts]
    if mask == "holes":
        sees = [s & (rng.random(s.shape) < 0.5) for s in sees]
    m = None if mask == "causal" else _words(torch, sees, -(-max(counts + [1]) // 32)) if R else None
    if spoil:
        spoil(q, k, v, sees, dev, c)
    perm = list(range(B)) if seqs is None else seqs
    scale = 1 / math.sqrt(D) if scale is None else scale
    out, lse = dev.attention(1, q, k, v, batch=B, row_offsets=None if isinstance(rows, int) else _ints(torch, offs.tolist()), max_rows=None if isinstance(rows, int) else max(counts + [1]),
                             seqs=None if seqs is None else _ints(torch, seqs), mask=m, scale=scale, lse=True)
    dev.check()
    out, lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    f = lambda t: t.double().cpu().numpy()  # noqa: E731
    qn, kn, vn = f(q), f(k), f(v)
    # relative rounding: of the weights and of the result to the operand type (2^-p of a format with p significant bits), of float32 sums and exponents (the score's size times 2^-21)
    unit = {"bfloat16": 2.0 ** -8, "float16": 2.0 ** -11, "float32": 2.0 ** -22}[dtype]
    for b in range(B):
        at = slice(offs[b], offs[b + 1])
        K, V = c.rows(perm[b], 1, 0), c.rows(perm[b], 1, 1)
        with np.errstate(invalid="ignore", over="ignore"):
            want, wl, mass = oc.attention(qn[at], kn[at], vn[at], K, V, sees[b], scale)
        z = scale * np.linalg.norm(np.nan_to_num(qn[at]), axis=-1) * max(np.linalg.norm(K, axis=-1).max(initial=0), np.linalg.norm(np.nan_to_num(kn[at], posinf=0, neginf=0), axis=-1).max(initial=0))
        z = z.max(initial=0)
        fin = np.isfinite(want)
        assert np.array_equal(fin, np.isfinite(out[at])), "non-finite values elsewhere"
        bound = unit * np.abs(want) + (2 * unit + (8 + z) * 2.0 ** -21) * mass + 1e-6 * (dtype == "float16")
        bad = fin & (np.abs(out[at] - want) > bound)
        assert not bad.any(), (b, np.argwhere(bad)[:5], np.abs(out[at] - want)[bad][:5], bound[bad][:5])
        fl = np.isfinite(wl)
        assert np.array_equal(wl[~fl & ~np.isnan(wl)], lse[at][~fl & ~np.isnan(wl)])
        assert (np.abs(lse[at] - wl)[fl] <= (8 + z) * 2.0 ** -20).all(), np.abs(lse[at] - wl)[fl].max()
    return dev, (q, k, v, m)


@pytest.mark.parametrize("dtype", ["bfloat16", "float16", "float32"])
@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("D,kv,G", [(64, 2, 1), (128, 2, 4), (128, 1, 7), (64, 1, 16)])
def test_attention_one_token(torch, dtype, fmt, D, kv, G):
    rng = np.random.default_rng(D + G)
    _check_attention(torch, rng, D, kv, G, [0, 1, 15, 16, 17, 127, 128, 129, 400], 1, fmt, dtype, mask="causal")


@pytest.mark.parametrize("rows", [2, 7, 16, 17, 23, 33, 64, 65, 100, 128])
@pytest.mark.parametrize("D,kv,G,fmt,dtype", [(128, 2, 1, "int8", "bfloat16"), (64, 2, 4, "e4m3", "float16"), (128, 1, 3, "e4m3", "bfloat16"), (64, 1, 1, "int8", "float32")])
def test_attention_trees(torch, rows, D, kv, G, fmt, dtype):
    rng = np.random.default_rng(rows)
    _check_attention(torch, rng, D, kv, G, [0, 31, 300], rows, fmt, dtype, strided=rows % 2 == 1)


@pytest.mark.parametrize("rows,n", [(65, 0), (130, 5), (257, 129), (300, 64), (128, 300)])
@pytest.mark.parametrize("D,kv,G", [(128, 1, 2), (64, 2, 1)])
def test_attention_prompts(torch, rows, n, D, kv, G):
    _check_attention(torch, np.random.default_rng(rows), D, kv, G, [n], rows, "int8", "bfloat16", mask="causal")


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("counts", [[5, 0, 40, 1], [0, 0, 3], [64, 63, 1, 65, 17]])
def test_attention_ragged_rows_and_other_sequences(torch, counts, dtype):
    rng = np.random.default_rng(sum(counts))
    B = len(counts)
    _check_attention(torch, rng, 128, 2, 2, [int(x) for x in rng.integers(0, 200, B)], counts, "int8", dtype, seqs=[int(x) for x in rng.permutation(B)])


@pytest.mark.parametrize("dtype", ["bfloat16", "float16", "float32"])
def test_attention_rows_that_see_nothing_or_little(torch, dtype):
    rng = np.random.default_rng(5)
    _check_attention(torch, rng, 64, 2, 2, [0, 0, 20], 9, "int8", dtype, mask="nothing")
    _check_attention(torch, rng, 128, 2, 2, [0, 3], 70, "e4m3", dtype, mask="holes")


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("rows", [6, 40, 90])
def test_attention_peaked_scores(torch, rows, dtype):
    # scores of up to hundreds: the running maximum moves, most weights vanish
    _check_attention(torch, np.random.default_rng(rows), 128, 2, 1, [500, 90], rows, "int8", dtype, peak=12.0)


@pytest.mark.parametrize("dtype", ["bfloat16", "float16", "float32"])
@pytest.mark.parametrize("rows", [8, 70])
def test_attention_values_in_masked_places_do_not_matter(torch, rows, dtype):
    def spoil(q, k, v, sees, dev, c):
        for b, s in enumerate(sees):
            dead = [j for j in range(1, rows) if s[:, j].sum() == 1][:3]          # rows that only they themselves see
            for j, x in zip(dead, (float("nan"), float("inf"), -float("inf"))):
                v[b * rows + j] = x
                if j == dead[0]:
                    k[b * rows + j] = float("nan")
        # bytes past a sequence's end: anything, NaN codes among it
        for b in range(len(sees)):
            n = int(c.lens[b])
            if n % 16:
                blk = dev.codes[1, :, int(c.table[b, n // 16])]
                t = torch.arange(16 * dev.head_dim, device="cuda")
                kt = (t // (8 * dev.head_dim)) * 8 + (t % 128) // 16
                vt = torch.tensor([PLACE.index(p) for p in range(16)], device="cuda")[t % 16]
                blk[:, 0, kt >= n % 16] = 0x7f
                blk[:, 1, vt >= n % 16] = 0xff
        free = torch.from_numpy(np.flatnonzero(c.refs == 0)).cuda()
        dev.codes[:, :, free] = 0x7f
        dev.scales[:, :, free] = float("nan")
    _check_attention(torch, np.random.default_rng(rows), 128, 2, 2, [37, 5, 130], rows, "e4m3", dtype, spoil=spoil)


def test_attention_values_of_very_unequal_size(torch):
    def spoil(q, k, v, sees, dev, c):
        f = torch.from_numpy(10.0 ** np.random.default_rng(3).uniform(-6, 3, tuple(dev.scales.shape))).float().cuda()
        f[..., 0] = 1.0
        f[:, :, ::5, 1] = 0.0                                                    # blocks of zeros: scale 0
        dev.scales *= f
        c.scales[:] = dev.scales.double().cpu().numpy()
    for rows in (1, 30, 80):
        _check_attention(torch, np.random.default_rng(rows), 128, 2, 1, [333, 64], rows, "int8", "bfloat16", spoil=spoil, mask="causal")


def test_attention_repeats_bit_for_bit_and_on_another_stream(torch):
    rng = np.random.default_rng(8)
    dev, (q, k, v, m) = _check_attention(torch, rng, 128, 4, 1, [900, 20], 33, "int8", "bfloat16")
    a = dev.attention(1, q, k, v, batch=2, mask=m)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        b = dev.attention(1, q, k, v, batch=2, mask=m)
    outs = [dev.attention(1, q, k, v, batch=2, mask=m) for _ in range(20)]        # both streams at once
    side.synchronize()
    torch.cuda.synchronize()
    assert torch.equal(a, b) and all(torch.equal(a, x) for x in outs)


@pytest.mark.parametrize("batch,heads,kv,D,n,rows,mask,fmt", [(1, 32, 32, 128, 2048, 1024, "causal", "int8"), (1, 32, 32, 128, 8192, 64, "tree", "int8"), (1, 32, 8, 128, 4100, 128, "tree", "e4m3"),
                                                              (3, 16, 4, 64, 3000, 23, "tree", "e4m3"), (1, 16, 4, 64, 0, 1500, "causal", "int8"), (5, 32, 8, 128, 3000, 1, "causal", "int8")])
def test_attention_many_tiles_a_cta(torch, batch, heads, kv, D, n, rows, mask, fmt):
    """Passes in which a CTA has many tiles and several units, against the float32 kernel (which the other tests hold to the definition) on the same values."""
    from paper_2503_14153_b200 import SpecCache
    rng = np.random.default_rng(n + rows)
    g = torch.Generator(device="cuda").manual_seed(n + rows)
    per = -(-n // 16) + 1
    dev = SpecCache(1, kv, D, batch * per + 3, batch, per, fmt=fmt)
    lens = [n - 37 * b for b in range(batch)]
    dev.reserve(_ints(torch, lens))
    dev.codes.copy_(torch.randint(0, 256, dev.codes.shape, generator=g, device="cuda", dtype=torch.uint8) & (0xff if fmt == "int8" else 0xbf))      # (e4m3: below 2)
    dev.codes[dev.codes == 0x80] = 0
    dev.scales.copy_(torch.rand(dev.scales.shape, generator=g, device="cuda") * (0.03 if fmt == "int8" else 2.0) + 1e-3)
    positive = SpecCache.from_tensors(dev.codes.clone(), dev.scales, dev.page_table, dev.refs, dev.lens, fmt=fmt)
    positive.codes[:, :, :, 1] = dev.codes[:, :, :, 1].view(torch.int8).abs().view(torch.uint8) if fmt == "int8" else dev.codes[:, :, :, 1] & 0x7f
    q, k, v = ((torch.randn((batch * rows, h, D), generator=g, device="cuda") * s).bfloat16() for h, s in ((heads, 1.5), (kv, 1.0), (kv, 1.0)))
    m = _words(torch, [_tree(rng, rows) for _ in range(batch)], -(-rows // 32)) if mask == "tree" else None
    out, lse = dev.attention(0, q, k, v, batch=batch, mask=m, lse=True)
    dev.check()
    want, wl = dev.attention(0, q.float(), k.float(), v.float(), batch=batch, mask=m, lse=True)
    mass = positive.attention(0, q.float(), k.float(), v.float().abs(), batch=batch, mask=m)
    # rounding of weights and result to bf16, of scores (up to some tens) and sums to float32 on both sides
    assert ((out.float() - want).abs() <= 2.0 ** -8 * want.abs() + (2.0 ** -7 + 2.0 ** -14) * mass).all()
    assert ((lse - wl).abs() <= 2.0 ** -14).all()


@pytest.mark.parametrize("batch,heads,kv,rows,n", [(4500, 4, 1, 1, 9), (300, 1, 1, 40, 20), (270, 2, 1, 50, 3), (4200, 1, 1, 12, 2)])
def test_attention_more_sequences_than_a_launch_deals(torch, batch, heads, kv, rows, n):
    from paper_2503_14153_b200 import SpecCache
    g = torch.Generator(device="cuda").manual_seed(batch)
    dev = SpecCache(1, kv, 64, 2 * batch, batch, 2)
    for b0 in range(0, batch, 1000):
        m = min(1000, batch - b0)
        seqs = torch.arange(b0, b0 + m, dtype=torch.int32, device="cuda")
        dev.reserve(torch.full((m,), n, dtype=torch.int32, device="cuda"), seqs=seqs)
    dev.codes.copy_(torch.randint(1, 256, dev.codes.shape, generator=g, device="cuda", dtype=torch.uint8))
    dev.codes[dev.codes == 0x80] = 1
    dev.scales.copy_(torch.rand(dev.scales.shape, generator=g, device="cuda") * 0.03 + 1e-3)
    q, k, v = (torch.randn((batch * rows, h, 64), generator=g, device="cuda").bfloat16() for h in (heads, kv, kv))
    out = dev.attention(0, q, k, v, batch=batch)
    dev.check()
    want = dev.attention(0, q.float(), k.float(), v.float(), batch=batch)
    # cached values are at most 4.0 in size and nearly all of the rows' below 4.2, and so are their weighted means; rounding of weights and results to bf16
    assert ((out.float() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -7 * 4.2).all()
    spread = (out.float() - want).square().mean().sqrt() / want.square().mean().sqrt()
    assert spread <= 2.0 ** -7


def test_attention_calls_of_other_sizes_share_a_workspace(torch):
    rng = np.random.default_rng(21)
    c = _filled(rng, 1, 4, 128, [700, 90, 1500], "int8")
    dev = _upload(torch, c)
    sizes = [(1, 1), (3, 1), (1, 64), (3, 20), (1, 300), (3, 5), (2, 128), (3, 1), (1, 1)]
    g = torch.Generator(device="cuda").manual_seed(5)
    made = [[torch.randn((b * r, h, 128), generator=g, device="cuda").bfloat16() for h in (8, 4, 4)] for b, r in sizes]
    alone = []
    for (b, r), x in zip(sizes, made):
        alone.append(_upload(torch, c).attention(0, *x, batch=b))
    for _ in range(3):
        for (b, r), x, want in zip(sizes, made, alone):
            assert torch.equal(dev.attention(0, *x, batch=b), want), (b, r)
    dev.check()


def test_attention_long_cache_past_two_gigabytes(torch):
    # block offsets of more than 2^31 bytes: a pool of 2.3 GB of which the sequence holds the last pages
    from paper_2503_14153_b200 import SpecCache
    kv, D, pages = 8, 128, 72000
    dev = SpecCache(1, kv, D, pages, 1, 8)
    rng = np.random.default_rng(4)
    c = _filled(rng, 1, kv, D, [100], "int8", spare=0)
    small = _upload(torch, c)
    for i in range(7):
        dev.codes[:, :, pages - 1 - i] = small.codes[:, :, int(c.table[0, i])]
        dev.scales[:, :, pages - 1 - i] = small.scales[:, :, int(c.table[0, i])]
        dev.page_table[0, i] = pages - 1 - i
    dev.lens[0] = 100
    for rows in (1, 64):
        q, k, v = (torch.randn((rows, h, D), device="cuda").bfloat16() for h in (16, kv, kv))
        a = dev.attention(0, q, k, v)
        b = small.attention(0, q, k, v)
        assert torch.equal(a, b)
    ka, va = dev.read(None, 112)
    kb, vb = small.read(None, 112)
    assert torch.equal(ka, kb) and torch.equal(va, vb)


def test_attention_marks_pages_out_of_range(torch):
    from paper_2503_14153_b200 import SpecError
    rng = np.random.default_rng(9)
    dev = _upload(torch, _filled(rng, 2, 2, 64, [40], "int8"))
    q = torch.randn((1, 2, 64), device="cuda").bfloat16()
    for bad in (-1, 10 ** 6):
        dev.page_table[0, 1] = bad
        dev.attention(0, q, q, q)
        with pytest.raises(SpecError, match="out of range"):
            dev.check()
    dev.attention(0, q, q, q, seqs=_ints(torch, [7]))
    with pytest.raises(SpecError):
        dev.check()
    dev.check()


# ---------------------------------------------------------------- store and read
@pytest.mark.parametrize("dtype", ["bfloat16", "float16", "float32"])
@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("D,kv", [(64, 3), (128, 2)])
def test_store_and_read(torch, dtype, fmt, D, kv):
    rng = np.random.default_rng(D + kv)
    lens, counts, rows = [0, 1, 15, 16, 30, 47, 0], [1, 3, 1, 5, 40, 0, 33], 40
    c = _filled(rng, 3, kv, D, lens, fmt, width=8, spare=12)
    dev = _upload(torch, c)
    B = len(lens)
    x = rng.standard_normal((2, 3, B * rows, kv, D)) * np.exp(rng.standard_normal((2, 3, B * rows, kv, 1)))
    k, v = (torch.from_numpy(x[i]).cuda().to(getattr(torch, dtype)) for i in range(2))
    path = np.stack([np.sort(rng.permutation(rows)[:40]) for _ in range(B)])
    granted = dev.reserve(_ints(torch, counts))
    assert granted.tolist() == c.reserve(range(B), counts) == counts
    assert np.array_equal(dev.page_table.cpu().numpy(), c.table)
    dev.store(k, v, granted, path=_ints(torch, path.tolist()))
    dev.check()
    exact = np.stack([k.double().cpu().numpy(), v.double().cpu().numpy()], axis=1)
    for b in range(B):
        c.store(b, exact[:, :, b * rows + path[b, :counts[b]]])
    touched = sorted({int(c.table[b, p]) for b in range(B) for p in range(lens[b] // 16, -(-(lens[b] + counts[b]) // 16)) if counts[b]})
    rest = [p for p in range(len(c.refs)) if p not in touched]
    sc = dev.scales.double().cpu().numpy()
    assert np.allclose(sc[:, :, touched], c.scales[:, :, touched], rtol=2.0 ** -22, atol=0) and np.array_equal(sc[:, :, rest].astype(np.float32), c.scales[:, :, rest].astype(np.float32))
    got, want = dev.codes.cpu().numpy(), _pool(c)
    assert np.array_equal(got[:, :, rest], want[:, :, rest])
    # a code may be the neighbour of the definition's where the value, in units of the scale, lies within float32 rounding of a tie
    if fmt == "int8":
        off = np.abs(got.view(np.int8).astype(int) - want.view(np.int8).astype(int))
    else:
        signed = lambda u: np.where(u & 0x80, -(u & 0x7f).astype(int), (u & 0x7f).astype(int))  # noqa: E731
        off = np.abs(signed(got) - signed(want))
    assert off.max() <= 1 and (off > 0).mean() < 2e-3
    # what is read back is what is stored
    start, window = [max(0, n - 3) for n in lens], 50
    for rd in ("float32", dtype):
        rk, rv = dev.read(_ints(torch, start), window, dtype=getattr(torch, rd))
        unit = {"float32": 2.0 ** -23, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}[rd]
        for w, r in enumerate((rk, rv)):
            r = r.double().cpu().numpy()
            for b in range(B):
                n = min(window, int(c.lens[b]) - start[b])
                for l in range(3):
                    y = c.rows(b, l, w)[start[b]:start[b] + n]
                    step = c.scales[l][:, c.table[b, (start[b] + np.arange(n)) // 16], w].T[..., None]
                    assert (np.abs(r[l, b, :n] - y) <= unit * np.abs(y) + step * (33.0 if fmt == "e4m3" else 1.01)).all()
                    assert (r[l, b, n:] == 0).all()


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_store_special_values(torch, fmt):
    from paper_2503_14153_b200 import SpecCache
    dev = SpecCache(1, 1, 64, 4, 2, 2, fmt=fmt)
    x = torch.zeros((1, 2, 1, 64), device="cuda")
    x[0, 0, 0, :6] = torch.tensor([float("inf"), -float("inf"), float("nan"), 2.0, -1.0, 1e-38])
    x[0, 1] = 1e-33
    dev.reserve(_ints(torch, [1, 1]))
    dev.store(x, x, _ints(torch, [1, 1]))
    k, v = dev.read(None, 1, dtype=torch.float32)
    assert torch.equal(k, v)
    got = k[0, 0, 0, 0, :7].tolist()
    assert got[:4] == pytest.approx([2.0, -2.0, 0.0, 2.0]) and got[4] == pytest.approx(-1.0, rel=0.07) and got[5:] == [0.0, 0.0]
    assert (k[0, 1] == 0).all() and dev.scales[0, 0, int(dev.page_table[1, 0])].tolist() == [0.0, 0.0]
    # a page of zeros takes rows of ordinary size as if it were new
    y = torch.full((1, 2, 1, 64), 0.5, device="cuda")
    dev.reserve(_ints(torch, [1, 1]))
    dev.store(y, y, _ints(torch, [1, 1]))
    assert dev.read(None, 2, dtype=torch.float32)[0][0, 1, 1, 0, 0].item() == pytest.approx(0.5)


def test_store_layers_strides_ragged_rows_and_marks(torch):
    from paper_2503_14153_b200 import SpecCache, SpecError
    kv, D = 2, 128
    dev = SpecCache(3, kv, D, 20, 3, 8)
    full = torch.randn((2, 11, 5 * kv, D), device="cuda").bfloat16()
    k, v = full[:, :, kv:2 * kv], full[:, :, 3 * kv:4 * kv]                          # strided views
    seqs, offs, path = _ints(torch, [2, 0]), _ints(torch, [0, 4, 11]), _ints(torch, [[1, 3, 0], [6, 2, 5]])
    got = dev.reserve(_ints(torch, [2, 3]), seqs=seqs)
    dev.store(k, v, got, seqs=seqs, row_offsets=offs, path=path, layer0=1)
    dev.check()
    rk, rv = dev.read(None, 3, batch=2, seqs=seqs, layer0=1, layers=2)
    for r, x in ((rk, k), (rv, v)):
        want = torch.zeros_like(r)
        want[:, 0, :2], want[:, 1] = x[:, [1, 3]], x[:, [4 + 6, 4 + 2, 4 + 5]]
        assert ((r - want).abs() <= want.abs().amax(dim=(2, 4), keepdim=True) / 127 * 0.51 + 0.01 * want.abs()).all()
    assert (dev.codes[0] == 0).all()
    dev.reserve(_ints(torch, [1]), seqs=_ints(torch, [2]))
    dev.store(k, v, _ints(torch, [1]), seqs=_ints(torch, [2]), path=_ints(torch, [[11]]))
    with pytest.raises(SpecError):
        dev.check()


# ---------------------------------------------------------------- pages
def test_pages_against_the_definition(torch):
    """A long random run of the four operations; every table, count, length and code is compared after each."""
    rng = np.random.default_rng(11)
    S, P = 7, 61
    c = oc.Cache(2, 2, 64, P, S, 9, "int8")
    c.codes[:] = rng.integers(-127, 128, c.codes.shape)
    c.scales[:] = rng.random(c.scales.shape).astype(np.float32)
    dev = _upload(torch, c)
    full = 0
    for step in range(150):
        kind = rng.integers(0, 8)
        if kind == 0:
            src, dst = [int(s) for s in range(S) if c.lens[s]], [int(s) for s in range(S) if not c.lens[s]]
            n = min(len(dst), rng.integers(1, 4)) if src else 0
            pairs = [(src[rng.integers(len(src))], d) for d in dst[:n]]
            if pairs:
                c.fork(*zip(*pairs))
                dev.fork(_ints(torch, [p[0] for p in pairs]), _ints(torch, [p[1] for p in pairs]))
        elif kind in (1, 2, 3, 4):
            seqs = [int(s) for s in rng.permutation(S)[:rng.integers(1, S + 1)]]
            counts = [int(x) for x in rng.choice([0, 1, 2, 5, 16, 17, 40, -3, 200], len(seqs))]
            want = c.reserve(seqs, counts)
            full += sum(w < x for w, x in zip(want, counts))
            assert dev.reserve(_ints(torch, counts), seqs=_ints(torch, seqs)).tolist() == want
        elif kind in (5, 6):
            seqs = [int(s) for s in rng.permutation(S)[:rng.integers(1, 4)]]
            keep = [int(x) for x in rng.integers(0, 100, len(seqs))] if kind == 5 else [0] * len(seqs)
            c.truncate(seqs, keep)
            dev.truncate(_ints(torch, keep) if kind == 5 else None, seqs=_ints(torch, seqs))
        else:
            assert dev.compact().item() == c.compact()
        dev.check()
        assert np.array_equal(dev.page_table.cpu().numpy(), c.table) and np.array_equal(dev.refs.cpu().numpy(), c.refs) and np.array_equal(dev.lens.cpu().numpy(), c.lens), step
        assert np.array_equal(dev.codes.cpu().numpy(), _pool(c)) and np.array_equal(dev.scales.cpu().numpy(), c.scales.astype(np.float32)), step
    assert full > 10                                                                # the pool did run out


def test_pages_many_sequences_and_pages(torch):
    from paper_2503_14153_b200 import SpecCache
    S = 1024
    dev = SpecCache(1, 1, 64, 9000, S, 9)
    counts = [(b * 37) % 140 for b in range(S)]
    c = oc.Cache(1, 1, 64, 9000, S, 9, "int8")
    assert dev.reserve(_ints(torch, counts)).tolist() == c.reserve(range(S), counts)
    assert np.array_equal(dev.page_table.cpu().numpy(), c.table) and np.array_equal(dev.refs.cpu().numpy(), c.refs)
    drop = list(range(0, S, 3))
    dev.truncate(seqs=_ints(torch, drop))
    c.truncate(drop, [0] * len(drop))
    assert dev.compact().item() == c.compact()
    assert np.array_equal(dev.page_table.cpu().numpy(), c.table) and np.array_equal(dev.refs.cpu().numpy(), c.refs)
    dev.truncate()
    assert (dev.refs == 0).all() and (dev.lens == 0).all() and (dev.page_table == -1).all()


def test_fork_refuses_a_sequence_in_use(torch):
    from paper_2503_14153_b200 import SpecCache, SpecError
    dev = SpecCache(1, 1, 64, 9, 3, 4)
    dev.reserve(_ints(torch, [20, 5, 0]))
    before = dev.refs.clone()
    dev.fork(_ints(torch, [0]), _ints(torch, [1]))
    assert torch.equal(before, dev.refs) and dev.lens.tolist() == [20, 5, 0]
    with pytest.raises(SpecError):
        dev.check()


# ---------------------------------------------------------------- rotary
@pytest.mark.parametrize("src,dst", [("float32", "bfloat16"), ("bfloat16", "bfloat16"), ("float32", "float32"), ("bfloat16", "float16"), ("float16", "float32")])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rows,H,kv,D,rot,shift", [(1, 32, 32, 128, 128, 0), (5, 8, 2, 64, 32, 0), (130, 3, 1, 96, 40, 0), (7, 4, 4, 64, 64, 1), (3, 2, 1, 66, 6, 0), (2, 1, 1, 8, 2, 0), (9, 40, 8, 128, 16, 0)])
def test_rotary(torch, src, dst, interleaved, rows, H, kv, D, rot, shift):
    from paper_2503_14153_b200 import rotary_frequencies, spec_rotary, spec_rotary_table
    rng = np.random.default_rng(rows)
    span = 70000
    args = dict(base=1e6, scaling=["none", "linear", "yarn"][rows % 3], factor=4.0, original=8192)
    table = spec_rotary_table(span, rot, **args)
    freq, gain = rotary_frequencies(rot, **args)
    pos = rng.integers(0, span, rows)
    flat = torch.from_numpy(rng.standard_normal(rows * (H + 2 * kv) * D + 8).astype(np.float32)).cuda().to(getattr(torch, src))
    x = flat[shift:shift + rows * (H + 2 * kv) * D].view(rows, H + 2 * kv, D)          # (shift 1: rows off every vector boundary)
    q, k, v = x.split((H, kv, kv), dim=1)
    qo, ko, vo = spec_rotary(q, k, v, _ints(torch, pos.tolist()), table, interleaved=interleaved, dtype=getattr(torch, dst))
    unit = {"float32": 2.0 ** -24, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}[dst]
    for y, t in ((qo, q), (ko, k)):
        t = t.double().cpu().numpy()
        want = oc.rotate(t, pos, freq, gain, interleaved)
        size = np.abs(t).max()
        # half a unit of the result; the table's entries and the products round to float32 (four roundings)
        assert (np.abs(y.double().cpu().numpy() - want) <= unit * np.abs(want) + 8 * 2.0 ** -24 * size * gain).all()
    assert torch.equal(vo, v.to(getattr(torch, dst)))


def test_rotary_positions_outside_the_table_and_no_v(torch):
    from paper_2503_14153_b200 import spec_rotary, spec_rotary_table
    table = spec_rotary_table(10, 64, 1e4)
    q = torch.randn((4, 2, 128), device="cuda")
    qo, ko, vo = spec_rotary(q, q[:, :1], None, _ints(torch, [9, 10, -1, 0]), table)
    assert vo is None and torch.isnan(qo[1:3, :, :64]).all() and torch.isfinite(qo[1:3, :, 64:]).all() and torch.isfinite(qo[[0, 3]]).all() and torch.equal(qo[3], q[3])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        b = spec_rotary(q, q[:, :1], None, _ints(torch, [9, 10, -1, 0]), table)[0]
    side.synchronize()
    assert torch.equal(torch.nan_to_num(b), torch.nan_to_num(qo))


def test_refusals_of_the_python_side(torch):
    from paper_2503_14153_b200 import SpecCache, SpecError, spec_rotary, spec_rotary_table
    dev = SpecCache(2, 2, 64, 8, 2, 4)
    q, k = torch.zeros((4, 4, 64), device="cuda").bfloat16(), torch.zeros((4, 2, 64), device="cuda").bfloat16()
    ok = dict(batch=2)
    for bad in (dict(batch=3), dict(mask=torch.zeros((4, 1), device="cuda")), dict(mask=torch.zeros((3, 1), dtype=torch.int32, device="cuda")), dict(seqs=torch.zeros(2, device="cuda")),
                dict(seqs=torch.zeros(2, dtype=torch.int32)), dict(row_offsets=_ints(torch, [0, 2, 4])), dict(out=torch.zeros((4, 4, 64), device="cuda"))):
        with pytest.raises(SpecError):
            dev.attention(0, q, k, k, **{**ok, **bad})
    for args in ((q, k, k.float()), (q, k[:3], k), (q[..., :32], k, k), (q, q, q), (q.cpu(), k, k), (q.double(), k.double(), k.double()), (q[:, :3], k, k), (q.transpose(1, 2).contiguous().transpose(1, 2), k, k)):
        with pytest.raises(SpecError):
            dev.attention(0, *args, **ok)
    with pytest.raises(SpecError):
        dev.attention(2, q, k, k, **ok)
    with pytest.raises(SpecError):
        dev.store(k[None], k[None], torch.zeros(2, dtype=torch.int64, device="cuda"))
    with pytest.raises(SpecError):
        dev.store(k[None].expand(3, -1, -1, -1), k[None].expand(3, -1, -1, -1), _ints(torch, [1, 1]))
    with pytest.raises(SpecError):
        dev.read(None, 4, dtype=torch.float64)
    with pytest.raises(SpecError):
        dev.fork(_ints(torch, [0, 1]), _ints(torch, [1]))
    for bad in (dict(head_dim=80), dict(fmt="int4"), dict(n_pages=0)):
        with pytest.raises(SpecError):
            SpecCache(**{**dict(n_layers=1, n_kv_heads=1, head_dim=64, n_pages=4, max_seqs=1, pages_per_seq=4), **bad})
    with pytest.raises(SpecError):
        SpecCache.from_tensors(dev.codes, dev.scales, dev.page_table.long(), dev.refs, dev.lens)
    table = spec_rotary_table(8, 64, 1e4)
    for args in ((q, k, k, _ints(torch, [0, 1, 2]), table), (q, k, k.float(), _ints(torch, [0] * 4), table), (q, k, k, _ints(torch, [0] * 4), table.double()), (q.double(), k.double(), None, _ints(torch, [0] * 4), table)):
        with pytest.raises(SpecError):
            spec_rotary(*args)
