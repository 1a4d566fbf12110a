"""Several tokens per sequence (kvq_rope_append, kvq_chunk_attention, kvq_window_attention) against plain implementations in 64 bits.

Appends are held byte for byte to the CPU oracle, which is given the keys rotated in binary32, one rounding per operation.

Attention is held to the formula in binary64 over the rows that kvq_dequantize returns, element by element, within

    (3 r + 2 delta) * sum_t p_t |V^_t|  +  r / 2 * sum_t p_t (V^_t - min V^_t)  +  r 2^-13 * sum_t |V^_t| / l  +  half a step of the output type,

l = sum_t p_t / p_max, with r = 2^-11 for 16-bit outputs and 2^-21 for binary32 ones.  16-bit outputs: the kernels round every reconstructed value (or its weight,
scale included) and every weight once to binary16, half a step 2^-11 of it each, and the weights' sum may follow the rounded weights or not
(numerator and denominator: one more).  Binary32 outputs: weights and values travel as two binary16 parts, so that 2^-22 of each is lost, and the
products are summed in binary32.  A weight that is rounded with its scale meets the code: the error is relative to p_t scale code, not to V^_t, which
is zero + scale code and may be much smaller where the two cancel.  scale code = V^_t less the least V^ of its token and group, whose code is 0; the
rounded product p_t scale is off by half a step, r / 2 of it.  Weights far below a row's largest fall among binary16's subnormals: their step there is 2^-24 of a largest weight of
at least 2^8, as are the steps of second parts.  delta is what the logits may be off by: 130 binary32 additions and the roundings of scale and
exponent, 2^-24 each, of sums whose terms are bounded by sum_d |q_d| times the greatest |K^| (twice: codes and zeros are summed apart).
"""
import math

import numpy as np
import pytest
import torch

from paper_2502_15075_amd import synth

pytestmark = pytest.mark.gpu

SIGNS = (0x9E3779B9, 0x7F4A7C15, 0xF39CC060, 0x5CEDC834)
SIGNS_V = (0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344)
SCALE = 1 / math.sqrt(128)
HALF_STEP = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}


@pytest.fixture(scope="module")
def kvq():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2502_15075_amd import kvq as m
    m.load()
    return m


def _layout(kvq, B, H, T, bk=4, bv=2, gk=64, gv=64, dtype=torch.float16, page=0, rot=0, rotv=0):
    pages = (T + page - 1) // page if page else 0
    return kvq.Layout(B, H, T, 128, bk, bv, gk, gv, raw_dtype=kvq.KVQ_BF16 if dtype == torch.bfloat16 else kvq.KVQ_F16, rotate_k=rot,
                      signs_k=SIGNS if rot else (0, 0, 0, 0), rotate_v=rotv, signs_v=SIGNS_V if rotv else (0, 0, 0, 0),
                      page_tokens=page, n_pages=B * pages + 3 if page else 0)


def _cache(kvq, L, fill, seed=0):
    cache = kvq.Cache(L, fill=fill)
    if L.page_tokens:
        pages = (L.max_seq + L.page_tokens - 1) // L.page_tokens
        perm = torch.randperm(L.n_pages, generator=torch.Generator().manual_seed(seed))[:L.batch * pages]
        cache.page_table = perm.to(torch.int32).view(L.batch, pages).cuda()
    return cache


def _filled(kvq, L, dtype, seed, heads, lens=None, fill=0xFF, **recipe):
    """A cache whose sequence b holds lens[b] tokens; every other byte is `fill` (0xFF: NaN scales and zeros)."""
    T = L.max_seq
    K, V, _ = synth.make_kvq(seed, L.batch, L.kv_heads, heads, T, dtype=dtype, **{"sigma_k": 2.0, "outlier_scale": 8.0, **recipe})
    cache = _cache(kvq, L, fill, seed)
    rows = _rows_appender(kvq, L, cache)
    for b in range(L.batch):
        rows(b, K[b], V[b], T if lens is None else lens[b])
    return cache


def _rows_appender(kvq, L, cache):
    """Appends n tokens to one sequence through quantize_append (a layout of batch 1 over that sequence's share)."""
    from dataclasses import replace
    L1 = replace(L, batch=1)

    def go(b, K, V, n):
        if n == 0:
            return
        if L.page_tokens:
            sub = kvq.Cache.__new__(kvq.Cache)
            sub.layout, sub.planes = L1, cache.planes
            sub.v_scale_exp = cache.v_scale_exp.view(L.batch, -1)[b]
            sub.page_table = cache.page_table[b:b + 1]
        else:
            sub = cache.batch_element(b, L1)
        kvq.quantize_append(L1, sub, K[None, :, :n].cuda(), V[None, :, :n].cuda(), 0)
    return go


def _dequantized(kvq, L, cache, T):
    k = torch.empty(L.batch, L.kv_heads, T, 128, dtype=torch.float32, device="cuda")
    v = torch.empty_like(k)
    kvq.dequantize(L, cache, 0, T, k, v)
    return k.double(), v.double()


def _reference(kvq, oracle, L, cache, q, q_lens, seq_lens, window, sinks, scale, out_dtype):
    """out and its tolerance, binary64, [B, n_q, H_q, 128]; rows behind q_lens are NaN."""
    B, n_q, Hq, _ = q.shape
    R = Hq // L.kv_heads
    T = max(1, max(seq_lens))
    K, V = _dequantized(kvq, L, cache, T)
    groups = V.view(*V.shape[:3], -1, L.group_v)
    lift = (groups - groups.amin(-1, keepdim=True)).reshape(V.shape) if L.bits_v != 16 else torch.zeros_like(V)
    qd = q.double().cuda()
    if L.rotate_k:                                     # the library's rotated query is rounded to binary16
        x = q.float().cpu().numpy().reshape(-1, 128)
        x = np.stack([oracle.unrotate(oracle.rotate(r, SIGNS).astype(np.float16).astype(np.float32), SIGNS) for r in x])
        qd = torch.from_numpy(x).double().view(q.shape).cuda()
    want = torch.full(q.shape, float("nan"), dtype=torch.float64, device="cuda")
    tol = torch.zeros_like(want)
    for b in range(B):
        n, length = q_lens[b], seq_lens[b]
        p = torch.arange(length - n, length, device="cuda")[:, None]
        t = torch.arange(length, device="cuda")[None]
        seen = t <= p
        if window:
            seen = seen & ((t > p - window) | (t < sinks))
        for h in range(L.kv_heads):
            k, v = K[b, h, :length], V[b, h, :length]
            for hq in range(h * R, (h + 1) * R):
                x = qd[b, :n, hq]
                if n == 0:
                    continue
                if length == 0:
                    want[b, :n, hq] = 0
                    continue
                s = (x @ k.t() * scale).masked_fill(~seen, -math.inf)
                top = s.amax(-1, keepdim=True)
                w = torch.where(seen, torch.exp(s - torch.where(top == -math.inf, torch.zeros_like(top), top)), torch.zeros_like(s))
                l = w.sum(-1, keepdim=True)
                l = torch.where(l == 0, torch.ones_like(l), l)
                want[b, :n, hq] = w @ v / l
                mag = w @ v.abs() / l
                delta = 2 * 132 * 2.0 ** -24 * scale * x.abs().sum(-1, keepdim=True) * k.abs().amax() / 2
                r = 2.0 ** -21 if out_dtype == torch.float32 else 2.0 ** -11
                tol[b, :n, hq] = (3 * r + 2 * delta) * mag + r / 2 * (w @ lift[b, h, :length] / l) + r * 2.0 ** -13 * (seen.double() @ v.abs()) / l
    tol += HALF_STEP[out_dtype] * want.abs().nan_to_num()
    return want, tol


def _assert_close(got, want, tol, what=""):
    got = got.double()
    live = ~want.isnan()
    assert bool(got[live].isfinite().all()), what
    over = ((got - want).abs() - tol)[live]
    assert bool((over <= 1e-30).all()), f"{what}: {int((over > 1e-30).sum())} of {over.numel()} off, worst {float(((got - want).abs() / tol)[live].max()):.2f} times the tolerance"


def _run_chunk(kvq, L, cache, q, q_lens, seq_lens, window, sinks, scale=SCALE, out_dtype=torch.float32, workspace=True, bound=None):
    B, n, Hq, _ = q.shape
    bound = L.max_seq if bound is None else bound
    out = torch.full(q.shape, 7.0, dtype=out_dtype, device="cuda")
    need = kvq.chunk_workspace_bytes(L, Hq, n, bound, window, sinks)
    ws = torch.full((max(16, need),), 0xFF, dtype=torch.uint8, device="cuda") if workspace else None
    ints = lambda x: None if x is None else torch.tensor(x, dtype=torch.int32, device="cuda")
    kvq.chunk_attention(L, cache, q.cuda(), ints(q_lens), ints(seq_lens), bound, window, sinks, scale, out, ws)
    torch.cuda.synchronize()
    return out


def _queries(seed, B, n, Hq, dtype):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(B, n, Hq, 128, generator=g).to(dtype)


# ---------------------------------------------------------------------------------------------------------------- rope_append

def _tables(rows, rotary):
    freq = 500000.0 ** (-torch.arange(0, rotary, 2, dtype=torch.float64) / rotary)
    angle = torch.arange(rows, dtype=torch.float64)[:, None] * freq
    return angle.cos().float(), angle.sin().float()


def _turned(x, cos, sin, rotary, interleaved):
    """x [..., n, 128] binary32; cos, sin [n, rotary / 2]; every operation rounded once."""
    x = x.clone()
    a, b = (x[..., 0:rotary:2], x[..., 1:rotary:2]) if interleaved else (x[..., :rotary // 2], x[..., rotary // 2:rotary])
    ra, rb = a * cos - b * sin, b * cos + a * sin
    if interleaved:
        x[..., 0:rotary:2], x[..., 1:rotary:2] = ra, rb
    else:
        x[..., :rotary // 2], x[..., rotary // 2:rotary] = ra, rb
    return x


def _oracle_append(oracle, L, planes, k, v, pos, dtype):
    """k [1, H, n, 128] binary32 (rotated), v of `dtype`: the four planes of a batch of one, through the oracle."""
    from dataclasses import replace
    bf = dtype == torch.bfloat16
    vf = v.float().numpy()
    k16 = synth.to_numpy_bits(k.to(dtype))
    v16 = synth.to_numpy_bits(v)
    part = lambda L1, src, kk, vv: oracle.quantize_append(L1, src, np.ascontiguousarray(kk), np.ascontiguousarray(vv), pos, bf16=bf)
    # (the oracle takes one type for both: each tensor in a call of its own, beside a quantized stand-in)
    if L.bits_k == 16:
        side = oracle.new_planes(replace(L, bits_v=8))
        part(replace(L, bits_v=8), [planes[0], planes[1], side[2], side[3]], k16, v16)
    else:
        side = oracle.new_planes(replace(L, bits_v=8))
        part(replace(L, bits_v=8), [planes[0], planes[1], side[2], side[3]], k.numpy(), vf)
    Lv = replace(L, bits_k=8, rotate_k=0)
    side = oracle.new_planes(Lv)
    part(Lv, [side[0], side[1], planes[2], planes[3]], v16, v16)


def _check_rope(kvq, oracle, bits=(4, 2), groups=(64, 64), dtype=torch.bfloat16, page=0, rot=(0, 0), rotary=128, interleaved=False, H=2,
                R=3, T=200, n=70, pos=(0, 31, 5, 130, 64), counts=(70, 1, 0, 70, 33), rows=None, with_q=True, in_place=False, strided=True):
    B = len(pos)
    rows = T if rows is None else rows
    L = _layout(kvq, B, H, T, *bits, *groups, dtype=dtype, page=page, rot=rot[0], rotv=rot[1])
    cache = _cache(kvq, L, 0xA5, 3)
    g = torch.Generator().manual_seed(11)
    big = torch.randn(B, n, (R + 2) * H + 1, 128, generator=g)           # one projection's output: q, k, v heads side by side
    big[..., R * H:(R + 1) * H, :] *= 2.0
    big[..., R * H:(R + 1) * H, [5, 37, 69, 101]] *= 8.0
    big = big.to(dtype)
    q, k, v = big[..., :R * H, :], big[..., R * H:(R + 1) * H, :].transpose(1, 2), big[..., (R + 1) * H:(R + 2) * H, :].transpose(1, 2)
    cos, sin = _tables(rows, rotary)
    dev = big.cuda()
    qd, kd, vd = dev[..., :R * H, :], dev[..., R * H:(R + 1) * H, :].transpose(1, 2), dev[..., (R + 1) * H:(R + 2) * H, :].transpose(1, 2)
    if not strided:
        qd, kd, vd = qd.contiguous(), kd.contiguous(), vd.contiguous()
    q_out = qd.contiguous() if in_place else torch.full((B, n, R * H, 128), 7.0, dtype=dtype, device="cuda")
    src = q_out if in_place else qd
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    got = kvq.rope_append(L, cache, src if with_q else None, kd, vd, ints(pos), kvq.Rope(cos.cuda(), sin.cuda(), interleaved),
                          q_out if with_q else None, n_tokens=None if counts is None else ints(counts))
    torch.cuda.synchronize()
    # the planes a sequence at a time
    planes = [p.cpu().numpy() if p is not None else np.zeros(0, np.uint8) for p in cache.planes[:4]]
    Lo = oracle.Layout(1, H, T if not page else (T + page - 1) // page * page, 128, *bits, *groups, raw_dtype=L.raw_dtype, rotate_k=rot[0],
                       signs_k=L.signs_k, rotate_v=rot[1], signs_v=L.signs_v)
    table = cache.page_table.cpu().numpy() if page else None
    if page:
        from dataclasses import replace
        flat = oracle.gather_pages(replace(Lo, batch=B), planes, table, page, L.n_pages)
        used = np.zeros(L.n_pages, bool)
        used[table.reshape(-1)] = True
        for p in planes:                                                  # pages of no sequence stay as they are
            if p.size:
                assert (p.reshape(L.n_pages, -1)[~used] == 0xA5).all()
    else:
        flat = planes
    want_q = (q_out.new_full(q_out.shape, 7.0) if not in_place else qd.contiguous()).cpu()
    for b in range(B):
        ref = oracle.new_planes(Lo, fill=0xA5)
        c = n if counts is None else min(max(counts[b], 0), n)
        first = max(0, -pos[b])
        c = min(c, min(T, rows) - pos[b])
        if c > first:
            at = pos[b] + first
            tc, ts = cos[at:pos[b] + c], sin[at:pos[b] + c]
            kt = _turned(k[b:b + 1, :, first:c].float(), tc, ts, rotary, interleaved)
            _oracle_append(oracle, Lo, ref, kt, v[b:b + 1, :, first:c].contiguous(), at, dtype)
            want_q[b, first:c] = _turned(q[b, first:c].float().transpose(0, 1), tc, ts, rotary, interleaved).transpose(0, 1).to(dtype)
        for name, mine, theirs in zip(("k_codes", "k_meta", "v_codes", "v_meta"), flat, ref):
            share = mine.reshape(B, -1)[b] if mine.size else mine
            bad = np.flatnonzero(share != theirs)
            assert bad.size == 0, f"sequence {b}, {name}: {bad.size} bytes differ, first at {bad[:5]}"
    if with_q:
        assert got is q_out
        same = (got.cpu().float() == want_q.float())
        assert bool(same.all()), f"rotated queries: {int((~same).sum())} differ, first at {torch.nonzero(~same)[:3].tolist()}"


@pytest.mark.parametrize("bits", [(4, 2), (2, 4), (8, 8), (4, 4), (1, 1), (3, 3), (6, 6), (16, 16), (16, 2), (4, 16), (8, 3), (2, 6), (6, 1)])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_rope_append_is_byte_identical(kvq, oracle, bits, dtype):
    _check_rope(kvq, oracle, bits=bits, dtype=dtype)


@pytest.mark.parametrize("rotary", [16, 32, 48, 64, 96, 112, 128])
@pytest.mark.parametrize("interleaved", [False, True])
def test_rope_append_rotary_widths(kvq, oracle, rotary, interleaved):
    _check_rope(kvq, oracle, rotary=rotary, interleaved=interleaved, groups=(32, 128))


@pytest.mark.parametrize("page", [64, 128])
@pytest.mark.parametrize("groups", [(32, 32), (128, 64)])
def test_rope_append_paged(kvq, oracle, page, groups):
    _check_rope(kvq, oracle, page=page, groups=groups)


@pytest.mark.parametrize("bits", [(4, 2), (8, 8), (1, 1), (3, 3), (6, 6), (16, 16), (2, 4)])
@pytest.mark.parametrize("R", [1, 4, 8])
@pytest.mark.parametrize("page", [0, 64])
def test_rope_append_single_token(kvq, oracle, bits, R, page):
    """The form of a decode loop: one token per sequence, among them one left out, one beyond the capacity and a negative position."""
    _check_rope(kvq, oracle, bits=bits, R=R, page=page, n=1, pos=(0, 31, 32, 199, 77, 200, -1), counts=(1, 1, 1, 1, 0, 1, 1))
    _check_rope(kvq, oracle, bits=bits, R=R, page=page, n=1, pos=(0, 31, 32, 199, 77), counts=None, interleaved=True, rotary=64)


@pytest.mark.parametrize("kw", [dict(rot=(1, 0)), dict(rot=(1, 1)), dict(with_q=False), dict(in_place=True), dict(strided=False),
                                dict(rows=150), dict(pos=(-3, 199, 200, 190, 1 << 30), counts=(70, 70, 70, 70, 70)), dict(counts=(-5, 1000, 70, 69, 2)),
                                dict(H=1, R=1, pos=(17,), counts=None), dict(n=2, counts=(2, 1, 0, 2, 2))])
def test_rope_append_variants(kvq, oracle, kw):
    _check_rope(kvq, oracle, **kw)


def test_rope_append_many_blocks(kvq, oracle):
    """Enough blocks for every shape of the launch."""
    _check_rope(kvq, oracle, T=3000, n=2901, pos=(3, 64), counts=(2901, 1777), H=8, R=4)


def test_rope_append_raises_the_value_scale_exponents(kvq):
    L = _layout(kvq, 2, 2, 64, 4, 2)
    for n in (1, 5):
        cache = kvq.Cache(L, fill=0)
        k = torch.zeros(2, 2, n, 128, dtype=torch.float16, device="cuda")
        v = torch.zeros_like(k)
        v[1, 0, 0, 3] = 60000.0                        # a group range of 60000 in 3 steps: scale 20000, exponent field 29
        cos, sin = _tables(64, 128)
        kvq.rope_append(L, cache, None, k, v, torch.tensor([0, 9], dtype=torch.int32, device="cuda"), kvq.Rope(cos.cuda(), sin.cuda()))
        assert cache.v_scale_exp.view(2, 2).tolist() == [[0, 0], [29, 0]]


# ---------------------------------------------------------------------------------------------------------------- attention

FORMATS = [(4, 2, 64, 64), (4, 4, 128, 32), (2, 2, 32, 128), (8, 8, 32, 32), (8, 2, 64, 128), (2, 8, 128, 64), (16, 16, 64, 64), (1, 1, 64, 64),
           (3, 3, 32, 64), (6, 6, 64, 32), (16, 4, 64, 64), (4, 16, 64, 64), (8, 4, 128, 128), (3, 6, 128, 128), (6, 1, 128, 64)]


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_chunk_attention_formats(kvq, oracle, fmt, dtype):
    B, H, R, T, n = 3, 2, 4, 333, 37
    L = _layout(kvq, B, H, T, *fmt, dtype=dtype)
    lens = [333, 70, 37]
    cache = _filled(kvq, L, dtype, sum(fmt), H * R, lens)
    q = _queries(1, B, n, H * R, dtype)
    q_lens = [37, 37, 20]
    out = _run_chunk(kvq, L, cache, q, q_lens, lens, 0, 0)
    want, tol = _reference(kvq, oracle, L, cache, q, q_lens, lens, 0, 0, SCALE, torch.float32)
    _assert_close(out, want, tol)
    assert bool((out[2, 20:] == 7.0).all())


@pytest.mark.parametrize("R", [1, 2, 3, 4, 5, 6, 7, 8])
@pytest.mark.parametrize("n,T", [(1, 1), (1, 65), (2, 64), (3, 1000), (16, 97), (65, 130), (200, 200)])
def test_chunk_attention_rows_and_lengths(kvq, oracle, R, n, T):
    L = _layout(kvq, 2, 3, T, 4, 2, page=64 if R % 2 else 0)
    lens = [T, max(1, T - 1)]
    cache = _filled(kvq, L, torch.float16, R, 3 * R, lens)
    q = _queries(2, 2, n, 3 * R, torch.float16)
    out = _run_chunk(kvq, L, cache, q, None, lens, 0, 0, out_dtype=torch.bfloat16)
    want, tol = _reference(kvq, oracle, L, cache, q, [n, n], lens, 0, 0, SCALE, torch.bfloat16)
    _assert_close(out, want, tol)


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (7, 3), (32, 0), (33, 64), (64, 4), (100, 65), (129, 130), (500, 4), (1000, 7), (0, 9)])
@pytest.mark.parametrize("n", [1, 5, 90])
def test_chunk_attention_windows(kvq, oracle, window, sinks, n):
    L = _layout(kvq, 4, 1, 700, 4, 4, page=128)
    lens = [700, 641, 90, 95]
    cache = _filled(kvq, L, torch.bfloat16, 5, 8, lens)
    q = _queries(3, 4, n, 8, torch.bfloat16)
    out = _run_chunk(kvq, L, cache, q, None, lens, window, sinks, out_dtype=torch.float16)
    want, tol = _reference(kvq, oracle, L, cache, q, [n] * 4, lens, window, sinks, SCALE, torch.float16)
    _assert_close(out, want, tol)


@pytest.mark.parametrize("rot", [(1, 0), (1, 1), (0, 1)])
@pytest.mark.parametrize("T,n", [(200, 50), (3001, 3)])
def test_chunk_attention_rotated_basis(kvq, oracle, rot, T, n):
    """The queries of a layout with rotated keys, outputs taken back from rotated values, from one part and from many."""
    L = _layout(kvq, 1, 2, T, 4, 4, rot=rot[0], rotv=rot[1])
    cache = _filled(kvq, L, torch.float16, 8, 8)
    q = _queries(4, 1, n, 8, torch.float16)
    out = _run_chunk(kvq, L, cache, q, None, None, 0, 0)
    want, tol = _reference(kvq, oracle, L, cache, q, [n], [T], 0, 0, SCALE, torch.float32)
    if rot[1]:                                         # weights and values are rounded in the rotated basis: a channel gets 1/sqrt(128) of all 128 errors
        tol = tol.norm(dim=-1, keepdim=True).expand_as(tol)
    _assert_close(out, want, tol)


def test_chunk_attention_rows_that_see_nothing(kvq, oracle):
    """Empty sequences, more query tokens than cached ones, no query tokens: zeros where nothing is seen, untouched rows elsewhere.  The
    caches hold NaN scales and zeros everywhere else."""
    L = _layout(kvq, 5, 2, 100, 4, 2)
    lens, q_lens = [0, 3, 100, 64, 0], [6, 6, 0, 6, 0]
    cache = _filled(kvq, L, torch.float16, 6, 4, lens)
    q = _queries(5, 5, 6, 4, torch.float16)
    for window, sinks in ((0, 0), (2, 1)):
        out = _run_chunk(kvq, L, cache, q, q_lens, lens, window, sinks)
        want, tol = _reference(kvq, oracle, L, cache, q, q_lens, lens, window, sinks, SCALE, torch.float32)
        _assert_close(out, want, tol)
        assert bool((out[0] == 0).all()) and bool((out[1, :3] == 0).all()) and bool((out[2] == 7.0).all()) and bool((out[4] == 7.0).all())


def test_device_values_are_clamped(kvq, oracle):
    L = _layout(kvq, 3, 2, 100, 4, 2)
    cache = _filled(kvq, L, torch.float16, 7, 4)
    q = _queries(6, 3, 5, 4, torch.float16)
    out = _run_chunk(kvq, L, cache, q, [9, -2, 5], [1 << 30, 50, -7], 0, 0)
    want, tol = _reference(kvq, oracle, L, cache, q, [5, 0, 5], [100, 50, 0], 0, 0, SCALE, torch.float32)
    _assert_close(out, want, tol)
    assert bool((out[1] == 7.0).all())


@pytest.mark.parametrize("T,n,Hq,H,fmt", [(5000, 1, 8, 1, (4, 2, 64, 64)), (20000, 4, 8, 1, (8, 8, 32, 32)), (9000, 17, 4, 2, (2, 4, 128, 64)),
                                          (4097, 1, 3, 3, (16, 16, 64, 64))])
def test_parts_of_a_long_sequence(kvq, oracle, T, n, Hq, H, fmt):
    """Few rows, many tokens: cut into parts; less workspace means fewer parts and the same answer."""
    L = _layout(kvq, 1, H, T, *fmt)
    cache = _filled(kvq, L, torch.float16, 9, Hq)
    q = _queries(7, 1, n, Hq, torch.float16)
    want, tol = _reference(kvq, oracle, L, cache, q, [n], [T], 0, 0, SCALE, torch.float32)
    assert kvq.chunk_workspace_bytes(L, Hq, n, T) > 0
    for workspace in (True, False):
        _assert_close(_run_chunk(kvq, L, cache, q, None, None, 0, 0, workspace=workspace), want, tol, f"workspace {workspace}")


@pytest.mark.parametrize("factor", [1e-3, 1.0, 300.0])
def test_queries_of_other_magnitudes(kvq, oracle, factor):
    """Tiny queries; and ones so large (up to the type's bound) that a group's sum leaves binary16."""
    L = _layout(kvq, 1, 1, 300, 8, 8, 32, 32)
    cache = _filled(kvq, L, torch.float16, 10, 8)
    q = (_queries(8, 1, 9, 8, torch.float32) * factor).abs().half()
    if factor > 100:
        q[0, 0, 0] = 65504.0
    scale = SCALE / max(1.0, factor)
    out = _run_chunk(kvq, L, cache, q, None, None, 0, 0, scale=scale)
    want, tol = _reference(kvq, oracle, L, cache, q, [9], [300], 0, 0, scale, torch.float32)
    _assert_close(out, want, tol)


@pytest.mark.parametrize("fmt", [(4, 2, 64, 64), (8, 8, 32, 32), (16, 16, 64, 64), (2, 1, 128, 128)])
@pytest.mark.parametrize("n", [1, 40])
def test_large_values(kvq, oracle, fmt, n):
    """Values over the whole range of binary16: reconstructions next to its end, scales of thousands."""
    L = _layout(kvq, 1, 2, 200, *fmt)
    g = torch.Generator().manual_seed(12)
    K = torch.randn(1, 2, 200, 128, generator=g).half()
    V = (torch.rand(1, 2, 200, 128, generator=g) * 2 - 1).mul(65504.0).half()
    V[..., 0], V[..., 1] = 65504.0, -65504.0
    cache = _cache(kvq, L, 0xFF)
    kvq.quantize_append(L, cache, K.cuda(), V.cuda(), 0)
    q = _queries(9, 1, n, 4, torch.float16)
    out = _run_chunk(kvq, L, cache, q, None, None, 0, 0)
    want, tol = _reference(kvq, oracle, L, cache, q, [n], [200], 0, 0, SCALE, torch.float32)
    _assert_close(out, want, tol)


def test_strided_queries(kvq, oracle):
    """Queries as a slice of a projection's output, heads and tokens in another order."""
    L = _layout(kvq, 2, 2, 150)
    cache = _filled(kvq, L, torch.bfloat16, 11, 6)
    big = _queries(10, 2, 7, 10, torch.bfloat16).cuda()
    q = big[:, :, 2:8]
    want, tol = _reference(kvq, oracle, L, cache, q.cpu(), [7, 7], [150, 150], 0, 0, SCALE, torch.float32)
    _assert_close(_run_chunk(kvq, L, cache, q, None, None, 0, 0), want, tol)
    swapped = q.transpose(1, 2).contiguous().transpose(1, 2)
    _assert_close(_run_chunk(kvq, L, cache, swapped, None, None, 0, 0), want, tol)


# Calls of many rows run as tiles of 256 rows (widths 2, 4 and 8) or 128: 200 query tokens of 8 query heads in 16 streams are several times the
# workgroups of the kernel for few rows that the device takes at once.

TILE_FORMATS = [(k, v, *g) for (k, v), g in zip([(k, v) for k in (2, 4, 8) for v in (2, 4, 8)],
                                                [(32, 64), (64, 32), (128, 128), (64, 64), (32, 32), (128, 64), (64, 128), (128, 32), (32, 128)])]
TILE_FORMATS += [(1, 1, 64, 64), (3, 6, 32, 128), (6, 3, 64, 32), (16, 16, 64, 64), (16, 4, 64, 32), (2, 16, 32, 64), (8, 1, 128, 64), (1, 8, 64, 32)]


@pytest.mark.parametrize("fmt", TILE_FORMATS)
@pytest.mark.parametrize("out_dtype", [torch.float32, torch.float16, torch.bfloat16])
def test_row_tiles_formats(kvq, oracle, fmt, out_dtype):
    B, H, R, T, n = 4, 4, 8, 333, 200
    page = 64 * (fmt[0] % 3)
    dtype = torch.float16 if out_dtype == torch.float16 else torch.bfloat16
    L = _layout(kvq, B, H, T, *fmt, dtype=dtype, page=page)
    lens, q_lens = [333, 200, 130, 257], [200, 200, 63, 1]
    cache = _filled(kvq, L, dtype, sum(fmt), H * R, lens)
    q = _queries(51, B, n, H * R, dtype)
    out = _run_chunk(kvq, L, cache, q, q_lens, lens, 0, 0, out_dtype=out_dtype)
    want, tol = _reference(kvq, oracle, L, cache, q, q_lens, lens, 0, 0, SCALE, out_dtype)
    _assert_close(out, want, tol)
    assert bool((out[2, 63:] == 7.0).all()) and bool((out[3, 1:] == 7.0).all())


@pytest.mark.parametrize("window,sinks", [(1, 0), (7, 3), (32, 0), (64, 4), (129, 130), (200, 1), (0, 9), (1000, 70)])
@pytest.mark.parametrize("R", [3, 8])
@pytest.mark.parametrize("bits", [(4, 4), (6, 6)])
def test_row_tiles_windows(kvq, oracle, window, sinks, R, bits):
    B, H, T, n = 4, 4, 500, 480 if R == 3 else 220
    L = _layout(kvq, B, H, T, *bits, page=128)
    lens = [500, 333, n, n - 37]                          # (the last one: rows that see nothing)
    cache = _filled(kvq, L, torch.float16, 52, H * R, lens)
    q = _queries(53, B, n, H * R, torch.float16)
    out = _run_chunk(kvq, L, cache, q, None, lens, window, sinks)
    want, tol = _reference(kvq, oracle, L, cache, q, [n] * B, lens, window, sinks, SCALE, torch.float32)
    _assert_close(out, want, tol)
    assert bool((out[3, :37] == 0).all())


@pytest.mark.parametrize("rot", [(1, 0), (1, 1), (0, 1)])
@pytest.mark.parametrize("fmt", [(4, 4, 64, 64), (8, 2, 32, 128), (3, 3, 64, 64)])
def test_row_tiles_rotated_basis(kvq, oracle, rot, fmt):
    B, H, R, T, n = 4, 4, 8, 250, 200
    L = _layout(kvq, B, H, T, *fmt, rot=rot[0], rotv=rot[1])
    cache = _filled(kvq, L, torch.float16, 54, H * R)
    q = _queries(55, B, n, H * R, torch.float16)
    out = _run_chunk(kvq, L, cache, q, None, None, 0, 0)
    want, tol = _reference(kvq, oracle, L, cache, q, [n] * B, [T] * B, 0, 0, SCALE, torch.float32)
    if rot[1]:                                         # (as in test_chunk_attention_rotated_basis)
        tol = tol.norm(dim=-1, keepdim=True).expand_as(tol)
    _assert_close(out, want, tol)


@pytest.mark.parametrize("fmt", [(4, 2, 64, 64), (8, 8, 32, 32), (3, 3, 64, 64)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (2500, 70)])
def test_row_tiles_in_parts(kvq, oracle, fmt, window, sinks):
    """Many rows of few sequences: parts, joined by a launch of their own; query tokens of sequences of different lengths see different
    numbers of parts, some rows none of them and some a single one."""
    B, H, R, T, n = 3, 1, 8, 6000, 700
    L = _layout(kvq, B, H, T, *fmt)
    lens, q_lens = [6000, 800, 120], [700, 700, 130]
    cache = _filled(kvq, L, torch.bfloat16, 56, H * R, lens)
    q = _queries(57, B, n, H * R, torch.bfloat16)
    want, tol = _reference(kvq, oracle, L, cache, q, q_lens, lens, window, sinks, SCALE, torch.bfloat16)
    for workspace in (True, False):
        out = _run_chunk(kvq, L, cache, q, q_lens, lens, window, sinks, out_dtype=torch.bfloat16, workspace=workspace)
        _assert_close(out, want, tol, f"workspace {workspace}")
        assert bool((out[2, 130:] == 7.0).all())


def test_row_tiles_scores_that_climb(kvq, oracle):
    """Each later token scores higher, by far more than a weight may hold: the running maximum is raised again and again.  And one sequence
    whose first token is the largest by as much."""
    B, H, R, T, n = 4, 4, 8, 400, 200
    L = _layout(kvq, B, H, T, 8, 4)
    g = torch.Generator().manual_seed(58)
    K = torch.randn(B, H, T, 128, generator=g)
    K[:, :, :, 0] = torch.arange(T) * 0.5
    K[1] = K[1].flip(1)
    V = torch.randn(B, H, T, 128, generator=g)
    cache = _cache(kvq, L, 0xFF)
    kvq.quantize_append(L, cache, K.half().cuda(), V.half().cuda(), 0)
    q = _queries(59, B, n, H * R, torch.float16)
    q[..., 0] = 12.0
    for out_dtype in (torch.float32, torch.float16):
        out = _run_chunk(kvq, L, cache, q, None, None, 0, 0, out_dtype=out_dtype)
        want, tol = _reference(kvq, oracle, L, cache, q, [n] * B, [T] * B, 0, 0, SCALE, out_dtype)
        _assert_close(out, want, tol)


@pytest.mark.parametrize("fmt", [(4, 2, 64, 64), (8, 8, 32, 32), (16, 16, 64, 64), (6, 3, 64, 32), (4, 16, 64, 64)])
@pytest.mark.parametrize("B,H,R,n", [(1, 1, 4, 1), (3, 2, 8, 6), (4, 4, 8, 200)])
def test_tokens_that_no_query_sees_need_be_no_numbers(kvq, fmt, B, H, R, n):
    """NaN and infinite tokens between the sinks and the oldest window, in the blocks where those begin and end: not a bit changes."""
    T, window, sinks = 500, 101, 5
    L = _layout(kvq, B, H, T, *fmt)
    g = torch.Generator().manual_seed(60)
    K, V = (torch.randn(B, H, T, 128, generator=g).half() for _ in range(2))
    q = _queries(61, B, n, H * R, torch.float16)
    outs = []
    for bad in (None, float("nan"), float("inf")):
        k, v = K.clone(), V.clone()
        if bad is not None:
            k[:, :, sinks:T - n - window + 1], v[:, :, sinks:T - n - window + 1] = bad, bad
        cache = _cache(kvq, L, 0xFF)
        kvq.quantize_append(L, cache, k.cuda(), v.cuda(), 0)
        cache.v_scale_exp.zero_()                         # (grows with any finite scale that was stored: no part of this)
        for out_dtype in (torch.float32, torch.float16):
            outs.append((out_dtype, _run_chunk(kvq, L, cache, q, None, None, window, sinks, out_dtype=out_dtype)))
    for dtype, out in outs:
        assert bool(out.isfinite().all())
        assert torch.equal(out, next(o for t, o in outs if t == dtype))


def test_the_largest_windows_and_sinks(kvq):
    """2^31 - 1 of either, with rows before the first token: the same as no window."""
    L = _layout(kvq, 3, 2, 200, 4, 2)
    lens = [200, 3, 0]
    cache = _filled(kvq, L, torch.float16, 62, 8, lens)
    q = _queries(63, 3, 9, 8, torch.float16)
    want = _run_chunk(kvq, L, cache, q, None, lens, 0, 0)
    huge = 2 ** 31 - 1
    for window, sinks in ((huge, 0), (huge, huge), (0, huge), (7, huge), (200, 3)):
        assert torch.equal(_run_chunk(kvq, L, cache, q, None, lens, window, sinks), want)


# ------------------------------------------------------------------------------------------------------ single tokens, a window

def _run_window(kvq, L, cache, q, seq_lens, window, sinks, out_dtype=torch.float32, bound=None, workspace=True):
    bound = L.max_seq if bound is None else bound
    out = torch.full(q.shape, 7.0, dtype=out_dtype, device="cuda")
    ws = torch.full((max(16, kvq.window_workspace_bytes(L, q.shape[1], bound, window, sinks)),), 0xFF, dtype=torch.uint8, device="cuda")
    lens = None if seq_lens is None else torch.tensor(seq_lens, dtype=torch.int32, device="cuda")
    kvq.window_attention(L, cache, q.cuda(), lens, bound, window, sinks, SCALE, out, ws if workspace else None)
    torch.cuda.synchronize()
    return out


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("R,dtype,page", [(1, torch.float16, 64), (4, torch.bfloat16, 0), (8, torch.float16, 128), (7, torch.bfloat16, 64)])
def test_window_attention_formats(kvq, oracle, fmt, R, dtype, page):
    B, H, T = 5, 2, 700
    L = _layout(kvq, B, H, T, *fmt, dtype=dtype, page=page)
    lens = [700, 1, 129, 333, 64]
    cache = _filled(kvq, L, dtype, 20 + R, H * R, lens)
    q = _queries(11, B, 1, H * R, dtype)
    want, tol = _reference(kvq, oracle, L, cache, q, [1] * B, lens, 200, 5, SCALE, torch.float32)
    _assert_close(_run_window(kvq, L, cache, q[:, 0], lens, 200, 5), want[:, 0], tol[:, 0])


@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (1, 1), (31, 4), (32, 0), (33, 33), (64, 64), (1024, 4), (4000, 100), (1 << 30, 1 << 30)])
@pytest.mark.parametrize("R", [1, 8])
def test_window_attention_windows(kvq, oracle, window, sinks, R):
    B, H, T = 6, 2, 5000
    L = _layout(kvq, B, H, T, 4, 2, page=64)
    lens = [5000, 4999, 1025, 32, 33, 0]
    cache = _filled(kvq, L, torch.float16, 30, H * R, lens)
    q = _queries(12, B, 1, H * R, torch.float16)
    want, tol = _reference(kvq, oracle, L, cache, q, [1] * B, lens, window, sinks, SCALE, torch.float16)
    for workspace in (True, False):
        out = _run_window(kvq, L, cache, q[:, 0], lens, window, sinks, torch.float16, workspace=workspace)
        _assert_close(out, want[:, 0], tol[:, 0])
        assert bool((out[5] == 0).all())


def test_a_window_over_everything_is_decode_attention(kvq):
    """Held to the decode call of the same cache: both are within 2e-3 of the oracle's figure, measured as that call's tests do."""
    B, H, R, T = 4, 8, 4, 3001
    L = _layout(kvq, B, H, T)
    cache = _filled(kvq, L, torch.float16, 31, H * R)
    q = _queries(13, B, 1, H * R, torch.float16)[:, 0].cuda()
    ws = torch.empty(max(16, kvq.decode_workspace_bytes(L, H * R, T)), dtype=torch.uint8, device="cuda")
    want = kvq.decode_attention(L, cache, q, T, SCALE, torch.empty(q.shape, dtype=torch.float32, device="cuda"), ws)
    got = _run_window(kvq, L, cache, q, None, T, 0)
    err = ((got - want).abs().amax(-1) / want.abs().amax(-1)).max()
    assert float(err) < 4e-3


# --------------------------------------------------------------------------------------------------------------- as they are used

def test_prompt_in_chunks_then_a_window_decode(kvq, oracle):
    """Two sequences of different prompts: chunks of 48 tokens appended with their positions' rotation and attended, drafted tokens
    verified, then single tokens behind a window.  Every step against the formula over the rows that the cache holds."""
    B, H, R, T, chunk = 2, 2, 4, 300, 48
    dtype = torch.bfloat16
    L = _layout(kvq, B, H, T, 4, 4, page=64, dtype=dtype)
    cache = _cache(kvq, L, 0xFF, 4)
    cos, sin = _tables(T, 128)
    rope = kvq.Rope(cos.cuda(), sin.cuda())
    g = torch.Generator().manual_seed(40)
    have, prompts = [0, 0], [131, 77]
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    steps = []
    while any(h < p for h, p in zip(have, prompts)):
        new = [min(chunk, p - h) for h, p in zip(have, prompts)]
        steps.append((chunk, new, 0, 0))
        have = [h + n for h, n in zip(have, new)]
    steps += [(5, [5, 5], 0, 0), (5, [3, 5], 40, 2)] + [(1, [1, 1], 40, 2)] * 4
    have = [0, 0]
    rows = torch.zeros(B, H, T, 128)                     # keys as the formula rotates them
    for n, new, window, sinks in steps:
        q = torch.randn(B, n, H * R, 128, generator=g).to(dtype)
        k = (2 * torch.randn(B, H, n, 128, generator=g)).to(dtype)
        v = torch.randn(B, H, n, 128, generator=g).to(dtype)
        turned = kvq.rope_append(L, cache, q.cuda(), k.cuda(), v.cuda(), ints(have), rope, n_tokens=ints(new))
        for b in range(B):
            p = slice(have[b], have[b] + new[b])
            rows[b, :, p] = _turned(k[b, :, :new[b]].float(), cos[p], sin[p], 128, False)
            turned_want = _turned(q[b, :new[b]].float().transpose(0, 1), cos[p], sin[p], 128, False).transpose(0, 1)
            assert torch.equal(turned[b, :new[b]].cpu(), turned_want.to(dtype))
        have = [h + m for h, m in zip(have, new)]
        kd, _ = _dequantized(kvq, L, cache, max(have))
        for b in range(B):                                # (4-bit groups of 64 channels: half a step of the group's range / 15, and the roundings of scale and zero)
            x = rows[b, :, :have[b]].unflatten(-1, (2, 64))
            half = (x.amax(-1) - x.amin(-1)) / 15 / 2 + x.abs().amax(-1) * 2.0 ** -9
            assert bool(((kd[b, :, :have[b]].cpu().float() - rows[b, :, :have[b]]).unflatten(-1, (2, 64)).abs().amax(-1) <= half).all())
        qt = turned.clone()
        if n == 1:
            out = _run_window(kvq, L, cache, qt[:, 0].contiguous(), have, window, sinks)[:, None]
        else:
            out = _run_chunk(kvq, L, cache, qt, new, have, window, sinks)
        want, tol = _reference(kvq, oracle, L, cache, qt.cpu(), new, have, window, sinks, SCALE, torch.float32)
        _assert_close(out, want, tol, f"{n} tokens after {have}")


def test_captured_steps_replay(kvq):
    """An append, a chunk and a window call captured into a graph; lengths and inputs change in place between the replays, and eager calls
    run between them.  Every replay equals the eager calls bit for bit."""
    B, H, R, T, n = 3, 2, 4, 2000, 6
    dtype = torch.float16
    L = _layout(kvq, B, H, T, 4, 2)
    caches = [_filled(kvq, L, dtype, 41, H * R) for _ in range(2)]
    cos, sin = _tables(T, 128)
    rope = kvq.Rope(cos.cuda(), sin.cuda())
    g = torch.Generator().manual_seed(42)
    mk = lambda *s: torch.randn(*s, generator=g).to(dtype).cuda()
    st = dict(q=mk(B, n, H * R, 128), k=mk(B, H, n, 128), v=mk(B, H, n, 128), pos=torch.zeros(B, dtype=torch.int32, device="cuda"),
              lens=torch.zeros(B, dtype=torch.int32, device="cuda"))

    def step(cache, o):
        kvq.rope_append(L, cache, st["q"], st["k"], st["v"], st["pos"], rope, o["q"])
        kvq.chunk_attention(L, cache, o["q"], None, st["lens"], T, 0, 0, SCALE, o["chunk"], o["ws"])
        kvq.window_attention(L, cache, o["last"].copy_(o["q"][:, -1]), st["lens"], T, 900, 4, SCALE, o["window"], o["ws1"])

    def outputs():
        return dict(q=torch.empty_like(st["q"]), chunk=torch.zeros(B, n, H * R, 128, device="cuda"), window=torch.zeros(B, H * R, 128, device="cuda"),
                    last=torch.empty(B, H * R, 128, dtype=dtype, device="cuda"),
                    ws=torch.empty(max(16, kvq.chunk_workspace_bytes(L, H * R, n, T)), dtype=torch.uint8, device="cuda"),
                    ws1=torch.empty(max(16, kvq.window_workspace_bytes(L, H * R, T, 900, 4)), dtype=torch.uint8, device="cuda"))
    eager, replayed = outputs(), outputs()

    def set_to(pos):
        st["pos"].copy_(torch.tensor(pos, dtype=torch.int32))
        st["lens"].copy_(torch.tensor([p + n for p in pos], dtype=torch.int32))
    set_to([0, 100, 1000])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(caches[1], replayed)
    torch.cuda.current_stream().wait_stream(side)
    step(caches[0], eager)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(caches[1], replayed)
    for i, pos in enumerate(([6, 106, 1006], [0, 1994, 31], [700, 32, 63], [5, 5, 5])):
        set_to(pos)
        st["q"].copy_(mk(B, n, H * R, 128)), st["k"].copy_(mk(B, H, n, 128)), st["v"].copy_(mk(B, H, n, 128))
        step(caches[0], eager)
        graph.replay()
        torch.cuda.synchronize()
        for name in ("q", "chunk", "window"):
            assert torch.equal(eager[name], replayed[name]), (i, name)
        for x, y in zip(caches[0].planes, caches[1].planes):
            assert x is None or torch.equal(x, y)


def test_two_streams_at_once(kvq, oracle):
    """Calls on two streams with a workspace each, on one cache."""
    L = _layout(kvq, 1, 2, 6000, 4, 2)
    cache = _filled(kvq, L, torch.float16, 43, 8)
    q = _queries(44, 1, 4, 8, torch.float16)
    want, tol = _reference(kvq, oracle, L, cache, q, [4], [6000], 0, 0, SCALE, torch.float32)
    qd = q.cuda()
    outs, spaces = [], []
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for s in streams:
        with torch.cuda.stream(s):
            out = torch.zeros(1, 4, 8, 128, device="cuda")
            ws = torch.empty(kvq.chunk_workspace_bytes(L, 8, 4, 6000), dtype=torch.uint8, device="cuda")
            for _ in range(3):
                kvq.chunk_attention(L, cache, qd, None, None, 6000, 0, 0, SCALE, out, ws)
        outs.append(out), spaces.append(ws)
    torch.cuda.synchronize()
    for out in outs:
        _assert_close(out, want, tol)
    assert torch.equal(outs[0], outs[1])


def test_offsets_beyond_32_bits(kvq, oracle):
    """The last sequence of planes of more than 4 GiB."""
    B, H, R, T = 5, 8, 2, 1 << 20
    L = _layout(kvq, B, H, T, 8, 8, 128, 128)
    assert kvq.cache_bytes(L)[0] >= 5 << 30
    cache = kvq.Cache(L)
    n, pos = 40, [5, 0, 7, 1, T - 40]
    g = torch.Generator().manual_seed(45)
    k, v = torch.randn(B, H, n, 128, generator=g).half(), torch.randn(B, H, n, 128, generator=g).half()
    cos, sin = _tables(64, 128)
    cos, sin = cos[:1].expand(T, -1).contiguous().cuda(), sin[:1].expand(T, -1).contiguous().cuda()      # (angle 0 everywhere)
    kvq.rope_append(L, cache, None, k.cuda(), v.cuda(), torch.tensor(pos, dtype=torch.int32, device="cuda"), kvq.Rope(cos, sin))
    kd, vd = torch.empty(B, H, n, 128, device="cuda"), torch.empty(B, H, n, 128, device="cuda")
    kvq.dequantize(L, cache, T - n, T, kd, vd)
    assert float((kd[4].cpu() - k[4].float()).abs().max()) < 0.02 and float((vd[4].cpu() - v[4].float()).abs().max()) < 0.02
    q = _queries(46, B, 3, H * R, torch.float16)
    lens = [0, 0, 0, 0, T]
    out = _run_chunk(kvq, L, cache, q, None, lens, 30, 0)
    x, keys, values = q[4].double().cuda(), kd[4].double(), vd[4].double()
    for i in range(3):
        seen = slice(n - 3 + i - 29, n - 3 + i + 1)
        for hq in range(H * R):
            w = torch.softmax(keys[hq // R, seen] @ x[i, hq] * SCALE, 0)
            got, want = out[4, i, hq].double(), w @ values[hq // R, seen]
            assert bool(((got - want).abs() <= 4 * 2.0 ** -11 * (w @ values[hq // R, seen].abs())).all())
