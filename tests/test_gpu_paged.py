"""The paged 8-bit cache against plain implementations (paged_reference.py): codes and tables exactly, attention against 64 bits.

Tolerances, derived from the arithmetic.  Scores: codes are exact in fp16, q enters as two fp16 terms (relative 2^-22), products are
exact and every sum is fp32 on the tensor core, which truncates: at most (d / 16 + 1) steps of 2^-23 of a partial sum, so below 1.1e-6 of the
largest partial sum and 1e-6 of the row's RMS in RMS; the aligner's sums (three bf16 terms, 2^-24, or fp32) stay below that too, with m + Hq terms.
Outputs in fp32: a probability's relative error is the score's absolute one (|score| <= 16: 16 x 4e-7) and __expf's (2 + |x| 2^-22), 8e-6 in the worst
case, mostly common to a row's numerator and denominator: 5e-6 in RMS.  Maxima over up to 1e6 entries: five sigma, ten times the RMS bound for safety of the
tails (cancellation in o).  bf16: half a unit in the last place, 2^-9 relative, on top."""
import numpy as np
import pytest
import torch

from paper_2408_01890_b200 import binding as lb
from paged_reference import BLOCK, Book, Mirror, shared_scores, softmax_v

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
FMT = {"s8": lb.S8, "e4m3": lb.E4M3}


def normal(rng, *shape, dtype=torch.float32):
    return torch.from_numpy(rng.standard_normal(shape, dtype=np.float32)).to(dtype)


def close(got, ref, rms, what):
    got, ref = got.double().cpu().numpy() if isinstance(got, torch.Tensor) else got, np.asarray(ref)
    assert np.isfinite(got).all(), what
    size = np.sqrt(np.mean(ref ** 2)) if ref.size else 0
    err = np.abs(got - ref)
    assert np.sqrt(np.mean(err ** 2)) <= rms * size and (err <= 10 * rms * size + 2 * rms * np.abs(ref)).all(), \
        "%s: rms %.2g of %.2g, max %.2g" % (what, np.sqrt(np.mean(err ** 2)), size, err.max())


RMS = {torch.float32: 5e-6, torch.bfloat16: 2.5e-3}
ROW_RMS = {torch.float32: 1e-6, torch.bfloat16: 2.5e-3}


def make(rng, kind, fmt, Hkv, P, d, r, lens, spare=3, garbage=True):
    """A layer whose pool is full of stale bytes (NaN codes and scales among them) and a table of scattered pages, entries behind a
    sequence's last page naming none; nothing appended yet."""
    per = max(1, -(-max(lens) // P)) + 1
    n_pages = len(lens) * per + spare
    layer = lb.PagedLayer(kind, Hkv, P, d, r if kind == lb.CACHE_SHARED else 0, dtype=FMT[fmt], n_pages=n_pages)
    layer.pool.fill_(0x7f if garbage else 0)          # e4m3: NaN
    if garbage:
        layer.scales.fill_(float("nan"))
    ids = rng.permutation(n_pages)[:len(lens) * per].reshape(len(lens), per).astype(np.int64)
    for b, n in enumerate(lens):
        ids[b, -(-n // P):] = rng.choice([-1, -7, n_pages, 2 ** 31 - 1])
    return layer, torch.from_numpy(ids.astype(np.int32)).cuda(), ids


def fill(rng, layer, table, lens, scale=1.0):
    """Appends random rows for all sequences."""
    kw = layer.r if layer.kind == lb.CACHE_SHARED else layer.d
    n = max(max(lens), 1)
    k, v = normal(rng, len(lens), n, layer.Hkv, kw) * scale, normal(rng, len(lens), n, layer.Hkv, layer.d)
    lb.lisa_paged_append(layer, table, k.cuda(), v.cuda(), None, torch.tensor(lens, dtype=torch.int32, device="cuda"))
    return k, v


# ------------------------------------------------------------------ rows in and out
ROWS = [  # kind, fmt, dtype, Hkv, d, r, page
    ("standard", "s8", "bf16", 3, 128, 0, 16), ("standard", "e4m3", "f32", 2, 128, 0, 64), ("standard", "s8", "f32", 1, 64, 0, 32),
    ("standard", "e4m3", "bf16", 5, 64, 0, 128), ("standard", "s8", "bf16", 2, 32, 0, 16), ("standard", "e4m3", "f32", 2, 32, 0, 32),
    ("shared", "s8", "bf16", 3, 128, 21, 32), ("shared", "e4m3", "bf16", 2, 128, 20, 16), ("shared", "s8", "f32", 2, 64, 1, 64),
    ("shared", "e4m3", "f32", 1, 32, 32, 128),
]


@pytest.mark.parametrize("kind,fmt,dtype,Hkv,d,r,P", ROWS)
def test_rows_are_appended_and_read_back(kind, fmt, dtype, Hkv, d, r, P):
    """Three appends behind one another (prompts of odd lengths, nothing, one token) leave exactly the codes and scales of the formula, in
    blocks that were partly filled too, and touch no other byte; reading gives code * scale."""
    rng = np.random.default_rng(d + r + P)
    kind = lb.CACHE_SHARED if kind == "shared" else lb.CACHE_STANDARD
    steps = [[37, 0, 16, 1, 130], [1, 5, 0, 15, 31], [1, 1, 1, 1, 1], [0, 64, 3, 0, 18]]
    total = np.sum(steps, 0).tolist()
    layer, table, ids = make(rng, kind, fmt, Hkv, P, d, r, total)
    mirror, first = Mirror(layer), np.zeros(5, np.int64)
    kw = r if kind == lb.CACHE_SHARED else d
    for i, counts in enumerate(steps):
        n = max(counts) + 2
        # rows inside larger tensors, heads further apart than their width; louder every step, so that scales grow
        k = normal(rng, 5, n, Hkv + 1, kw, dtype=DT[dtype])[:, :, 1:] * (1 + 2 * i)
        v = normal(rng, 5, n, Hkv, 2 * d, dtype=DT[dtype])[..., d:] * (1 + i % 2)
        kd, vd = torch.zeros((5, n, Hkv + 1, kw), dtype=DT[dtype], device="cuda"), torch.zeros((5, n, Hkv, 2 * d), dtype=DT[dtype], device="cuda")
        kd[:, :, 1:], vd[..., d:] = k.cuda(), v.cuda()
        lb.lisa_paged_append(layer, table, kd[:, :, 1:], vd[..., d:], torch.tensor(first, dtype=torch.int32, device="cuda"),
                             torch.tensor(counts, dtype=torch.int32, device="cuda"))
        mirror.append(ids, (k.float().numpy(), v.float().numpy()), first.tolist(), counts)
        first += counts
    have = Mirror(layer)
    for a, b in zip(have.codes + [have.scales], mirror.codes + [mirror.scales]):
        assert np.array_equal(a, b, equal_nan=True)
    assert lb.lisa_check() == lb.OK
    at = torch.tensor([3, 0, 17, 0, 15], dtype=torch.int32)
    count = [total[b] - int(at[b]) for b in range(5)]
    n = max(count) + 3
    k, v = torch.full((5, n, Hkv, kw), 7.0, dtype=DT[dtype], device="cuda"), torch.full((5, n, Hkv, d), 7.0, dtype=DT[dtype], device="cuda")
    lb.lisa_paged_read(layer, table, at.cuda(), k, v, torch.tensor(count, dtype=torch.int32, device="cuda"))
    for b in range(5):
        for i, got in enumerate((k, v)):
            want = np.stack([mirror.codes[i][ids[b, p // P], :, p % P] * mirror.scales[ids[b, p // P], :, p % P // BLOCK, i, None]
                             for p in range(int(at[b]), total[b])])
            assert torch.equal(got[b, :count[b]].cpu(), torch.from_numpy(want).to(DT[dtype]))
            assert (got[b, count[b]:] == 7).all()


@pytest.mark.parametrize("fmt", FMT)
def test_values_that_are_not_finite_and_zeros(fmt):
    """A block that is given a NaN or an infinity has the scale NaN, in that head and half alone, until it is written from its start;
    zeros have the scale 0; the smallest and the largest finite values come through."""
    rng = np.random.default_rng(0)
    layer, table, ids = make(rng, lb.CACHE_STANDARD, fmt, 4, 32, 32, 0, [48])
    mirror = Mirror(layer)
    k, v = normal(rng, 1, 40, 4, 32), normal(rng, 1, 40, 4, 32)
    k[0, 3, 1, 5], k[0, 20, 2, 0], v[0, 17, 0, 31] = float("inf"), float("nan"), -float("inf")
    k[0, :16, 3], v[0, 16:32, 3] = 0, 3.0e38
    v[0, 0:16, 2] = 1e-42                            # a denormal scale
    first, counts = [0], [40]
    lb.lisa_paged_append(layer, table, k.cuda(), v.cuda())
    mirror.append(ids, (k.numpy(), v.numpy()), first, counts)
    k2, v2 = normal(rng, 1, 9, 4, 32), normal(rng, 1, 9, 4, 32)
    at = torch.tensor([14], dtype=torch.int32, device="cuda")          # into the blocks with the infinity and the NaN
    lb.lisa_paged_append(layer, table, k2.cuda(), v2.cuda(), at)
    mirror.append(ids, (k2.numpy(), v2.numpy()), [14], [9])
    have = Mirror(layer)
    assert np.isnan(have.scales[ids[0, 0], 1, 0, 0])                                       # block 0: an older infinity stays
    assert not np.isnan(have.scales[ids[0, 0], 2, 1, 0])                                   # block 1 was written from its start
    for a, b in zip(have.codes + [have.scales], mirror.codes + [mirror.scales]):
        assert np.array_equal(a, b, equal_nan=True)


def test_positions_beyond_the_table_are_dropped_and_reported():
    rng = np.random.default_rng(1)
    layer, table, ids = make(rng, lb.CACHE_SHARED, "s8", 2, 16, 64, 8, [32, 32])
    table = table[:, :2].contiguous()
    before = layer.pool.clone()
    k, v = normal(rng, 2, 8, 2, 8).cuda(), normal(rng, 2, 8, 2, 64).cuda()
    lb.lisa_paged_append(layer, table, k, v, torch.tensor([32, -5], dtype=torch.int32, device="cuda"))
    assert torch.equal(layer.pool, before)
    assert lb.lisa_check() == lb.ERR_INVALID_ARG and lb.lisa_check() == lb.OK
    bad = table.clone()
    bad[1, 1] = layer.n_pages
    lb.lisa_paged_append(layer, bad, k, v, torch.tensor([0, 16], dtype=torch.int32, device="cuda"))
    assert torch.equal(layer.pool[ids[1, 1]], before[ids[1, 1]]) and not torch.equal(layer.pool[ids[0, 0]], before[ids[0, 0]])
    assert lb.lisa_check() == lb.ERR_INVALID_ARG


# ------------------------------------------------------------------ attention
ATTEND = [  # fmt, Hq, Hkv, d, page, q dtype, row dtype, lengths
    ("s8", 8, 8, 128, 16, "bf16", "f32", [1, 15, 16, 17, 0, 333]),
    ("e4m3", 32, 8, 128, 64, "bf16", "bf16", [700, 1, 65, 2000]),
    ("s8", 8, 1, 128, 32, "f32", "f32", [129, 640]),            # eight heads to a KV head: two column tiles
    ("e4m3", 12, 1, 128, 128, "f32", "f32", [31, 513]),          # twelve: two passes
    ("s8", 6, 2, 64, 16, "f32", None, [5, 257]),
    ("e4m3", 10, 2, 64, 32, "f32", "f32", [40, 0, 1]),
    ("s8", 4, 4, 32, 64, "f32", "f32", [128, 3]),
    ("e4m3", 64, 4, 32, 16, "bf16", "f32", [100]),
    ("s8", 40, 40, 128, 64, "f32", "f32", [1500, 1111]),
]


@pytest.mark.parametrize("fmt,Hq,Hkv,d,P,q_dtype,rows,lens", ATTEND)
def test_anchor_attention(fmt, Hq, Hkv, d, P, q_dtype, rows, lens):
    """Ragged batches over pages full of stale bytes; entries of the table and of the rows behind a length are neither read nor written."""
    rng = np.random.default_rng(Hq * d + P)
    layer, table, ids = make(rng, lb.CACHE_STANDARD, fmt, Hkv, P, d, 0, lens)
    fill(rng, layer, table, lens)
    mirror = Mirror(layer)
    B, L = len(lens), max(lens)
    q = (normal(rng, B, 1, Hq, d) * 1.5).to(DT[q_dtype])
    out = torch.empty((B, 1, Hq, d), dtype=DT[q_dtype], device="cuda")
    row = None if rows is None else torch.full((B, Hq, L + 5), 9.0, dtype=DT[rows], device="cuda")
    lb.lisa_attn_anchor_paged(q.cuda(), layer, table, L=L, seq_lens=torch.tensor(lens, dtype=torch.int32, device="cuda"), out=out, out_scores=row)
    assert lb.lisa_check() == lb.OK
    for b, n in enumerate(lens):
        if n == 0:
            assert (out[b] == 0).all() and (row is None or (row[b] == 9).all())
            continue
        K, V = mirror.rows(ids[b], n, 0), mirror.rows(ids[b], n, 1)
        a = np.einsum("hd,hnd->hn", q[b, 0].double().numpy(), np.repeat(K, Hq // Hkv, 0)) / np.sqrt(d)
        close(out[b, 0], softmax_v(a, V, Hq // Hkv), RMS[out.dtype], "o of sequence %d" % b)
        if row is not None:
            close(row[b, :, :n], a, ROW_RMS[row.dtype], "row of sequence %d" % b)
            assert (row[b, :, n:] == 9).all()


def test_a_sequence_alone_and_in_a_batch():
    """However many CTAs a sequence is split over, its result is the same to rounding; uniform lengths without seq_lens too, and a
    workspace made for the larger call serves the smaller."""
    rng = np.random.default_rng(2)
    lens = [4097] * 3
    layer, table, ids = make(rng, lb.CACHE_STANDARD, "s8", 8, 64, 128, 0, lens)
    fill(rng, layer, table, lens)
    q = normal(rng, 3, 1, 32, 128).cuda()
    ws = lb.paged_decode_workspace(layer, 3, 32, 4097)
    whole = lb.lisa_attn_anchor_paged(q, layer, table, L=4097, workspace=ws)
    for b in range(3):
        close(lb.lisa_attn_anchor_paged(q[b:b + 1], layer, table[b:b + 1], L=4097, workspace=ws), whole[b:b + 1].double().cpu().numpy(), 5e-6, "alone")
    assert torch.equal(whole, lb.lisa_attn_anchor_paged(q, layer, table, L=4097, seq_lens=torch.full((3,), 9999, dtype=torch.int32, device="cuda")))


def test_extreme_scales_and_scores():
    """Blocks whose V differ by 2^60 in magnitude, in either order; scores far apart; huge and tiny queries."""
    rng = np.random.default_rng(3)
    lens = [96, 96]
    layer, table, ids = make(rng, lb.CACHE_STANDARD, "s8", 2, 16, 128, 0, lens)
    k, v = normal(rng, 2, 96, 2, 128), normal(rng, 2, 96, 2, 128)
    for blk in range(6):
        v[0, 16 * blk:16 * blk + 16] *= 2.0 ** (10 * blk)
        v[1, 16 * blk:16 * blk + 16] *= 2.0 ** (-10 * blk)
    lb.lisa_paged_append(layer, table, k.cuda(), v.cuda())
    mirror = Mirror(layer)
    q = normal(rng, 2, 1, 2, 128)
    q[0, 0, 1] *= 1e-30
    q[1, 0, 0] *= 40.0                               # scores of several hundred: one position takes it all
    got = lb.lisa_attn_anchor_paged(q.cuda(), layer, table, L=96)
    for b in range(2):
        K, V = mirror.rows(ids[b], 96, 0), mirror.rows(ids[b], 96, 1)
        a = np.einsum("hd,hnd->hn", q[b, 0].double().numpy(), K) / np.sqrt(128)
        ref = softmax_v(a, V, 1)
        for h in range(2):                           # (scores of some hundred are off by some 1e-4 absolutely)
            close(got[b, 0, h], ref[h], 5e-6 if np.abs(a[h]).max() < 16 else 5e-4, "sequence %d head %d" % (b, h))


def test_values_that_are_not_finite_reach_their_own_head_alone():
    rng = np.random.default_rng(4)
    lens = [50]
    layer, table, ids = make(rng, lb.CACHE_STANDARD, "e4m3", 4, 32, 128, 0, lens)
    k, v = normal(rng, 1, 50, 4, 128), normal(rng, 1, 50, 4, 128)
    k[0, 7, 1, 3], v[0, 49, 2, 0] = float("nan"), float("inf")
    lb.lisa_paged_append(layer, table, k.cuda(), v.cuda())
    got = lb.lisa_attn_anchor_paged(normal(rng, 1, 1, 8, 128).cuda(), layer, table, L=50)
    bad = torch.isnan(got[0, 0]).all(1).cpu().tolist()
    assert bad == [False, False, True, True, True, True, False, False] and torch.isfinite(got[0, 0, [0, 1, 6, 7]]).all()


def test_absent_pages_are_skipped_and_reported():
    """Positions on a page that the table does not name count as absent; a sequence of nothing else gives 0."""
    rng = np.random.default_rng(5)
    lens = [64, 64]
    layer, table, ids = make(rng, lb.CACHE_STANDARD, "s8", 2, 16, 64, 0, lens)
    fill(rng, layer, table, lens)
    mirror = Mirror(layer)
    holes = table.clone()
    holes[0, 1], holes[1, :] = -1, layer.n_pages
    q = normal(rng, 2, 1, 2, 64)
    got = lb.lisa_attn_anchor_paged(q.cuda(), layer, holes, L=64)
    keep = [p for p in range(64) if p // 16 != 1]
    K, V = mirror.rows(ids[0], 64, 0)[:, keep], mirror.rows(ids[0], 64, 1)[:, keep]
    close(got[0, 0], softmax_v(np.einsum("hd,hnd->hn", q[0, 0].double().numpy(), K) / 8, V, 1), 5e-6, "absent page")
    assert (got[1] == 0).all()
    assert lb.lisa_check() == lb.ERR_INVALID_ARG and lb.lisa_check() == lb.OK


def test_pages_beyond_four_gigabytes():
    """Pages at the end of a pool of more than 2^32 bytes."""
    rng = np.random.default_rng(6)
    probe = lb.PagedLayer(lb.CACHE_STANDARD, 40, 128, 128, n_pages=1)
    n_pages = (1 << 32) // probe.layout.page_bytes + 8
    for kind, r in ((lb.CACHE_STANDARD, 0), (lb.CACHE_SHARED, 21)):
        layer = lb.PagedLayer(kind, 40, 128, 128, r, n_pages=n_pages if r == 0 else n_pages * 2)
        n_all = layer.n_pages
        table = torch.tensor([[n_all - 1, n_all - 5, n_all - 2]], dtype=torch.int32, device="cuda")
        lens = [300]
        fill(rng, layer, table, lens)
        k, v = torch.empty((1, 300, 40, r or 128), device="cuda"), torch.empty((1, 300, 40, 128), device="cuda")
        lb.lisa_paged_read(layer, table, None, k, v)
        K, V = k[0].double().cpu().numpy().transpose(1, 0, 2), v[0].double().cpu().numpy().transpose(1, 0, 2)
        if r == 0:
            q = normal(rng, 1, 1, 40, 128)
            got = lb.lisa_attn_anchor_paged(q.cuda(), layer, table, L=300)
            a = np.einsum("hd,hnd->hn", q[0, 0].double().numpy(), K) / np.sqrt(128)
        else:
            link, prev = make_link(rng, 40, r, 80), normal(rng, 1, 40, 300)
            got = lb.lisa_attn_shared_decode_paged(prev.cuda(), link, layer, table, L=300, out=torch.empty((1, 1, 40, 128), device="cuda"))
            a = shared_scores(prev[0].double().numpy(), link.qp[0, 0].double().cpu().numpy(), K, link)
        close(got[0, 0], softmax_v(a, V, 1), 5e-6, "o")
        del layer, k, v
        torch.cuda.empty_cache()


def make_link(rng, Hq, r, m, B=1, act=lb.ACT_RELU, integrate=lb.INTEGRATE_ADD, layers=2, w="bf16", bias=False, qp="bf16"):
    qp = normal(rng, B, 1, Hq, r, dtype=DT[qp]).cuda()
    if integrate == lb.INTEGRATE_PLUS:
        return lb.Link(qp, None, integrate=integrate)
    h_in = 2 * Hq if integrate == lb.INTEGRATE_CONCAT else Hq
    t = lambda *s: (normal(rng, *s) * (s[0] ** -0.5 if len(s) == 2 else 0.3)).to(DT[w]).cuda()
    m = Hq if layers == 1 else m
    return lb.Link(qp, None, t(h_in, m), t(m, Hq) if layers == 2 else None, t(m) if bias else None, t(Hq) if bias and layers == 2 else None,
                   act=act, integrate=integrate, ffn_layers=layers)


ADD, CONCAT, PLUS = lb.INTEGRATE_ADD, lb.INTEGRATE_CONCAT, lb.INTEGRATE_PLUS
SHARED = [  # fmt, Hq, Hkv, d, r, m, page, integrate, layers, act, weights, bias, rows, lengths
    ("s8", 32, 32, 128, 21, 64, 16, ADD, 2, lb.ACT_RELU, "bf16", False, "f32", [1, 15, 16, 17, 0, 333]),
    ("e4m3", 32, 8, 128, 21, 64, 64, ADD, 2, lb.ACT_SILU, "bf16", True, "bf16", [700, 1, 65, 1300]),
    ("s8", 40, 40, 128, 21, 80, 64, ADD, 2, lb.ACT_RELU, "bf16", True, "f32", [129, 640]),
    ("e4m3", 40, 10, 128, 20, 72, 32, ADD, 2, lb.ACT_NONE, "bf16", False, "f32", [257, 31]),
    ("s8", 32, 32, 128, 20, 256, 128, CONCAT, 2, lb.ACT_RELU, "bf16", True, "f32", [513, 40]),
    ("e4m3", 40, 40, 128, 20, 128, 16, CONCAT, 2, lb.ACT_SILU, "bf16", False, "bf16", [300]),
    ("s8", 32, 4, 128, 32, 40, 32, CONCAT, 2, lb.ACT_RELU, "bf16", False, "f32", [200, 77]),      # eight heads to a KV head
    ("s8", 32, 32, 64, 1, 64, 16, ADD, 2, lb.ACT_RELU, "bf16", False, "f32", [130]),
    ("e4m3", 32, 2, 128, 8, 64, 64, ADD, 2, lb.ACT_RELU, "bf16", False, "f32", [1000]),           # sixteen
    ("s8", 4, 4, 32, 8, 16, 16, ADD, 2, lb.ACT_RELU, "f32", True, "f32", [50, 0, 128]),
    ("e4m3", 32, 32, 128, 21, 64, 64, ADD, 2, lb.ACT_RELU, "f32", False, "f32", [100]),
    ("s8", 32, 8, 128, 21, 0, 16, PLUS, 2, lb.ACT_RELU, "bf16", False, "f32", [99, 1]),
    ("e4m3", 40, 40, 128, 21, 40, 32, ADD, 1, lb.ACT_RELU, "bf16", True, "f32", [140]),
    ("s8", 5, 5, 64, 7, 13, 32, CONCAT, 2, lb.ACT_SILU, "f32", True, "bf16", [61]),
    ("s8", 64, 64, 32, 5, 256, 16, CONCAT, 2, lb.ACT_RELU, "bf16", True, "f32", [33]),
]


@pytest.mark.parametrize("fmt,Hq,Hkv,d,r,m,P,integrate,layers,act,w,bias,rows,lens", SHARED)
@pytest.mark.parametrize("keep", [True, False])
def test_shared_attention(fmt, Hq, Hkv, d, r, m, P, integrate, layers, act, w, bias, rows, lens, keep):
    rng = np.random.default_rng(Hq * r + m + P)
    layer, table, ids = make(rng, lb.CACHE_SHARED, fmt, Hkv, P, d, r, lens)
    fill(rng, layer, table, lens)
    mirror = Mirror(layer)
    B, L = len(lens), max(lens)
    link = make_link(rng, Hq, r, m, B, act, integrate, layers, w, bias, "f32" if w == "f32" else "bf16")
    prev = torch.full((B, Hq, L + 3), float("nan"), dtype=DT[rows])
    for b, n in enumerate(lens):
        prev[b, :, :n] = normal(rng, Hq, n)
    row = torch.full((B, Hq, L + 5), 9.0, dtype=DT[rows], device="cuda") if keep else None
    out = torch.empty((B, 1, Hq, d), dtype=torch.float32 if keep else torch.bfloat16, device="cuda")
    lb.lisa_attn_shared_decode_paged(prev.cuda(), link, layer, table, L=L, seq_lens=torch.tensor(lens, dtype=torch.int32, device="cuda"),
                                     out=out, out_scores=row)
    assert lb.lisa_check() == lb.OK
    for b, n in enumerate(lens):
        if n == 0:
            assert (out[b] == 0).all() and (row is None or (row[b] == 9).all())
            continue
        KP, V = mirror.rows(ids[b], n, 0), mirror.rows(ids[b], n, 1)
        a = shared_scores(prev[b, :, :n].double().numpy(), link.qp[b, 0].double().cpu().numpy(), KP, link)
        close(out[b, 0], softmax_v(a, V, Hq // Hkv), RMS[out.dtype], "o of sequence %d" % b)
        if row is not None:
            close(row[b, :, :n], a, ROW_RMS[row.dtype], "row of sequence %d" % b)
            assert (row[b, :, n:] == 9).all()


def check_batch(rng, kind, fmt, Hq, Hkv, P, r, m, lens, integrate=lb.INTEGRATE_ADD, ragged=True, some=None):
    """A batch through one layer against 64 bits, for the sequences `some` (all when None)."""
    layer, table, ids = make(rng, kind, fmt, Hkv, P, 128, r, lens)
    fill(rng, layer, table, lens)
    mirror = Mirror(layer)
    B, L = len(lens), max(lens)
    seq = torch.tensor(lens, dtype=torch.int32, device="cuda") if ragged else None
    out, row = torch.empty((B, 1, Hq, 128), device="cuda"), torch.full((B, Hq, L), 9.0, device="cuda")
    if kind == lb.CACHE_STANDARD:
        q = normal(rng, B, 1, Hq, 128)
        lb.lisa_attn_anchor_paged(q.cuda(), layer, table, L=L, seq_lens=seq, out=out, out_scores=row)
    else:
        link, prev = make_link(rng, Hq, r, m, B, integrate=integrate), normal(rng, B, Hq, L)
        lb.lisa_attn_shared_decode_paged(prev.cuda(), link, layer, table, L=L, seq_lens=seq, out=out, out_scores=row)
    assert lb.lisa_check() == lb.OK
    for b in range(B) if some is None else some:
        n = lens[b]
        if n == 0:
            assert (out[b] == 0).all() and (row[b] == 9).all()
            continue
        K, V = mirror.rows(ids[b], n, 0), mirror.rows(ids[b], n, 1)
        if kind == lb.CACHE_STANDARD:
            a = np.einsum("hd,hnd->hn", q[b, 0].double().numpy(), np.repeat(K, Hq // Hkv, 0)) / np.sqrt(128)
        else:
            a = shared_scores(prev[b, :, :n].double().numpy(), link.qp[b, 0].double().cpu().numpy(), K, link)
        close(out[b, 0], softmax_v(a, V, Hq // Hkv), 5e-6, "o of sequence %d" % b)
        close(row[b, :, :n], a, 1e-6, "row of sequence %d" % b)
        assert (row[b, :, n:] == 9).all()


@pytest.mark.parametrize("fmt", FMT)
@pytest.mark.parametrize("kind", [lb.CACHE_STANDARD, lb.CACHE_SHARED])
def test_many_short_sequences(fmt, kind):
    """150 sequences of lengths 0 .. 200, pages of 16."""
    rng = np.random.default_rng(20)
    lens = [0, 1, 200] + rng.integers(0, 200, 147).tolist()
    check_batch(rng, kind, fmt, 32, 4, 16, 21, 64, lens, some=list(range(0, 150, 7)) + [0, 1, 2, 149])


@pytest.mark.parametrize("lens", [[0] * 33 + [77] + [0] * 30 + [129], [5] * 128, [0, 0, 0]])
def test_batches_that_are_mostly_idle_or_all_alike(lens):
    rng = np.random.default_rng(21)
    if max(lens) == 0:
        layer, table, _ = make(rng, lb.CACHE_STANDARD, "s8", 2, 16, 128, 0, [16, 16, 16])
        out = lb.lisa_attn_anchor_paged(normal(rng, 3, 1, 4, 128).cuda(), layer, table, L=16, seq_lens=torch.zeros(3, dtype=torch.int32, device="cuda"))
        assert (out == 0).all()
        return
    check_batch(rng, lb.CACHE_SHARED, "s8", 32, 8, 16, 21, 64, lens)
    check_batch(rng, lb.CACHE_STANDARD, "e4m3", 4, 4, 16, 0, 0, lens)


@pytest.mark.parametrize("fmt,integrate,r,Hkv", [("s8", lb.INTEGRATE_ADD, 21, 32), ("e4m3", lb.INTEGRATE_ADD, 32, 32), ("e4m3", lb.INTEGRATE_CONCAT, 20, 16),
                                                 ("s8", lb.INTEGRATE_CONCAT, 25, 16), ("e4m3", lb.INTEGRATE_ADD, 24, 8)])
@pytest.mark.parametrize("ragged", [True, False])
def test_many_chunks_to_a_cta(fmt, integrate, r, Hkv, ragged):
    """64 sequences of 600: several chunks to a CTA of the scores, one after another, and every rank the blocks' layouts distinguish."""
    rng = np.random.default_rng(22)
    lens = [600] + (rng.integers(300, 601, 63).tolist() if ragged else [600] * 63)
    check_batch(rng, lb.CACHE_SHARED, fmt, 32, Hkv, 64, r, 64, lens, integrate, ragged, some=[0, 1, 31, 32, 63])


@pytest.mark.parametrize("fmt", FMT)
@pytest.mark.parametrize("Hq,Hkv", [(16, 8), (3, 1), (5, 1), (6, 6)])
def test_every_number_of_heads_to_a_kv_head(fmt, Hq, Hkv):
    rng = np.random.default_rng(Hq)
    check_batch(rng, lb.CACHE_STANDARD, fmt, Hq, Hkv, 32, 0, 0, [333, 17, 0, 1000])


def test_a_long_sequence_over_the_whole_card():
    """One sequence of 30001 positions: split over wide CTAs, sums of many units."""
    rng = np.random.default_rng(23)
    for fmt in FMT:
        check_batch(rng, lb.CACHE_STANDARD, fmt, 4, 1, 128, 0, 0, [30001], ragged=False)


@pytest.mark.parametrize("fmt", FMT)
@pytest.mark.parametrize("Hkv", [8, 4, 2, 1])
@pytest.mark.parametrize("n", [40, 3001])
def test_masks_in_the_previous_row(fmt, Hkv, n):
    """A row of -inf where positions are masked, handed on as it is (no aligner): masked positions weigh nothing, wherever they lie; a head with nothing else gives 0;
    NaN and +inf reach their own head alone."""
    rng = np.random.default_rng(n + Hkv)
    layer, table, ids = make(rng, lb.CACHE_SHARED, fmt, Hkv, 32, 64, 8, [n])
    fill(rng, layer, table, [n])
    mirror = Mirror(layer)
    link = make_link(rng, 8, 8, 0, integrate=PLUS)
    prev, inf = normal(rng, 1, 8, n), float("inf")
    prev[0, 0] = -inf
    prev[0, 1, :n - 1] = -inf
    prev[0, 2, 1:] = -inf
    prev[0, 3, :n // 2] = -inf
    prev[0, 4, ::3] = -inf
    prev[0, 5, n // 3] = float("nan")
    prev[0, 6, n - 2] = inf
    out = lb.lisa_attn_shared_decode_paged(prev.cuda(), link, layer, table, L=n, out=torch.empty((1, 1, 8, 64), device="cuda"))[0, 0]
    a = shared_scores(prev[0].double().numpy(), link.qp[0, 0].double().cpu().numpy(), mirror.rows(ids[0], n, 0), link)
    assert (out[0] == 0).all() and torch.isnan(out[5]).all() and torch.isnan(out[6]).all()
    keep, V = [1, 2, 3, 4, 7], np.repeat(mirror.rows(ids[0], n, 1), 8 // Hkv, 0)
    close(out[keep], softmax_v(a[keep], V[keep], 1), 5e-6, "masked")


@pytest.mark.parametrize("rows", ["f32", "bf16"])
def test_a_mask_of_the_lowest_value_in_the_previous_row(rows):
    """The largest finite scores of either sign (a mask in the row of the layer before) stay finite in that layer's own sums: an aligner of zeros there passes
    nothing on, and no other position notices."""
    rng = np.random.default_rng(8)
    Hq, n = 32, 200
    layer, table, ids = make(rng, lb.CACHE_SHARED, "s8", 8, 16, 128, 21, [n])
    fill(rng, layer, table, [n])
    mirror = Mirror(layer)
    link = make_link(rng, Hq, 21, 64)
    link.w1[3] = 0                                   # head 3 does not enter
    prev = normal(rng, 1, Hq, n).to(DT[rows])
    prev[0, 3, ::7] = torch.finfo(DT[rows]).min
    prev[0, 3, 1::7] = torch.finfo(DT[rows]).max
    row = torch.empty((1, Hq, n), dtype=DT[rows], device="cuda")
    out = lb.lisa_attn_shared_decode_paged(prev.cuda(), link, layer, table, L=n, out=torch.empty((1, 1, Hq, 128), device="cuda"), out_scores=row)
    a = shared_scores(prev[0].double().numpy(), link.qp[0, 0].double().cpu().numpy(), mirror.rows(ids[0], n, 0), link)
    close(row[0], a, ROW_RMS[row.dtype], "row")
    close(out[0, 0], softmax_v(a, mirror.rows(ids[0], n, 1), 4), 5e-6, "o")


# ------------------------------------------------------------------ pages
def same(pages, book):
    assert np.array_equal(pages.table.cpu().numpy(), book.table)
    assert np.array_equal(pages.lens.cpu().numpy(), book.lens)
    assert np.array_equal(pages.refs.cpu().numpy(), book.refs)


@pytest.mark.parametrize("B,max_pages,n_pages,P,seed", [(1, 3, 5, 16, 0), (7, 40, 150, 16, 1), (33, 70, 1500, 32, 2), (64, 9, 300, 128, 3),
                                                        (1024, 5, 6000, 16, 4), (5, 33, 3000, 64, 5)])
def test_bookkeeping_follows_the_plain_one(B, max_pages, n_pages, P, seed):
    """A random run of forks, frees, reserves and compactions, pages of two layers (of unlike sizes) moving along; what does not fit changes nothing."""
    rng = np.random.default_rng(seed)
    cache = lb.PagedCache([lb.CACHE_STANDARD, lb.CACHE_SHARED], n_pages, 2 if B < 1000 else 1, P, 32, 5)
    for l in cache.layers:
        l.pool.copy_(torch.randint(0, 256, l.pool.shape, dtype=torch.uint8, device="cuda"))
    want = [l.pool.cpu().numpy().copy() for l in cache.layers]
    pages, book = lb.Pages.empty(B, max_pages, n_pages, P), Book(B, max_pages, n_pages, P)
    dev = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")
    for step in range(30):
        what = rng.choice(["reserve", "reserve", "fork", "free", "compact", "permute"])
        moves = []
        if what == "reserve":
            n_new = rng.integers(-2, 2 * P, B) if step < 20 else rng.integers(0, max_pages * P, B)
            if rng.random() < 0.3:
                n_new[:] = 1
            moves = book.reserve(n_new)
            lb.lisa_pages_reserve(pages, cache, None if (n_new == 1).all() else dev(n_new))
            assert lb.lisa_check() == (lb.ERR_NO_PAGES if moves is None else lb.OK)
            if moves is None:
                moves = []
            else:
                book.lens += np.maximum(n_new, 0)
                pages.lens += dev(np.maximum(n_new, 0))
        elif what == "compact":
            moves = book.compact()
            lb.lisa_pages_compact(pages, cache)
        else:
            parent = {"fork": rng.integers(0, B, B), "free": np.where(rng.random(B) < 0.4, -1, np.arange(B)), "permute": rng.permutation(B)}[what]
            book.fork(parent)
            lb.lisa_pages_fork(pages, dev(parent))
        same(pages, book)
        for w in want:
            for src, dst in moves:
                w[dst] = w[src]
    for l, w in zip(cache.layers, want):
        assert np.array_equal(l.pool.cpu().numpy(), w)
    assert lb.lisa_check() == lb.OK


@pytest.mark.parametrize("n_pages,n_new,fits", [(6, [32, 33, 16], True), (5, [32, 33, 16], False), (5, [32, 33, 0], True), (100, [64, 1, 1], True),
                                                (100, [1, 65, 1], False)])
def test_what_does_not_fit_changes_nothing(n_pages, n_new, fits):
    """Too few free pages, or a row longer than the table is wide: all rows stay as they are."""
    cache = lb.PagedCache([lb.CACHE_STANDARD], n_pages, 1, 16, 32)
    pages, book = lb.Pages.empty(3, 4, n_pages, 16), Book(3, 4, n_pages, 16)
    lb.lisa_pages_reserve(pages, cache, torch.tensor(n_new, dtype=torch.int32, device="cuda"))
    assert (book.reserve(n_new) is not None) == fits
    same(pages, book)
    assert lb.lisa_check() == (lb.OK if fits else lb.ERR_NO_PAGES) and lb.lisa_check() == lb.OK


def test_parents_out_of_range_free_their_rows_and_are_reported():
    pages, book = lb.Pages.empty(3, 4, 10, 16), Book(3, 4, 10, 16)
    cache = lb.PagedCache([lb.CACHE_STANDARD], 10, 1, 16, 32)
    n = torch.tensor([40, 20, 16], dtype=torch.int32, device="cuda")
    lb.lisa_pages_reserve(pages, cache, n)
    book.reserve([40, 20, 16])
    pages.lens += n
    book.lens += [40, 20, 16]
    lb.lisa_pages_fork(pages, torch.tensor([3, 1, -2], dtype=torch.int32, device="cuda"))
    book.fork([3, 1, -2])
    same(pages, book)
    assert lb.lisa_check() == lb.ERR_INVALID_ARG


def test_pages_are_copied_in_every_layer():
    rng = np.random.default_rng(9)
    cache = lb.PagedCache([lb.CACHE_SHARED, lb.CACHE_STANDARD, lb.CACHE_SHARED], 30, 3, 64, 128, 21, dtype=lb.E4M3)
    for l in cache.layers:
        l.pool.copy_(torch.randint(0, 256, l.pool.shape, dtype=torch.uint8, device="cuda"))
    want = [l.pool.clone() for l in cache.layers]
    ids = rng.permutation(30)
    src, dst = ids[:11].tolist() + [30, 2], ids[11:22].tolist() + [int(ids[22]), -1]
    lb.lisa_pages_copy(cache, torch.tensor(src, dtype=torch.int32, device="cuda"), torch.tensor(dst, dtype=torch.int32, device="cuda"))
    for l, w in zip(cache.layers, want):
        w[dst[:11]] = w[src[:11]]
        assert torch.equal(l.pool, w)
    assert lb.lisa_check() == lb.ERR_INVALID_ARG             # the two pairs with an id outside the pools


def test_a_forked_sequence_writes_to_its_own_copy():
    """Fork, reserve, append on a side stream: the child's token changes the child alone, and both attend to what they hold."""
    rng = np.random.default_rng(10)
    cache = lb.PagedCache([lb.CACHE_STANDARD], 12, 2, 16, 64)
    layer = cache.layers[0]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        pages = lb.Pages.empty(2, 4, 12, 16)
        lb.lisa_pages_reserve(pages, cache, torch.tensor([37, 0], dtype=torch.int32, device="cuda"))
        k, v = normal(rng, 2, 37, 2, 64), normal(rng, 2, 37, 2, 64)
        lb.lisa_paged_append(layer, pages.table, k.cuda(), v.cuda(), pages.lens, torch.tensor([37, 0], dtype=torch.int32, device="cuda"))
        pages.lens += torch.tensor([37, 0], dtype=torch.int32, device="cuda")
        lb.lisa_pages_fork(pages, torch.tensor([0, 0], dtype=torch.int32, device="cuda"))
        assert pages.table[0, :3].equal(pages.table[1, :3]) and pages.refs.sum() == 6
        lb.lisa_pages_reserve(pages, cache)
        assert pages.table[0, :2].equal(pages.table[1, :2]) and pages.table[0, 2] != pages.table[1, 2]
        k1, v1 = normal(rng, 2, 1, 2, 64) * 3, normal(rng, 2, 1, 2, 64) * 3
        lb.lisa_paged_append(layer, pages.table, k1.cuda(), v1.cuda(), pages.lens)
        pages.lens += 1
        q = normal(rng, 2, 1, 4, 64)
        got = lb.lisa_attn_anchor_paged(q.cuda(), layer, pages.table, L=38, seq_lens=pages.lens)
        assert lb.lisa_check() == lb.OK
    mirror, ids = Mirror(layer), pages.table.cpu().numpy()
    for b in range(2):
        K, V = mirror.rows(ids[b], 38, 0), mirror.rows(ids[b], 38, 1)
        assert np.abs(K[:, 37] - k1[b, 0].numpy()).max() < 0.1 and np.abs(K[:, :37] - k[0].numpy().transpose(1, 0, 2)).max() < 0.1
        a = np.einsum("hd,hnd->hn", q[b, 0].double().numpy(), np.repeat(K, 2, 0)) / 8
        close(got[b, 0], softmax_v(a, V, 2), 5e-6, "o of %d" % b)


def test_a_step_replayed_from_a_graph():
    """Reserve, append and attend captured once, lengths and tables on the device: replays do what single calls do."""
    rng = np.random.default_rng(11)
    B, H, P = 3, 2, 16

    def setup():
        r = np.random.default_rng(12)
        cache = lb.PagedCache([lb.CACHE_STANDARD], 40, H, P, 64)
        cache.layers[0].pool.zero_()
        pages = lb.Pages.empty(B, 8, 40, P)
        n = torch.tensor([15, 1, 30], dtype=torch.int32, device="cuda")
        lb.lisa_pages_reserve(pages, cache, n)
        k, v = normal(r, B, 30, H, 64).cuda(), normal(r, B, 30, H, 64).cuda()
        lb.lisa_paged_append(cache.layers[0], pages.table, k, v, pages.lens, n)
        pages.lens += n
        return cache, pages

    kd, vd, q = normal(rng, B, 1, H, 64).cuda(), normal(rng, B, 1, H, 64).cuda(), normal(rng, B, 1, H, 64).cuda()

    def step(cache, pages, out, ws):
        lb.lisa_pages_reserve(pages, cache)
        lb.lisa_paged_append(cache.layers[0], pages.table, kd, vd, pages.lens)
        pages.lens.add_(1)
        lb.lisa_attn_anchor_paged(q, cache.layers[0], pages.table, L=8 * P, seq_lens=pages.lens, out=out, workspace=ws)

    outs = []
    for graph in (False, True):
        cache, pages = setup()
        out = torch.empty((B, 1, H, 64), device="cuda")
        ws = lb.paged_decode_workspace(cache.layers[0], B, H, 8 * P)
        if graph:
            torch.cuda.synchronize()
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                step(cache, pages, out, ws)
        for _ in range(20):
            g.replay() if graph else step(cache, pages, out, ws)
        torch.cuda.synchronize()
        outs.append([out.clone(), pages.table.clone(), pages.lens.clone(), pages.refs.clone(), cache.layers[0].pool.clone()])
    for a, b in zip(*outs):
        assert torch.equal(a, b)
    assert outs[0][2].tolist() == [35, 21, 50]
