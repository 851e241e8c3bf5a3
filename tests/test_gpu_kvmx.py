"""The microscaled key/value cache on the GPU against its float64 reference."""
import math

import numpy as np
import pytest

import oracle as O
from harness import NAN_BITS, dev_bf16, dev_i32, host_bits, host_f32
from oracle import mxkv_ref as M
from workloads import make_rng, normal_bf16

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def A(gpu):
    from paper_2606_15319_amd import ardit
    return ardit


def _sync():
    import torch
    torch.cuda.synchronize()


def _u8(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a)).to("cuda")


class Pool:
    """A pool on the host and the device, and the page ids of each stream."""

    def __init__(self, A, H, d, lat, frames, bits, lens, seed=0, shared=0, fill=0xFF, spare=2):
        T = lat[0] * lat[1]
        self.A, self.H, self.d, self.T, self.bits = A, H, d, T, bits
        self.dims = A.make_dims(H * d, H, d, 128, frames, lat[0], lat[1])
        need = [-(-n // T) for n in lens]
        pages = shared + sum(f - min(shared, f) for f in need) + spare
        perm = [int(x) for x in np.random.default_rng(seed).permutation(pages)]
        at = shared
        self.ids = []
        for f in need:
            own = f - min(shared, f)
            self.ids.append(perm[:min(shared, f)] + perm[at:at + own])
            at += own
        self.n_pages, self.span = pages, max(need + [1])
        self.host = M.Pages(pages, H, d, T, bits, fill)
        # entries of no use to a stream lie far outside the pool
        table = np.full((len(lens), self.span), 1 << 30, np.int32)
        for b, i in enumerate(self.ids):
            table[b, :len(i)] = i
        self.table = dev_i32(table)

    def fill(self, lens, seed, shared=0, scale=1.0):
        """Draws each stream's keys and values, packs them, returns the values they stand for."""
        rng = make_rng(seed)
        out = []
        for b, n in enumerate(lens):
            k, v = [], []
            for f, page in enumerate(self.ids[b]):
                m = min(self.T, n - f * self.T)
                if f < shared and out:
                    kk, vv = out[0][0][f * self.T:f * self.T + m], out[0][1][f * self.T:f * self.T + m]
                else:
                    kk, vv = self.host.pack(page, scale * normal_bf16(rng, (m, self.H, self.d)).astype(np.float64),
                                            normal_bf16(rng, (m, self.H, self.d)).astype(np.float64))
                k.append(kk)
                v.append(vv)
            shape = (0, self.H, self.d)
            out.append((np.concatenate(k) if k else np.zeros(shape), np.concatenate(v) if v else np.zeros(shape)))
        self.upload()
        return out

    def upload(self):
        h = self.host
        self.dev = [_u8(x) for x in (h.k_codes, h.k_scales, h.v_codes, h.v_scales)]

    def download(self):
        h = self.host
        h.k_codes, h.k_scales, h.v_codes, h.v_scales = [t.cpu().numpy() for t in self.dev]

    def kv(self):
        fmt = self.A.KV_E4M3 if self.bits == 8 else self.A.KV_E2M1
        return self.A.kv_mx(*self.dev, self.table, self.n_pages, self.span, fmt)


def _attend(A, pool, q_lens, caches, q, shared=0, stream=None, ws=None, o=None):
    import torch
    batch = A.Batch(q_lens, caches)
    n = A.ardit_workspace_size(pool.dims, batch)
    if ws is None:
        ws = torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")
    if o is None:
        o = torch.full_like(q, float("nan"))
    A.ardit_attn_fwd_mx(stream, pool.dims, batch, q, pool.kv(), shared, o, ws, ws.numel())
    return o


def _check_attention(got, q, k, v, independent=True):
    """got [R, H, d] against float64.  Rounding the weights to bf16 moves the numerator by
    at most 2^-8 sum p |v|, the denominator (a sum of the rounded weights) by 2^-8 of itself;
    the store rounds by 2^-8; 2^-10 more of the weights covers the scores (queries split
    into two E4M3 parts, 2^-21 of a block's largest element per product, and fp32 sums)
    and exp2.  Over many keys the errors cancel: a weight's is uniform within its half
    step, at most 2^-8 / sqrt(3) of it, independent of the others (not those of a key that
    comes again: then only the first bound holds)."""
    d = q.shape[-1]
    s = np.einsum("rhd,khd->hrk", q, k) / math.sqrt(d)
    p = np.exp(s - s.max(-1, keepdims=True))
    p /= p.sum(-1, keepdims=True)
    ref = np.einsum("hrk,khd->rhd", p, v)
    spread = np.einsum("hrk,khd->rhd", p, np.abs(v))
    err = np.abs(got - ref)
    tiny = 2.0 ** -120
    assert np.all(err <= (2.0 ** -7 + 2.0 ** -10) * spread + 2.0 ** -8 * np.abs(ref) + tiny)
    if not independent:
        return
    p2 = p * p
    var = np.einsum("hrk,khd->rhd", p2, v * v) + p2.sum(-1).T[:, :, None] * ref * ref
    sd = 2.0 ** -8 / math.sqrt(3) * np.sqrt(var + ref * ref) + 2.0 ** -10 * np.sqrt(var) + tiny
    z = err / sd
    assert np.sqrt(np.mean(z * z)) <= 1.2 and z.max() <= 7.0, (np.sqrt(np.mean(z * z)), z.max())


# ------------------------------------------------------------------- append
APPENDS = [   # H, d, (lat_h, lat_w), frames, cached frames per stream, first positions
    (4, 64, (8, 8), 3, [2], [6]),
    (2, 128, (6, 12), 1, [0, 5, 1], [0, 7, 100000]),       # T = 72: a tile of 8 keys behind a whole one
    (10, 64, (4, 8), 2, [3, 0], [3, 9]),                   # T = 32: half a tile
    (1, 128, (7, 8), 3, [1], [1]),                         # T = 56, width 128
    (13, 128, (8, 8), 1, [1], [2]),                        # rows of 1664: one to a wave
    (20, 128, (6, 12), 1, [0], [3]),                       # 2560: one to two waves
    (32, 128, (8, 8), 1, [0], [0]),                        # 4096: the widest of those
    (33, 128, (8, 8), 1, [0], [2]),                        # 4224: one to four waves
    (64, 128, (8, 8), 1, [1], [4]),                        # the widest rows
    (12, 128, (30, 52), 1, [1], [11]),
]


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("H,d,lat,frames,cached,pos", APPENDS)
def test_append(A, bits, H, d, lat, frames, cached, pos):
    """Queries, codes and scales of a chunk; every other byte of the pool as it was."""
    import torch
    D, T = H * d, lat[0] * lat[1]
    L = frames * T
    pool = Pool(A, H, d, lat, frames, bits, [(c + frames) * T for c in cached], seed=1, fill=0xA5)
    pool.upload()
    rng = make_rng(7)
    qkv = normal_bf16(rng, (L * len(cached), 3 * D))
    g = [1 + 0.02 * normal_bf16(rng, (D,)) for _ in range(2)]
    gq, gk = dev_bf16(g[0]), dev_bf16(g[1])
    gains = [host_f32(gq), host_f32(gk)]
    q = torch.full((L * len(cached), D), float("nan"), dtype=torch.bfloat16, device="cuda")
    A.ardit_kv_append_mx(None, pool.dims, A.Batch([L] * len(cached), [c * T for c in cached], pos),
                         dev_bf16(qkv), gq, gk, pool.kv(), q)
    _sync()
    pool.download()
    got_q = host_f32(q).astype(np.float64)
    written = set()
    for b, c in enumerate(cached):
        x = qkv[b * L:(b + 1) * L].astype(np.float64)
        where = O.chunk_positions(frames, lat[0], lat[1], pos[b])
        qr = O.rope3d(O.rms_norm(x[:, :D], 1e-6, gains[0]).reshape(L, H, d), where, 10000.0)
        kr = O.rope3d(O.rms_norm(x[:, D:2 * D], 1e-6, gains[1]).reshape(L, H, d), where, 10000.0)
        vr = x[:, 2 * D:].reshape(L, H, d)
        e = np.abs(got_q[b * L:(b + 1) * L] - qr.reshape(L, D))
        # a bf16 store, and fp32 sums of 8192 squares and products: 2e-6 of the values rotated
        assert np.all(e <= 2.0 ** -8 * np.abs(qr.reshape(L, D)) + 2e-5)
        for f in range(frames):
            page = pool.ids[b][c + f]
            written.add(page)
            ku, vu = pool.host.unpack(page)
            kf, vf = kr[f * T:(f + 1) * T], vr[f * T:(f + 1) * T]
            assert np.array_equal(vu, M.rounded(vf, bits, 0)), "values are exact"
            want = M.rounded(kf, bits, -1)
            # the code of a key may differ where its value is next to a border: it is then as near
            off = np.abs(ku - kf) - np.abs(want - kf)
            assert np.all(off <= 4e-5) and np.mean(ku != want) <= 1e-4
            n = T % 64
            if n:     # the padding of the last tile's values is zero
                codes = pool.host._codes(pool.host.v_codes[page])[:, -1, :, n:]
                assert not codes.any()
    rest = [p for p in range(pool.n_pages) if p not in written]
    for a in (pool.host.k_codes, pool.host.k_scales, pool.host.v_codes, pool.host.v_scales):
        assert (a[rest] == 0xA5).all()
    assert (pool.host.k_codes[:, :, T:] == 0xA5).all() and (pool.host.k_scales[:, :, T:] == 0xA5).all()


@pytest.mark.parametrize("bits", [8, 4])
def test_append_extreme_values(A, bits):
    """Zero rows, blocks of one large element, tiny and huge values, infinities and NaN in the values."""
    import torch
    H, d, T = 2, 64, 64
    D = H * d
    pool = Pool(A, H, d, (8, 8), 1, bits, [T], fill=0)
    pool.upload()
    rng = make_rng(8)
    qkv = normal_bf16(rng, (T, 3 * D)).astype(np.float32)
    v = qkv[:, 2 * D:]
    v[:, 0] = 0.0
    v[:, 1] *= np.float32(2.0 ** 100)
    v[:, 2] *= np.float32(2.0 ** -100)
    v[:, 3] = np.float32(2.0 ** -126)
    v[5, 4] = 3000.0
    v[:, 5] = 6.0
    v[:, 6] = -7.0
    v[40, 7] = np.inf
    v[3, 8] = np.nan
    v[:, 9] = 255.0
    qkv[9, :2 * D] = 0.0        # norm of a zero row
    dev = dev_bf16(qkv)
    qkv = host_f32(dev).astype(np.float64)
    one = dev_bf16(np.ones(D, np.float32))
    q = torch.empty((T, D), dtype=torch.bfloat16, device="cuda")
    A.ardit_kv_append_mx(None, pool.dims, A.Batch([T], [0], [0]), dev, one, one, pool.kv(), q)
    _sync()
    pool.download()
    k, vu = pool.host.unpack(pool.ids[0][0])
    want = M.rounded(qkv[:, 2 * D:].reshape(T, H, d), bits, 0)
    assert np.array_equal(vu, want, equal_nan=True)
    assert np.isnan(vu[32:, 0, 7]).all() and np.isfinite(vu[:32, 0, 7]).all() and np.isnan(vu[:32, 0, 8]).all()
    assert not k[9].any() and not host_f32(q)[9].any()


# ---------------------------------------------------------------- read-back
@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("H,d,lat,lens,cached", [
    (3, 128, (6, 12), [1, 77, 0, 300], [0, 2, 1, 0]),
    (2, 64, (4, 8), [33, 64], [0, 1]),
    (2, 64, (8, 8), [130, 1, 64], [3, 0, 0]),
    (2, 128, (30, 52), [1600, 3119], [0, 1]),
    (40, 128, (8, 8), [100], [0]),
])
def test_read_back(A, bits, H, d, lat, lens, cached):
    """Exact values in bf16, and every token that is not asked for as it was."""
    import torch
    T = lat[0] * lat[1]
    total = [c * T + n for c, n in zip(cached, lens)]
    pool = Pool(A, H, d, lat, 1, bits, total, seed=3)
    held = pool.fill(total, 11)
    # a pool of its own, in another order, with the other frames' entries outside it
    own = [-(-n // T) for n in lens]
    perm = np.random.default_rng(5).permutation(sum(own) + 1)
    table = np.full((len(lens), pool.span), -7, np.int32)
    at = 0
    ids = []
    for b, (c, m) in enumerate(zip(cached, own)):
        ids.append(perm[at:at + m])
        table[b, c:c + m] = perm[at:at + m]
        at += m
    k = torch.full((len(perm), H, T, d), -3.0, dtype=torch.bfloat16, device="cuda")
    v = torch.full((len(perm), H, d, T), -3.0, dtype=torch.bfloat16, device="cuda")
    dst = A.kv_paged(k, v, dev_i32(table), len(perm), pool.span)
    A.ardit_kv_read_mx(None, pool.dims, A.Batch(lens, [c * T for c in cached]), pool.kv(), dst)
    _sync()
    kg, vg = host_f32(k), host_f32(v)
    want_k, want_v = np.full(kg.shape, -3.0), np.full(vg.shape, -3.0)
    for b, (c, n) in enumerate(zip(cached, lens)):
        for f, page in enumerate(ids[b]):
            m = min(T, n - f * T)
            at = (c + f) * T
            want_k[page, :, :m] = held[b][0][at:at + m].transpose(1, 0, 2)
            want_v[page, :, :, :m] = held[b][1][at:at + m].transpose(1, 2, 0)
    assert np.array_equal(kg, want_k) and np.array_equal(vg, want_v)


# ---------------------------------------------------------------- attention
ATTN = [   # H, d, lattice, rows, cached frames
    (2, 128, (8, 8), [1], [0]),                                # one row, one key
    (3, 128, (6, 12), [1, 0, 2, 33], [0, 3, 11, 2]),
    (4, 64, (4, 8), [5, 32, 31], [9, 0, 1]),                   # half tiles
    (2, 64, (6, 12), [17, 192, 1, 0, 65], [3, 64, 20, 8, 1]),
    (2, 128, (30, 52), [3, 100], [2, 1]),                      # tiles of 24 keys at each frame's end
    (1, 128, (8, 8), [1], [300]),
    (20, 64, (8, 8), [1] * 24, list(range(24))),               # more items than one round
    (2, 128, (7, 8), [255, 256, 257], [4, 4, 4]),
    (2, 128, (6, 12), [700], [31]),
    (4, 64, (8, 8), [300, 513], [7, 12]),
    (10, 128, (12, 20), [2000], [2]),
    (40, 128, (8, 8), [64], [3]),
    (8, 64, (6, 12), [17, 0, 700, 1, 192, 65], [30, 8, 16, 201, 64, 90]),   # long and short streams together
    (4, 128, (8, 8), [1000, 1, 30], [20, 70, 3]),
    (2, 128, (8, 8), [1] * 30 + [40], [1] * 30 + [2]),         # spans of a few tiles, a wave each
    (2, 64, (8, 8), [5, 9], [30, 31]),
]


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("H,d,lat,rows,cached", ATTN)
def test_attention(A, bits, H, d, lat, rows, cached):
    T = lat[0] * lat[1]
    lens = [c * T + m for c, m in zip(cached, rows)]
    pool = Pool(A, H, d, lat, 1, bits, lens, seed=2)       # (unwritten bytes are NaN codes and scales)
    held = pool.fill(lens, 21)
    q = normal_bf16(make_rng(22), (sum(rows), H, d))
    o = _attend(A, pool, rows, [c * T for c in cached], dev_bf16(q.reshape(-1, H * d)))
    _sync()
    got = host_f32(o).astype(np.float64).reshape(-1, H, d)
    at = 0
    for b, m in enumerate(rows):
        pick = np.unique(np.concatenate([np.arange(m)[:40], np.arange(m)[-40:], np.arange(0, m, 7)]))
        if m:
            _check_attention(got[at + pick], q[at + pick].astype(np.float64), *held[b])
        at += m


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("d,rows", [(64, [3, 40]), (128, [3, 300])])
def test_what_lies_outside_does_not_matter(A, bits, d, rows):
    """The padding, tokens past the last and other pages: NaN codes and scales, or zeros."""
    lat, T, H = (6, 12), 72, 2
    cached = [2, 5]
    lens = [c * T + m for c, m in zip(cached, rows)]
    out = []
    q = normal_bf16(make_rng(32), (sum(rows), H * d))
    for fill in (0xFF, 0x00, 0x7F):
        pool = Pool(A, H, d, lat, 1, bits, lens, seed=4, fill=fill)
        pool.fill(lens, 31)
        o = _attend(A, pool, rows, [c * T for c in cached], dev_bf16(q))
        _sync()
        out.append(host_bits(o))
        assert np.isfinite(host_f32(o)).all()
    assert np.array_equal(out[0], out[1]) and np.array_equal(out[0], out[2])


@pytest.mark.parametrize("rows", [2, 300])
def test_scores_far_apart_and_out_of_range(A, rows):
    """One key takes all the weight; and queries so large that scores overflow: -inf weighs nothing."""
    H, d, lat, T = 2, 128, (8, 8), 64
    n = 20 * T + rows
    pool = Pool(A, H, d, lat, 1, 8, [n], seed=6)
    held = pool.fill([n], 41, scale=40.0)
    q = normal_bf16(make_rng(42), (rows, H, d))
    o = _attend(A, pool, [rows], [20 * T], dev_bf16(q.reshape(rows, -1)))
    _sync()
    _check_attention(host_f32(o).astype(np.float64).reshape(rows, H, d), q.astype(np.float64), *held[0])
    # the first twelve frames' keys point away from the query: -inf, then finite scores
    k, v = np.ones((n, H, d)), normal_bf16(make_rng(43), (n, H, d)).astype(np.float64)
    k[:12 * T] = -(2.0 ** 100)
    k[12 * T:] *= 2.0 ** -104
    for f, page in enumerate(pool.ids[0]):
        m = min(T, n - f * T)
        pool.host.pack(page, k[f * T:f * T + m], v[f * T:f * T + m])
    pool.upload()
    q = np.full((rows, H, d), 2.0 ** 100, np.float32)
    o = _attend(A, pool, [rows], [20 * T], dev_bf16(q.reshape(rows, -1)))
    _sync()
    want = M.rounded(v[12 * T:].reshape(-1, H, d), 8, 0)      # (frames are whole tiles: the same blocks)
    _check_attention(host_f32(o).astype(np.float64).reshape(rows, H, d), np.zeros((rows, H, d)),
                     np.zeros_like(want), want)


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("rows", [3, 300])
def test_a_nan_block_stays_with_its_readers(A, bits, rows):
    """A block marked not finite makes NaN of its head's rows, of that stream, and nothing else."""
    H, d, lat, T = 3, 128, (8, 8), 64
    lens = [3 * T + rows, 2 * T + 4]
    pool = Pool(A, H, d, lat, 1, bits, lens, seed=7)
    pool.fill(lens, 51)
    q = dev_bf16(normal_bf16(make_rng(52), (rows + 4, H * d)))
    clean = _attend(A, pool, [rows, 4], [3 * T, 2 * T], q)
    pool.host.k_scales[pool.ids[0][1], 1, 17, 2] = 255
    pool.upload()
    got = _attend(A, pool, [rows, 4], [3 * T, 2 * T], q)
    _sync()
    a, b = host_f32(clean).reshape(-1, H, d), host_f32(got).reshape(-1, H, d)
    assert np.isnan(b[:rows, 1]).all()
    assert np.array_equal(a[:rows, [0, 2]], b[:rows, [0, 2]]) and np.array_equal(a[rows:], b[rows:])


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("H,d,lat,rows,cached,shared", [
    (2, 128, (8, 8), [1, 1, 1, 1], [5, 5, 6, 9], 5),
    (4, 64, (6, 12), [3, 1, 24, 0, 7, 12], [40, 41, 44, 0, 40, 57], 40),
    (2, 128, (6, 12), [1] * 40, [30] * 40, 30),
    (2, 64, (8, 8), [33, 70], [4, 6], 3),
    (2, 128, (8, 8), [0, 5, 5], [0, 9, 9], 1),                 # the first stream has no rows, nor pages
    (2, 128, (8, 8), [300, 290], [6, 5], 4),
    (2, 64, (8, 8), [7], [6], 6),
])
def test_shared_prefix(A, bits, H, d, lat, rows, cached, shared):
    """One history continued by a batch: the same answers as stream by stream."""
    T = lat[0] * lat[1]
    lens = [c * T + m for c, m in zip(cached, rows)]
    first = next(i for i, m in enumerate(rows) if m)
    order = [first] + [i for i in range(len(rows)) if i != first]
    pool = Pool(A, H, d, lat, 1, bits, [lens[i] if rows[i] else 0 for i in order], seed=8, shared=shared)
    held = pool.fill([lens[i] if rows[i] else 0 for i in order], 61, shared=shared)
    back = [order.index(i) for i in range(len(rows))]
    pool.table = pool.table[back].contiguous()
    held = [held[i] for i in back]
    q = normal_bf16(make_rng(62), (sum(rows), H, d))
    o = _attend(A, pool, rows, [c * T for c in cached], dev_bf16(q.reshape(-1, H * d)), shared)
    _sync()
    got = host_f32(o).astype(np.float64).reshape(-1, H, d)
    at = 0
    for b, m in enumerate(rows):
        if m:
            _check_attention(got[at:at + m], q[at:at + m].astype(np.float64), *held[b])
        at += m


def test_bad_table_entries_read_inside_the_pool_and_debug_checks_name_them(A):
    H, d, lat, T = 2, 64, (8, 8), 64
    pool = Pool(A, H, d, lat, 1, 8, [3 * T, 3 * T], seed=9, fill=0)
    pool.fill([3 * T, 3 * T], 71)
    good = pool.table.clone()
    q = dev_bf16(normal_bf16(make_rng(72), (6, H * d)))
    pool.table[0, 1] = -5
    pool.table[1, 2] = 1 << 29
    o = _attend(A, pool, [3, 3], [2 * T, 2 * T], q)          # (clamped into the pool)
    _sync()
    assert np.isfinite(host_f32(o)).all()
    A.ardit_debug_checks(1)
    try:
        with pytest.raises(A.ArditError) as e:
            _attend(A, pool, [3, 3], [2 * T, 2 * T], q)
        assert e.value.status == -3
        pool.table = good
        with pytest.raises(A.ArditError) as e:
            _attend(A, pool, [3, 3], [2 * T, 2 * T], q, shared=1)
        assert e.value.status == -1
        _attend(A, pool, [3, 3], [2 * T, 2 * T], q)
        _sync()
    finally:
        A.ardit_debug_checks(0)


def test_append_drops_what_a_bad_entry_names(A):
    import torch
    H, d, T = 2, 64, 64
    D = H * d
    pool = Pool(A, H, d, (8, 8), 2, 8, [2 * T], fill=0xA5)
    pool.upload()
    pool.table[0, 1] = pool.n_pages
    qkv = dev_bf16(normal_bf16(make_rng(81), (2 * T, 3 * D)))
    one = dev_bf16(np.ones(D, np.float32))
    q = torch.empty((2 * T, D), dtype=torch.bfloat16, device="cuda")
    A.ardit_kv_append_mx(None, pool.dims, A.Batch([2 * T], [0], [0]), qkv, one, one, pool.kv(), q)
    _sync()
    pool.download()
    keep = pool.ids[0][0]
    for a in (pool.host.k_codes, pool.host.v_codes, pool.host.k_scales, pool.host.v_scales):
        assert (np.delete(a, keep, 0) == 0xA5).all() and not (a[keep] == 0xA5).all()


def test_other_streams_and_the_same_bits_twice(A):
    """Two HIP streams at once with a workspace each, twice: the bits of calls one after the other."""
    import torch
    H, d, lat, T = 4, 128, (6, 12), 72
    rows, cached = [2, 40], [30, 11]
    lens = [c * T + m for c, m in zip(cached, rows)]
    pool = Pool(A, H, d, lat, 1, 4, lens, seed=10)
    pool.fill(lens, 91)
    caches = [c * T for c in cached]
    qs = [dev_bf16(normal_bf16(make_rng(92 + i), (sum(rows), H * d))) for i in range(2)]
    want = [host_bits(_attend(A, pool, rows, caches, q)) for q in qs]
    n = A.ardit_workspace_size(pool.dims, A.Batch(rows, caches))
    ws = [torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda") for _ in qs]
    out = [torch.full_like(q, float("nan")) for q in qs]
    streams = [torch.cuda.Stream() for _ in qs]
    _sync()
    for _ in range(2):
        for s, q, w, o in zip(streams, qs, ws, out):
            _attend(A, pool, rows, caches, q, stream=s, ws=w, o=o)
        _sync()
        for o, x in zip(out, want):
            assert np.array_equal(host_bits(o), x)


def test_captured_and_replayed(A):
    """Append, attention and read-back in one graph, replayed on new inputs, against eager calls."""
    import torch
    H, d, lat, T = 2, 128, (6, 12), 72
    D = H * d
    pool = Pool(A, H, d, lat, 1, 8, [6 * T], seed=12)
    pool.fill([6 * T], 101)
    batch = A.Batch([T], [5 * T], [5])
    n = A.ardit_workspace_size(pool.dims, batch)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    one = dev_bf16(np.ones(D, np.float32))
    qkv = dev_bf16(normal_bf16(make_rng(102), (T, 3 * D)))
    q, o = torch.empty((2, T, D), dtype=torch.bfloat16, device="cuda")
    k16 = torch.zeros((1, H, T, d), dtype=torch.bfloat16, device="cuda")
    v16 = torch.zeros((1, H, d, T), dtype=torch.bfloat16, device="cuda")
    t16 = dev_i32(np.zeros((1, 6), np.int32))

    def step():
        A.ardit_kv_append_mx(None, pool.dims, batch, qkv, one, one, pool.kv(), q)
        A.ardit_attn_fwd_mx(None, pool.dims, batch, q, pool.kv(), 0, o, ws, n)
        A.ardit_kv_read_mx(None, pool.dims, batch, pool.kv(), A.kv_paged(k16, v16, t16, 1, 6))

    step()
    _sync()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for i in range(3):
        qkv.copy_(dev_bf16(normal_bf16(make_rng(103 + i), (T, 3 * D))))
        for t in (q, o, k16, v16):
            t.fill_(float("nan"))
        g.replay()
        _sync()
        got = [host_bits(t).copy() for t in (q, o, k16, v16)]
        step()
        _sync()
        for a, t in zip(got, (q, o, k16, v16)):
            assert np.array_equal(a, host_bits(t)) and np.isfinite(host_f32(t)).all()


@pytest.mark.parametrize("bits", [8, 4])
def test_pages_past_four_gigabytes(A, bits):
    """A pool whose last pages lie past 2^32 bytes and whose tiles' byte offsets pass 32 bits."""
    import torch
    H, d, lat, T = 40, 128, (30, 52), 1560
    tile = 25 * 64 * H * d * bits // 8
    pages = (1 << 32) // tile + 3
    small = Pool(A, H, d, lat, 1, bits, [T + 5], seed=13, spare=0)
    held = small.fill([T + 5], 111)
    dev = [torch.full((pages,) + t.shape[1:], 0x7F, dtype=torch.uint8, device="cuda") for t in small.dev]
    for t, s in zip(dev, small.dev):
        t[pages - 2:] = s
    small.dev = dev
    small.table = small.table + (pages - 2)
    small.n_pages = pages
    q = normal_bf16(make_rng(112), (5, H, d))
    o = _attend(A, small, [5], [T], dev_bf16(q.reshape(5, -1)))
    k16 = torch.zeros((1, H, T, d), dtype=torch.bfloat16, device="cuda")
    v16 = torch.zeros((1, H, d, T), dtype=torch.bfloat16, device="cuda")
    t16 = dev_i32(np.zeros((1, 2), np.int32))
    A.ardit_kv_read_mx(None, small.dims, A.Batch([T], [0]), small.kv(), A.kv_paged(k16, v16, t16, 1, 2))
    _sync()
    got = host_f32(o).astype(np.float64).reshape(5, H, d)
    _check_attention(got, q.astype(np.float64), *held[0])
    assert np.array_equal(host_f32(k16)[0].transpose(1, 0, 2), held[0][0][:T])
    assert np.array_equal(host_f32(v16)[0].transpose(2, 0, 1), held[0][1][:T])


def test_a_chunk_written_and_attended(A):
    """The run of a denoising step: projections in, cache grown, attention out, against the whole in float64."""
    import torch
    H, d, lat, frames = 4, 128, (6, 12), 2
    D, T = H * d, 72
    L = frames * T
    pool = Pool(A, H, d, lat, frames, 8, [3 * L], seed=14, fill=0)
    pool.upload()
    rng = make_rng(121)
    one = dev_bf16(np.ones(D, np.float32))
    held_k, held_v = [], []
    for chunk in range(3):
        qkv = normal_bf16(rng, (L, 3 * D))
        q = torch.empty((L, D), dtype=torch.bfloat16, device="cuda")
        o = torch.empty_like(q)
        batch = A.Batch([L], [chunk * L], [chunk * frames])
        n = A.ardit_workspace_size(pool.dims, batch)
        ws = torch.empty(n, dtype=torch.uint8, device="cuda")
        A.ardit_kv_append_mx(None, pool.dims, batch, dev_bf16(qkv), one, one, pool.kv(), q)
        A.ardit_attn_fwd_mx(None, pool.dims, batch, q, pool.kv(), 0, o, ws, n)
        _sync()
        pool.download()
        for f in range(frames):
            k, v = pool.host.unpack(pool.ids[0][chunk * frames + f])
            held_k.append(k)
            held_v.append(v)
        _check_attention(host_f32(o).astype(np.float64).reshape(L, H, d),
                         host_f32(q).astype(np.float64).reshape(L, H, d),
                         np.concatenate(held_k), np.concatenate(held_v))
        # and the cache is that of the projections
        x = qkv.astype(np.float64)
        kr = O.rope3d(O.rms_norm(x[:, D:2 * D], 1e-6).reshape(L, H, d),
                      O.chunk_positions(frames, *lat, chunk * frames), 10000.0)
        k = np.concatenate(held_k[-frames:])
        assert np.all(np.abs(k - kr) <= np.abs(M.rounded(kr, 8) - kr) + 4e-5)


@pytest.mark.parametrize("bits", [8, 4])
def test_values_at_the_end_of_bf16(A, bits):
    """The largest numbers: 4 bits stop at 6 2^125, 8 bits round 248 2^120 and more to infinity."""
    import torch
    H, d, T = 2, 64, 64
    D = H * d
    pool = Pool(A, H, d, (8, 8), 1, bits, [T], fill=0)
    pool.upload()
    rng = make_rng(131)
    qkv = normal_bf16(rng, (T, 3 * D)).astype(np.float32)
    v = qkv[:, 2 * D:]
    end = np.float32(255 * 2.0 ** 120)           # the largest bf16 number
    v[:, 0] = end
    v[::2, 1], v[1::2, 1] = -end, np.float32(2.0 ** 126)
    v[:, 2] = np.float32(247 * 2.0 ** 120)
    v[:, 3] = np.float32(1.5 * 2.0 ** 127)       # 6 2^125 itself
    v[:, 4] = -np.float32(2.0 ** 127)
    dev = dev_bf16(qkv)
    assert np.array_equal(host_f32(dev)[:, 2 * D:2 * D + 5], v[:, :5])
    one = dev_bf16(np.ones(D, np.float32))
    q = torch.empty((T, D), dtype=torch.bfloat16, device="cuda")
    A.ardit_kv_append_mx(None, pool.dims, A.Batch([T], [0], [0]), dev, one, one, pool.kv(), q)
    k16 = torch.zeros((1, H, T, d), dtype=torch.bfloat16, device="cuda")
    v16 = torch.zeros((1, H, d, T), dtype=torch.bfloat16, device="cuda")
    A.ardit_kv_read_mx(None, pool.dims, A.Batch([T], [0]), pool.kv(),
                       A.kv_paged(k16, v16, dev_i32(np.zeros((1, 1), np.int32)), 1, 1))
    _sync()
    want = M.rounded(host_f32(dev)[:, 2 * D:].astype(np.float64).reshape(T, H, d), bits, 0)
    if bits == 8:
        assert (want[:, 0, 0] == 2.0 ** 128).all() and np.abs(want[:, 0, 2:5]).max() < 2.0 ** 128
        want = np.where(np.abs(want) == 2.0 ** 128, np.copysign(np.inf, want), want)
    else:
        assert (want[:, 0, 0] == 6 * 2.0 ** 125).all()
    assert np.array_equal(host_f32(v16)[0].transpose(2, 0, 1), want)
    pool.download()
    assert np.array_equal(host_f32(k16)[0].transpose(1, 0, 2), pool.host.unpack(pool.ids[0][0])[0])


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("rows", [3, 300])
def test_queries_that_are_not_finite_stay_rows_of_their_own(A, d, rows):
    """A NaN or an infinity in a query makes NaN of its row and head, the others are as without it."""
    H, lat, T = 2, (8, 8), 64
    pool = Pool(A, H, d, lat, 1, 8, [9 * T + rows], seed=15)
    held = pool.fill([9 * T + rows], 141)
    q = normal_bf16(make_rng(142), (rows, H, d)).astype(np.float32)
    q[1, 0, 7] = np.nan
    q[2, 1, 40] = -np.inf
    o = _attend(A, pool, [rows], [9 * T], dev_bf16(q.reshape(rows, -1)))
    _sync()
    got = host_f32(o).astype(np.float64).reshape(rows, H, d)
    assert np.isnan(got[1, 0]).all() and np.isnan(got[2, 1]).all()
    k, v = held[0]
    for h in range(H):
        rest = np.array([r for r in range(rows) if r != 1 + h])
        _check_attention(got[rest][:, h:h + 1], q[rest][:, h:h + 1].astype(np.float64), k[:, h:h + 1], v[:, h:h + 1])


@pytest.mark.parametrize("rows", [[2, 37], [300, 5]])
def test_one_page_many_times_and_rows_behind_the_last(A, rows):
    """Table entries that name a page again; arrays longer than the batch; knobs that ask for nothing."""
    import torch
    H, d, lat, T = 2, 128, (6, 12), 72
    cached = [12, 7]
    lens = [T, T]
    pool = Pool(A, H, d, lat, 1, 4, lens, seed=16)
    held = pool.fill(lens, 151)
    table = np.array([[pool.ids[0][0]] * 17, [pool.ids[1][0], pool.ids[0][0]] + [pool.ids[1][0]] * 15], np.int32)
    pool.table, pool.span = dev_i32(table), 17
    q = normal_bf16(make_rng(152), (sum(rows), H, d))
    o = torch.full((sum(rows) + 9, H * d), float("nan"), dtype=torch.bfloat16, device="cuda")
    batch = A.Batch(rows, [c * T for c in cached], sparsity=[0.0, 0.0], quant=[0, 0])
    n = A.ardit_workspace_size(pool.dims, batch)
    ws = torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")
    A.ardit_attn_fwd_mx(None, pool.dims, batch, dev_bf16(q.reshape(-1, H * d)), pool.kv(), 0, o, ws, n)
    _sync()
    assert (host_bits(o)[sum(rows):] == host_bits(torch.full_like(o[:1], float("nan")))[0]).all()
    got = host_f32(o).astype(np.float64)[:sum(rows)].reshape(-1, H, d)
    at = 0
    for b, m in enumerate(rows):
        keys = [np.concatenate([held[int(p == pool.ids[1][0])][i] for p in table[b]])[:cached[b] * T + m] for i in range(2)]
        _check_attention(got[at:at + m], q[at:at + m].astype(np.float64), *keys, independent=False)
        at += m
    # and read back: the same page to two pages of the other pool
    k16 = torch.zeros((2, H, T, d), dtype=torch.bfloat16, device="cuda")
    v16 = torch.zeros((2, H, d, T), dtype=torch.bfloat16, device="cuda")
    t16 = dev_i32(np.array([[1, 0] + [-1] * 15, [-1] * 17], np.int32))
    A.ardit_kv_read_mx(None, pool.dims, A.Batch([2 * T, 0], [0, 0]), pool.kv(), A.kv_paged(k16, v16, t16, 2, 17))
    _sync()
    for i in range(2):
        assert np.array_equal(host_f32(k16)[i].transpose(1, 0, 2), held[0][0])
        assert np.array_equal(host_f32(v16)[i].transpose(2, 0, 1), held[0][1])


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("H,rows,cached", [
    (64, [1275, 505], [120, 130]),     # more items than CUs, of two lengths: two to a CU
    (8, [4600, 4607], [440, 148]),     # the longest take the whole time: one to a CU
    (20, [4600], [100]),               # a full round, and a split one
    (64, [1280, 1024], [121, 121]),
])
def test_many_items_at_64(A, bits, H, rows, cached):
    """Chunks of narrow heads by the hundred, their keys a few pages named again and again."""
    d, lat, T = 64, (8, 8), 64
    pool = Pool(A, H, d, lat, 1, bits, [7 * T], seed=17)
    held = pool.fill([7 * T], 161)[0]
    rng = np.random.default_rng(18)
    pool.span = max(c + -(-m // T) for c, m in zip(cached, rows))
    pick = rng.integers(0, 7, (len(rows), pool.span))
    pool.table = dev_i32(np.array(pool.ids[0], np.int32)[pick])
    q = normal_bf16(make_rng(162), (sum(rows), H, d))
    o = _attend(A, pool, rows, [c * T for c in cached], dev_bf16(q.reshape(-1, H * d)))
    _sync()
    got = host_f32(o).astype(np.float64).reshape(-1, H, d)
    assert np.isfinite(got).all()
    heads = [0, 1, H // 2, H - 1]
    at = 0
    for b, m in enumerate(rows):
        k, v = [x.reshape(7, T, H, d)[:, :, heads][pick[b]].reshape(-1, len(heads), d)[:cached[b] * T + m] for x in held]
        some = at + np.unique(np.concatenate([rng.integers(0, m, 24), [0, m - 1]]))
        _check_attention(got[some][:, heads], q[some][:, heads].astype(np.float64), k, v, independent=False)
        at += m


@pytest.mark.parametrize("shared", [0, 3])
@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("rows", [[40] * 64, [1] * 64, [9, 1] * 32])
def test_as_many_streams_as_there_can_be(A, bits, rows, shared):
    """64 streams, each a run of workgroups of its own or a wave each, and a prefix that makes 65."""
    H, d, lat, T = 2, 64, (8, 8), 64
    cached = [3 + b % 5 for b in range(64)]
    lens = [c * T + m for c, m in zip(cached, rows)]
    pool = Pool(A, H, d, lat, 1, bits, lens, seed=19, shared=shared)
    held = pool.fill(lens, 171, shared=shared)
    q = normal_bf16(make_rng(172), (sum(rows), H, d))
    o = _attend(A, pool, rows, [c * T for c in cached], dev_bf16(q.reshape(-1, H * d)), shared)
    _sync()
    got = host_f32(o).astype(np.float64).reshape(-1, H, d)
    at = 0
    for b, m in enumerate(rows):
        _check_attention(got[at:at + m], q[at:at + m].astype(np.float64), *held[b])
        at += m


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("H,d,rows,cached", [
    (12, 128, [4600], [200]),               # 216 items, six tails to each idle CU
    (10, 128, [2300, 2290], [180, 180]),    # 180 of two streams
    (12, 64, [4600], [260]),
])
def test_a_round_whose_items_shed_their_tails(A, bits, H, d, rows, cached):
    """Items that leave a part of the CUs idle, their keys a few pages named again and again."""
    lat, T = (8, 8), 64
    pool = Pool(A, H, d, lat, 1, bits, [7 * T], seed=21)
    held = pool.fill([7 * T], 181)[0]
    rng = np.random.default_rng(22)
    pool.span = max(c + -(-m // T) for c, m in zip(cached, rows))
    pick = rng.integers(0, 7, (len(rows), pool.span))
    pool.table = dev_i32(np.array(pool.ids[0], np.int32)[pick])
    q = normal_bf16(make_rng(182), (sum(rows), H, d))
    o = _attend(A, pool, rows, [c * T for c in cached], dev_bf16(q.reshape(-1, H * d)))
    _sync()
    got = host_f32(o).astype(np.float64).reshape(-1, H, d)
    assert np.isfinite(got).all()
    at = 0
    for b, m in enumerate(rows):
        k, v = [x.reshape(7, T, H, d)[pick[b]].reshape(-1, H, d)[:cached[b] * T + m] for x in held]
        some = at + np.unique(np.concatenate([rng.integers(0, m, 16), [0, m - 1]]))
        _check_attention(got[some], q[some].astype(np.float64), k, v, independent=False)
        at += m
