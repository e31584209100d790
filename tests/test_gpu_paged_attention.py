"""Attention of new tokens over a paged cache, against the definition in 64 bits: sizes, types, layouts, masks, what stands where nobody looks."""
import numpy as np
import pytest
import torch

import paper_2608_03537_b200 as cf
from oracle import kv_oracle as orc
from tests import kv, parity as P

pytestmark = pytest.mark.gpu


class Call:
    """A cache with sequences in it, and a call's other tensors.  Rows of no sequence hold NaN (8 bits: large codes with NaN scales)."""

    def __init__(self, lengths, T, Hq, H, D, page, name, quantized, device, seed=0, layout="heads first", window=0, cap=0.0, slopes=False, alpha=None, spare=0, dims=4, scale=1.0):
        self.lengths, self.T, self.D, self.window, self.cap = np.asarray(lengths), T, D, window, cap
        self.alpha = D ** -0.5 if alpha is None else alpha
        B, r = len(lengths), np.random.RandomState(seed)
        g = torch.Generator(device=device).manual_seed(seed)
        need = -(-np.maximum(self.lengths, 0) // page)
        pages = int(need.sum()) + 2
        self.cache = kv.Cache(pages, H, page, D, name, quantized, device, layout)
        width = max(1, int(need.max())) + spare
        self.table = np.full((B, width), -1, np.int32)
        order, at = r.permutation(pages), 0
        for b in range(B):
            self.table[b, :need[b]] = order[at:at + need[b]]
            at += need[b]
            n = np.arange(self.lengths[b])
            if len(n):
                where = [torch.from_numpy(x).to(device) for x in (self.table[b, n // page].astype(np.int64), n % page)]
                for side in "kv":
                    x = torch.randn(len(n), H, D, device=device, generator=g)
                    if quantized:   # scales of all sizes
                        x = x * torch.exp(torch.randn(len(n), H, 1, device=device, generator=g))
                    self.cache.put(side, *where, x)
        t = kv.TYPES[name]
        wide = torch.randn(B, T, Hq + 2, D, device=device, generator=g)
        self.q = (scale * wide).to(t)[:, :, 1:Hq + 1]   # (a view: heads of a wider projection)
        self.out, self.lse = P.guarded((B, T, Hq, D), t, -77.0, device), P.guarded((B, T, Hq), torch.float32, -77.0, device)
        self.slopes = 2.0 ** (-8 * torch.arange(1, Hq + 1, dtype=torch.float32, device=device) / Hq) if slopes else None
        self.device_table, self.device_lengths = torch.from_numpy(self.table).to(device), torch.from_numpy(self.lengths.astype(np.int32)).to(device)
        self.dims = dims

    def run(self, **kw):
        one = self.dims == 3
        q, out, lse = (t[:, 0] if one else t for t in (self.q, self.out, self.lse))
        c = self.cache
        more = dict(window=self.window, max_length=kw.get("max_length"), **c.scales())
        n = cf.paged_attention_workspace_size(q, c.k, c.v, self.device_table, **more)
        assert n <= cf.PAGED_ATTENTION_WORKSPACE_BYTES
        ws = P.guarded((max(16, n),), torch.uint8, 255, q.device)
        args = dict(alpha=self.alpha, softcap=self.cap, slopes=self.slopes, lse=lse, workspace=ws, **more)
        args.update(kw)
        out = args.pop("out", out)
        assert cf.paged_attention(q, c.k, c.v, self.device_table, self.device_lengths, out, **args) is out
        torch.cuda.synchronize()
        P.check_canaries({"out": self.out, "lse": self.lse, "workspace": ws})
        c.check_canaries()

    def check(self, max_length=None):
        q, dtype = kv.f64(self.q), self.out.dtype
        # (a row that no sequence holds may be NaN: the oracle does not look at it)
        want, lse, weight = orc.attention(q, self.cache.values("k"), self.cache.values("v"), self.table, self.lengths, self.alpha, self.cap, None if self.slopes is None else kv.f64(self.slopes),
                                          self.window, max_length)
        bound, lse_bound = kv.attention_bounds(want, lse, weight, max(1, int(self.lengths.max())), self.D, dtype, self.cache.quantized, self.cap)
        got, got_lse = kv.f64(self.out), kv.f64(self.lse)
        assert np.array_equal(np.isinf(got_lse), np.isinf(lse)) and not np.isnan(got_lse).any() and not np.isnan(got).any()
        fine = np.isfinite(lse)
        assert np.all(np.abs(got_lse[fine] - lse[fine]) <= lse_bound[fine])
        assert np.all(got[~fine] == 0)
        worst = np.max(np.abs(got - want) / bound)
        assert worst <= 1, worst


TYPES = [("bf16", False), ("f16", False), ("bf16", True), ("f16", True)]
# lengths, new tokens, query heads, key heads, D, page
SHAPES = [([1], 1, 1, 1, 64, 16), ([1], 1, 8, 8, 128, 1), ([1000], 1, 32, 8, 128, 16), ([0, 5, 64, 65, 0, 200, 16, 17], 1, 4, 2, 64, 24), ([300, 7, 1, 129], 1, 12, 12, 80, 33), ([513, 40], 3, 10, 2, 96, 100),
          ([2000, 31, 1200], 1, 16, 1, 128, 64), ([700, 90], 5, 16, 2, 256, 64), ([64, 128, 192], 8, 9, 3, 128, 64), ([5000], 1, 8, 1, 256, 128), ([333, 1, 2, 3], 2, 28, 4, 64, 7), ([100, 64, 70], 64, 2, 1, 64, 16),
          ([40, 3, 90], 16, 4, 4, 112, 16), ([20], 4, 24, 1, 128, 8), ([37] * 200, 1, 2, 2, 64, 16), ([9000, 20], 1, 20, 4, 48, 16)]


@pytest.mark.parametrize("name,quantized", TYPES)
@pytest.mark.parametrize("lengths,T,Hq,H,D,page", SHAPES)
def test_attention(lengths, T, Hq, H, D, page, name, quantized, cuda_device):
    c = Call(lengths, T, Hq, H, D, page, name, quantized, cuda_device, seed=Hq + D)
    c.run()
    c.check()


@pytest.mark.parametrize("name,quantized", TYPES)
@pytest.mark.parametrize("window,cap,slopes,T,D", [(1, 0.0, False, 1, 64), (17, 0.0, True, 3, 128), (64, 5.0, False, 1, 256), (300, 30.0, True, 8, 64), (0, 2.0, True, 1, 128), (2 ** 31 - 1, 0.0, True, 4, 128),
                                                  (500, 0.0, False, 2, 96)])
def test_masks_caps_and_slopes(window, cap, slopes, T, D, name, quantized, cuda_device):
    c = Call([800, 0, 3, 64, 300, 129], T, 6, 3, D, 24, name, quantized, cuda_device, seed=window % 1000, window=window, cap=cap, slopes=slopes)
    c.run()
    c.check()


@pytest.mark.parametrize("name,quantized", TYPES)
@pytest.mark.parametrize("layout", ["rows first", "padded"])
def test_layouts(layout, name, quantized, cuda_device):
    for page in (16, 10):
        c = Call([200, 33, 70], 1, 8, 4, 128, page, name, quantized, cuda_device, seed=page, layout=layout, spare=3, dims=3)
        c.run()
        c.check()


@pytest.mark.parametrize("quantized", [False, True])
@pytest.mark.parametrize("page", [16, 20])
def test_keys_and_values_laid_out_differently(page, quantized, cuda_device):
    """Keys [pages, heads, page, D], values [pages, page, heads, D], scales with strides of their own."""
    c = Call([300, 41, 128], 2, 6, 3, 64, page, "f16", quantized, cuda_device, seed=8)
    c.run()
    first = c.out.clone()
    c.cache.v = c.cache.v.transpose(1, 2).contiguous().transpose(1, 2)
    if quantized:
        c.cache.ks = c.cache.ks.transpose(0, 2).contiguous().transpose(0, 2)
    for t in (c.cache.v, c.cache.ks):
        if t is not None:
            t._base_tensor = t
    c.cache.check_canaries = lambda label="": None
    c.run()
    c.check()
    assert torch.equal(first, c.out)


@pytest.mark.parametrize("quantized", [False, True])
@pytest.mark.parametrize("D", [8, 16, 40, 72, 136, 176, 248])
def test_unusual_widths(D, quantized, cuda_device):
    if quantized and D % 16:
        return
    c = Call([300, 0, 77, 1], 2, 12, 2, D, 16, "bf16", quantized, cuda_device, seed=D, slopes=True)
    c.run()
    c.check()


@pytest.mark.parametrize("quantized", [False, True])
@pytest.mark.parametrize("T,Hq,H,D", [(1, 8, 2, 128), (4, 16, 2, 64), (7, 28, 2, 128), (3, 6, 3, 256)])
def test_outputs_over_the_queries(T, Hq, H, D, quantized, cuda_device):
    c = Call([2000, 0, 300, 45, 1000], T, Hq, H, D, 16, "bf16", quantized, cuda_device, seed=T)
    c.run()
    first, own = c.out.clone(), c.q.clone()
    c.run(out=c.q)
    assert torch.equal(c.q, first)
    c.q.copy_(own)
    c.check()


def test_many_sequences(cuda_device):
    """More sequences than a CTA has threads, most of them short, some empty."""
    r = np.random.RandomState(2)
    lengths = np.where(r.rand(1500) < 0.1, 0, np.ceil(2.0 ** r.uniform(0, 7, 1500))).astype(np.int64)
    c = Call(lengths, 1, 2, 1, 64, 16, "bf16", False, cuda_device, seed=6)
    c.run()
    c.check()


@pytest.mark.parametrize("name,quantized", TYPES)
def test_large_scores(name, quantized, cuda_device):
    """Scores hundreds apart, rising and falling along the sequence: the running maximum is renewed again and again."""
    c = Call([700, 250], 2, 8, 2, 64, 16, name, quantized, cuda_device, seed=3, scale=12.0, alpha=1.0)
    c.run()
    c.check()
    c.alpha = -1.0
    c.run()
    c.check()


@pytest.mark.parametrize("quantized", [False, True])
def test_maximum_length_and_bad_lengths(quantized, cuda_device):
    """Lengths beyond the limit, or the table, are cut; negative ones are empty; pages that are none hold nothing."""
    c = Call([300, 120, 64, 90], 1, 4, 2, 64, 16, "bf16", quantized, cuda_device, seed=1)
    c.run(max_length=100)
    c.check(max_length=100)
    last = torch.arange(10, 16, device=cuda_device)   # rows of the last sequence's last page that no token has written: a longer length sees them
    for side in "kv":
        c.cache.put(side, torch.full_like(last, int(c.table[3, 5])), last, torch.randn(6, 2, 64, device=cuda_device))
    full = c.lengths
    c.lengths = np.array([300, -5, 64, 2 ** 31 - 1])
    c.device_lengths = torch.tensor(c.lengths, dtype=torch.int32, device=cuda_device)
    c.run()
    c.lengths = np.array([300, 0, 64, c.table.shape[1] * 16])     # (the last one's table ends in -1)
    c.check()
    c.lengths = full
    c.device_lengths = torch.from_numpy(full.astype(np.int32)).to(cuda_device)
    c.table[0, 3], c.table[1, :], c.table[2, 1], c.table[3, 0] = -1, 10 ** 6, -2 ** 31, 2 ** 31 - 1
    c.device_table = torch.from_numpy(c.table).to(cuda_device)
    c.run()
    c.check()


@pytest.mark.parametrize("quantized", [False, True])
def test_a_sequence_shorter_than_its_new_tokens(quantized, cuda_device):
    """Tokens in front of position 0 see nothing."""
    c = Call([3, 8, 1, 0], 8, 4, 2, 64, 16, "bf16", quantized, cuda_device)
    c.run()
    c.check()
    assert torch.all(c.out[0, :5] == 0) and torch.all(torch.isinf(c.lse[0, :5]))


@pytest.mark.parametrize("name", ["bf16", "f16"])
@pytest.mark.parametrize("quantized", [False, True])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_what_a_token_does_not_see_does_not_reach_it(bad, quantized, name, cuda_device):
    """The last new token's key or value (or scale) is not finite: the tokens before it are as without it."""
    for side in "kv":
        c = Call([50, 130, 17], 4, 4, 2, 64, 16, name, quantized, cuda_device, seed=2)
        for b, n in enumerate(c.lengths):
            page, row = c.table[b, (n - 1) // 16], (n - 1) % 16
            cache, scale = (c.cache.k, c.cache.ks) if side == "k" else (c.cache.v, c.cache.vs)
            if quantized:
                scale[page, :, row] = bad
            else:
                cache[page, :, row, 5] = bad
        c.run()
        got = kv.f64(c.out)
        assert np.isfinite(got[:, :3]).all() and not np.isfinite(got[:, 3]).all()
        values = {s: c.cache.values(s) for s in "kv"}
        want, lse, weight = orc.attention(kv.f64(c.q)[:, :3], values["k"], values["v"], c.table, c.lengths - 1, c.alpha)
        bound, _ = kv.attention_bounds(want, lse, weight, 130, 64, c.out.dtype, quantized)
        assert np.all(np.abs(got[:, :3] - want) <= bound)


@pytest.mark.parametrize("name", ["bf16", "f16"])
def test_what_a_window_hides(name, cuda_device):
    """Positions in front of the window, in the same pages, are not finite."""
    c = Call([200, 64, 300], 3, 4, 2, 128, 64, name, False, cuda_device, seed=4, window=20)
    for b, n in enumerate(c.lengths):
        for pos in range(n - 3 + 1 - 20):
            for t in (c.cache.k, c.cache.v):
                t[c.table[b, pos // 64], :, pos % 64] = float("nan")
    c.run()
    got = kv.f64(c.out)
    assert np.isfinite(got).all()
    keys, values = np.nan_to_num(c.cache.values("k")), np.nan_to_num(c.cache.values("v"))
    want, lse, weight = orc.attention(kv.f64(c.q), keys, values, c.table, c.lengths, c.alpha, window=20)
    bound, _ = kv.attention_bounds(want, lse, weight, 300, 128, c.out.dtype, False)
    assert np.all(np.abs(got - want) <= bound)


@pytest.mark.parametrize("quantized", [False, True])
def test_a_visible_nan_reaches_its_rows_alone(quantized, cuda_device):
    c = Call([100, 100], 1, 4, 2, 64, 16, "bf16", quantized, cuda_device)
    if quantized:
        c.cache.vs[c.table[0, 2], 1, 3] = float("nan")
    else:
        c.cache.v[c.table[0, 2], 1, 3] = float("nan")
    c.run()
    assert torch.isnan(c.out[0, :, 2:]).all() and torch.isfinite(c.out[0, :, :2]).all() and torch.isfinite(c.out[1]).all() and torch.isfinite(c.lse).all()


def test_values_and_scales_of_all_sizes(cuda_device):
    """8 bits: rows with scales from 2^-100 to 2^100, the largest last, first and in the middle."""
    for turn in (1, -1, 3):
        c = Call([64 * 5], 1, 4, 1, 64, 16, "bf16", True, cuda_device)
        exponents = (np.arange(320) * turn % 320 - 160) * 200 / 320
        pos = np.arange(320)
        c.cache.vs[c.table[0, pos // 16], 0, pos % 16] = torch.from_numpy(2.0 ** exponents).float().to(cuda_device)
        c.run()
        values = c.cache.values("v")
        want, lse, weight = orc.attention(kv.f64(c.q), c.cache.values("k"), values, c.table, c.lengths, c.alpha)
        bound, _ = kv.attention_bounds(want, lse, weight, 320, 64, torch.bfloat16, True)
        assert np.all(np.abs(kv.f64(c.out) - want) <= bound)


def test_offsets_beyond_32_bits(cuda_device):
    """Pages behind 2^31 elements."""
    pages, page, D = 150000, 64, 256
    if torch.cuda.mem_get_info()[0] < 12 << 30:
        pytest.skip("not enough free memory")
    cache = torch.zeros(pages, 1, page, D, dtype=torch.bfloat16, device=cuda_device)
    small = torch.randn(4, 1, page, D, device=cuda_device).bfloat16()
    far = [pages - 1, pages - 3, 2, pages - 2]
    for i, n in enumerate(far):
        cache[n] = small[i]
    q = torch.randn(1, 4, D, device=cuda_device).bfloat16()
    got = []
    for c, table in ((cache, far), (small, [0, 1, 2, 3])):
        out = torch.zeros_like(q)
        ws = torch.empty(cf.PAGED_ATTENTION_WORKSPACE_BYTES, dtype=torch.uint8, device=cuda_device)
        cf.paged_attention(q, c, c, torch.tensor([table], dtype=torch.int32, device=cuda_device), torch.tensor([250], dtype=torch.int32, device=cuda_device), out, workspace=ws)
        got.append(out)
    assert torch.equal(*got) and got[0].abs().sum() > 0
    del cache


def test_same_bits_again_and_whatever_the_workspace_held(cuda_device):
    c = Call([4000, 77, 900], 2, 16, 2, 128, 16, "bf16", False, cuda_device, seed=9)
    first = []
    for fill in (0, 255, 127):
        n = cf.paged_attention_workspace_size(c.q, c.cache.k, c.cache.v, c.device_table)
        ws = torch.full((n,), fill, dtype=torch.uint8, device=cuda_device)
        c.run(workspace=ws)
        first.append((c.out.clone(), c.lse.clone()))
    c.check()
    assert all(torch.equal(a, first[0][0]) and torch.equal(l, first[0][1]) for a, l in first)


def test_graphs_that_share_a_workspace_and_calls_on_two_streams(cuda_device):
    """Two captured calls on one workspace, replayed one behind the other with other lengths; and two calls at once, with a workspace each."""
    a, b = Call([900, 64], 1, 8, 2, 128, 16, "bf16", False, cuda_device, seed=1), Call([30, 2000, 5], 1, 6, 6, 64, 16, "bf16", True, cuda_device, seed=2)
    ws = [torch.empty(cf.PAGED_ATTENTION_WORKSPACE_BYTES, dtype=torch.uint8, device=cuda_device) for _ in range(2)]

    def call(c, w, stream=None):
        cf.paged_attention(c.q, c.cache.k, c.cache.v, c.device_table, c.device_lengths, c.out, lse=c.lse, workspace=w, stream=stream, **c.cache.scales())

    call(a, ws[0])
    call(b, ws[0])
    graphs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
    for c, graph in zip((a, b), graphs):
        with torch.cuda.graph(graph):
            call(c, ws[0])
    a.lengths, b.lengths = np.array([700, 3]), np.array([30, 1500, 0])
    for c in (a, b):
        c.device_lengths.copy_(torch.from_numpy(c.lengths.astype(np.int32)))
        c.out.fill_(-77)
    for _ in range(3):
        for graph in graphs:
            graph.replay()
    torch.cuda.synchronize()
    for c in (a, b):
        c.check()
        c.out.fill_(-77)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(5):
        call(a, ws[0])
        call(b, ws[1], stream=side)
    torch.cuda.synchronize()
    for c in (a, b):
        c.check()


def test_refusals(cuda_device):
    c = Call([100, 20], 2, 4, 2, 64, 16, "bf16", False, cuda_device, spare=4000)   # (room for long sequences: a call that needs a workspace)
    before = c.out.clone()
    n = cf.paged_attention_workspace_size(c.q, c.cache.k, c.cache.v, c.device_table)
    assert n > 0
    ws = torch.empty(n + 16, dtype=torch.uint8, device=cuda_device)
    q8 = kv.Cache(9, 2, 16, 64, "bf16", True, cuda_device)

    def call(q=c.q, k=c.cache.k, v=c.cache.v, table=c.device_table, lengths=c.device_lengths, out=c.out, workspace=ws, **kw):
        cf.paged_attention(q, k, v, table, lengths, out, workspace=workspace, **kw)

    for kw in (dict(q=c.q.half()), dict(out=c.out.half()), dict(k=c.cache.k.half()), dict(table=c.device_table.long()), dict(lengths=c.device_lengths[:1]), dict(lengths=c.device_lengths.long()), dict(q=c.q[..., :32]),
               dict(out=c.out[:, :1]), dict(slopes=torch.ones(3, device=cuda_device)), dict(lse=torch.ones(2, 2, 5, device=cuda_device)), dict(k=q8.k, v=q8.v), dict(table=c.device_table.cpu()),
               dict(q=c.q.float(), out=c.out.float()), dict(workspace=ws.cpu()), dict(window=-1), dict(max_length=0), dict(k=q8.k, v=q8.v, k_scale=q8.ks, v_scale=q8.vs.half())):
        with pytest.raises(AssertionError):
            call(**kw)
    q3 = torch.zeros(2, 2, 3, 64, dtype=torch.bfloat16, device=cuda_device)
    long = torch.zeros(2, 65, 4, 64, dtype=torch.bfloat16, device=cuda_device)
    for kw, status in ((dict(q=q3, out=q3.clone()), cf.ERR_INVALID_ARG), (dict(workspace=None), cf.ERR_WORKSPACE), (dict(workspace=ws[:n - 1]), cf.ERR_WORKSPACE), (dict(workspace=ws[8:]), cf.ERR_ALIGNMENT),
                       (dict(softcap=-1.0), cf.ERR_INVALID_ARG), (dict(alpha=float("nan")), cf.ERR_INVALID_ARG), (dict(q=long, out=long.clone()), cf.ERR_UNSUPPORTED)):
        with pytest.raises(cf.ComfuseError) as e:
            call(**kw)
        assert e.value.status == status, kw
    torch.cuda.synchronize()
    assert torch.equal(c.out, before)
