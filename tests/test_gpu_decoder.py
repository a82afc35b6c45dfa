"""The operators around the GEMVs on the GPU against the 64-bit oracle.

Tolerances, from the operators' own roundings (fp16 rounds to 2^-11 relative, and to 2^-25 absolute
below 2^-14; fp32 to 2^-24):
 - cache codes and their powers of two without norms: equal (every step is exact or one fp32 rounding
   that the test repeats). fp16 rows with norms or rotation: 2^-11 relative, plus 8 fp32 roundings of
   the values that enter.
 - reading back: exact.
 - attention: the weights are rounded to fp16, 2^-11 of sum p |v| / sum p; the logits' fp32 error e_z
   (products of D terms and the scale: (D + 4) 2^-24 sum |q k| scale, at most 2^-9 here, doubled by
   the quotient) enters as a relative error of each weight; the result is rounded to fp16 once. The
   bound taken is (2^-11 + 2 e_z + 2^-18) spread + 2^-11 |out| + n 2^-25 max|v| (weights below fp16's
   normal range, against a sum of at least 1) + 2^-24.
 - norms: fp32 sums of n squares in any order, (n/64 + 16) 2^-24 relative at most twice over, and
   the rounding of the output's type.
"""
import numpy as np
import pytest

from oracle import decoder as od

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

FMTS = {"f16": od.F16, "fp8": od.FP8, "fp4": od.FP4}


@pytest.fixture(scope="module")
def qt():
    import paper_2609_00224_gb300 as m
    m.load()
    return m


def gpu(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t if dtype is None else t.to(dtype)


class Case:
    """A cache of random rows, all other memory filled with the worst bits (NaN), and its batch."""

    def __init__(self, qt, fmt, q_len, ctx_len, hq, hkv, dim, page, seed=0, max_q=None, extra_pages=2, poison=True):
        rng = np.random.default_rng(seed)
        self.qt, self.fmt, self.q_len, self.ctx_len, self.hq, self.hkv, self.dim, self.page = (
            qt, FMTS[fmt], q_len, ctx_len, hq, hkv, dim, page)
        self.rng = rng
        counts = [-(-max(c, 0) // page) for c in ctx_len]
        n_pages = sum(counts) + extra_pages
        order = rng.permutation(n_pages)
        self.pages, at = [], 0
        for c in counts:
            self.pages.append(order[at:at + c])
            at += c
        row = dim if self.fmt != od.FP4 else dim // 2
        shape = (n_pages, hkv, page, row)
        self.pool, self.scales, self.seq = {}, {}, {"k": [], "v": []}
        for side in "kv":
            if self.fmt == od.F16:
                pool = np.full(shape, np.nan if poison else 0, dtype=np.float16)
            else:
                pool = np.full(shape, 0x7f, dtype=np.uint8)  # E4M3: NaN
            sc = None if self.fmt == od.F16 else np.full((n_pages, hkv, page, dim // 32), 143, dtype=np.uint8)
            for s, c in enumerate(ctx_len):
                c = max(c, 0)
                x = rng.standard_normal((c, hkv, dim)) * (2.0 if side == "k" else 1.0)
                codes, scale = od.encode(x, self.fmt)
                for p in range(c):
                    pool[self.pages[s][p // page], :, p % page] = codes[p]
                    if sc is not None:
                        sc[self.pages[s][p // page], :, p % page] = scale[p]
                self.seq[side].append(od.decode(codes, scale, self.fmt))
            self.pool[side], self.scales[side] = pool, sc
        most = max([len(p) for p in self.pages] + [1])
        table = np.full((len(q_len), most), -7, dtype=np.int32)  # never followed out of the cache
        for s, p in enumerate(self.pages):
            table[s, :len(p)] = p
        self.table = table
        self.starts = np.concatenate(([0], np.cumsum(q_len))).astype(np.int32)
        self.tokens = int(self.starts[-1])
        self.t = {side: gpu(self.pool[side]) for side in "kv"}
        self.ts = {side: None if self.scales[side] is None else gpu(self.scales[side]) for side in "kv"}
        self.cache = qt.KVCache(self.t["k"], self.t["v"], self.ts["k"], self.ts["v"], fmt=self.fmt)
        self.batch = qt.KVBatch(gpu(self.starts), gpu(np.array(ctx_len, dtype=np.int32)), gpu(table), self.tokens,
                                max_q or max(list(q_len) + [1]))


def check_attention(c, window=0, scale=None, q_scale=1.0, lse=True):
    scale = c.dim ** -0.5 if scale is None else scale
    q = (c.rng.standard_normal((c.tokens, c.hq, c.dim)) * q_scale).astype(np.float16)
    ws = c.qt.attention_workspace()
    lse_t = torch.full((c.tokens, c.hq), float("nan"), device="cuda") if lse else None
    out = torch.full((c.tokens, c.hq, c.dim), float("nan"), dtype=torch.float16, device="cuda")
    c.qt.qtea_attention(c.cache, c.batch, gpu(q), scale=scale, window=window, out=out, lse=lse_t)
    again = c.qt.qtea_attention(c.cache, c.batch, gpu(q), scale=scale, window=window)
    torch.cuda.synchronize()
    assert c.qt.qtea_attention_status(ws) == 0
    assert torch.equal(out.view(torch.int16), again.view(torch.int16)), "not reproducible"
    got = out.cpu().numpy().astype(np.float64)
    ref, ref_lse, spread = od.attention(q, c.seq["k"], c.seq["v"], c.q_len, c.ctx_len, scale, window)
    e_z = 0.0
    for s in range(len(c.q_len)):
        if len(c.seq["k"][s]) and c.q_len[s]:
            rows = np.abs(q[c.starts[s]:c.starts[s + 1]].astype(np.float64))
            group = c.hq // c.hkv
            for h in range(c.hkv):
                z = rows[:, h * group:(h + 1) * group].reshape(-1, c.dim) @ np.abs(c.seq["k"][s][:, h]).T
                e_z = max(e_z, (c.dim + 4) * 2.0 ** -24 * float(z.max()) * abs(scale))
    vmax = max([float(np.abs(v).max()) for v in c.seq["v"] if v.size] + [0.0])
    n = max(list(c.ctx_len) + [0])
    lim = (2.0 ** -11 + 2 * e_z + 2.0 ** -18) * spread + 2.0 ** -11 * np.abs(ref) + n * 2.0 ** -25 * vmax + 2.0 ** -24
    err = np.abs(got - ref)
    assert np.all(np.isfinite(got)) and np.all(err <= lim), f"worst {np.nanmax(err / lim):.3g} of the bound"
    if lse:
        gl = lse_t.cpu().numpy().astype(np.float64)
        empty = ~np.isfinite(ref_lse)
        assert np.all(gl[empty] == -np.inf)
        gl, rl = gl[~empty], ref_lse[~empty]
        assert np.all(np.abs(gl - rl) <= 2 * e_z + 2.0 ** -18 * (1 + np.abs(rl)))


ATT = [
    # name, q_len, ctx_len, hq, hkv, dim, page, window
    ("one token", [1], [1], 4, 2, 128, 16, 0),
    ("one sequence, page's last", [1], [64], 32, 8, 128, 16, 0),
    ("odd context", [1], [517], 32, 8, 128, 32, 0),
    ("group of 5, ragged", [1, 1, 1, 1], [300, 1, 129, 63], 40, 8, 128, 64, 0),
    ("group of 8", [1, 1], [1000, 77], 16, 2, 128, 128, 0),
    ("group of 1", [1, 1, 1], [90, 200, 33], 3, 3, 64, 16, 0),
    ("group of 12", [1, 2], [40, 200], 24, 2, 64, 32, 0),
    ("group of 16, two tokens", [2, 1], [130, 64], 16, 1, 128, 16, 0),
    ("group of 32", [1, 3], [70, 150], 32, 1, 128, 16, 0),
    ("few tokens", [3, 1, 4, 2], [100, 50, 4, 65], 8, 2, 128, 16, 0),
    ("16 tokens, group 4", [16, 7], [200, 16], 8, 2, 128, 32, 0),
    ("empty rows", [5, 1, 3], [2, 0, 1], 8, 2, 128, 16, 0),
    ("no tokens for some", [0, 3, 0], [40, 30, 0], 8, 2, 64, 16, 0),
    ("window inside a page", [1, 4], [500, 90], 8, 2, 128, 64, 5),
    ("window of one", [2, 1], [40, 17], 8, 2, 64, 16, 1),
    ("window over pages", [6], [400], 8, 2, 128, 16, 100),
    ("window wider than all", [2], [40], 8, 2, 128, 16, 1000),
    ("a prompt", [150], [150], 8, 2, 128, 16, 0),
    ("a chunk after others", [70, 1, 130], [300, 9, 131], 8, 2, 64, 32, 0),
    ("a windowed prompt", [140], [200], 8, 4, 128, 16, 37),
    ("a prompt, group of 5", [60], [60], 10, 2, 128, 16, 0),
    ("16 tokens, group of 8", [16, 16, 16], [300, 16, 129], 16, 2, 128, 64, 0),
    ("prompt and decode steps", [200, 1, 1, 33], [200, 700, 3, 40], 8, 2, 128, 32, 0),
    ("small chunk over many units", [40, 3], [3000, 2000], 4, 1, 128, 64, 0),
    ("two row tiles over many units", [70], [1800], 4, 1, 64, 128, 0),
    ("windows through row tiles", [130, 90], [500, 90], 4, 1, 64, 16, 64),
    ("nine tokens, group of 32", [9], [100], 32, 1, 64, 16, 0),
    ("a chunk with empty rows", [50, 40], [20, 0], 4, 2, 64, 16, 0),
    ("many sequences", [1] * 70, list(range(1, 71)), 4, 1, 64, 16, 0),
]


@pytest.mark.parametrize("fmt", list(FMTS))
@pytest.mark.parametrize("case", ATT, ids=[c[0] for c in ATT])
def test_attention(qt, fmt, case):
    _, q_len, ctx, hq, hkv, dim, page, window = case
    check_attention(Case(qt, fmt, q_len, ctx, hq, hkv, dim, page, seed=len(ctx) + dim), window)


@pytest.mark.parametrize("fmt", list(FMTS))
def test_attention_long_context_is_split(qt, fmt):
    check_attention(Case(qt, fmt, [1, 2], [9001, 30], 8, 2, 128, 64, seed=9))


def test_attention_large_logits_and_negative_scale(qt):
    c = Case(qt, "f16", [2, 1], [150, 70], 8, 2, 128, 16, seed=2)
    check_attention(c, q_scale=8.0)
    check_attention(c, scale=-0.2)
    check_attention(c, scale=0.0)


@pytest.mark.parametrize("fmt", list(FMTS))
@pytest.mark.parametrize("dim", [64, 128])
def test_chunk_attention_large_logits_scales_and_alignment(qt, fmt, dim):
    c = Case(qt, fmt, [100, 33], [400, 50], 4, 1, dim, 16, seed=31)
    check_attention(c, q_scale=8.0)  # rows whose maximum grows by far more than fp16's range from unit to unit
    check_attention(c, scale=-0.2)
    check_attention(c, scale=0.0)
    q = torch.randn(c.tokens, 4, dim, device="cuda").half()
    ref = qt.qtea_attention(c.cache, c.batch, q)
    flat = torch.zeros(c.tokens * (4 * dim + 2) + 2, device="cuda").half()
    odd = flat[2:].view(c.tokens, 4 * dim + 2)[:, :4 * dim].unflatten(1, (4, dim))  # 4-byte aligned rows
    odd.copy_(q)
    out = torch.zeros_like(flat)[2:].view(c.tokens, 4 * dim + 2)[:, :4 * dim].unflatten(1, (4, dim))
    qt.qtea_attention(c.cache, c.batch, odd, out=out)
    assert torch.equal(out, ref)


def test_chunk_attention_last_keys_dominate(qt):
    """Keys that grow with their position: every unit outruns the reference of the one before."""
    c = Case(qt, "f16", [40], [700], 4, 1, 128, 16, seed=32)
    for p in range(700):
        row = (c.seq["k"][0][p] * (1 + p / 40)).astype(np.float16)
        c.seq["k"][0][p] = row.astype(np.float64)
        c.t["k"][c.pages[0][p // 16], :, p % 16] = gpu(row)
    check_attention(c)


def test_attention_into_its_queries_and_strided_rows(qt):
    c = Case(qt, "fp8", [2, 3], [50, 40], 8, 2, 128, 16, seed=3)
    wide = torch.randn(c.tokens, 12, 128, device="cuda").half()
    q = wide[:, 2:10]
    ref = qt.qtea_attention(c.cache, c.batch, q.contiguous())
    got = torch.zeros(c.tokens, 20, 128, device="cuda").half()
    qt.qtea_attention(c.cache, c.batch, q, out=got[:, 5:13])
    assert torch.equal(got[:, 5:13], ref) and not got[:, :5].any() and not got[:, 13:].any()
    qt.qtea_attention(c.cache, c.batch, q, out=q)
    assert torch.equal(q, ref)


def test_attention_rows_of_no_sequence_are_untouched_and_long_ones_are_cut(qt):
    c = Case(qt, "f16", [4, 2], [40, 30], 8, 2, 64, 16, seed=4)
    q = torch.randn(c.tokens + 3, 8, 64, device="cuda").half()
    full = qt.qtea_attention(c.cache, c.batch, q[:c.tokens])
    b = qt.KVBatch(c.batch.q_start, c.batch.ctx_len, c.batch.pages, c.tokens + 3, 2)  # at most 2 tokens each
    out = torch.full_like(q, 7.0)
    qt.qtea_attention(c.cache, b, q, out=out)
    assert torch.equal(out[[0, 1, 4, 5]], full[[0, 1, 4, 5]])
    assert (out[[2, 3, 6, 7, 8]] == 7.0).all()


def test_attention_lengths_and_pages_out_of_range_are_bounded(qt):
    """Lengths past the table, negative ones, pages outside the cache: results are unspecified, the call
    reads nothing outside the cache (addresses are clamped in the kernel) and others' rows stay right."""
    c = Case(qt, "f16", [1, 1, 1], [64, 64, 64], 8, 2, 128, 16, seed=5)
    q = torch.randn(3, 8, 128, device="cuda").half()
    table = c.batch.pages.clone()
    table[0] = torch.tensor([1 << 30, -(1 << 30), 2, c.cache.n_pages], dtype=torch.int32, device="cuda")
    ctx = torch.tensor([1 << 30, -5, 64], dtype=torch.int32, device="cuda")
    out = qt.qtea_attention(c.cache, qt.KVBatch(c.batch.q_start, ctx, table, 3, 1), q)
    assert not out[1].any()
    # the others' lengths change how the work is split, so the third row is held to its own bound
    ref, _, spread = od.attention(q[2:].cpu().numpy(), c.seq["k"][2:], c.seq["v"][2:], [1], [64], 128 ** -0.5)
    err = np.abs(out[2:].cpu().numpy().astype(np.float64) - ref)
    assert np.all(err <= (2.0 ** -11 + 2.0 ** -12) * spread + 2.0 ** -11 * np.abs(ref) + 2.0 ** -16)


def test_attention_replays_in_a_graph_with_other_lengths(qt):
    c = Case(qt, "fp8", [1, 1], [200, 90], 8, 2, 128, 16, seed=6)
    q = torch.randn(2, 8, 128, device="cuda").half()
    out = torch.empty_like(q)
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        qt.qtea_attention(c.cache, c.batch, q, out=out)
    s.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        qt.qtea_attention(c.cache, c.batch, q, out=out)
    for lens in ([200, 90], [17, 90], [1, 64]):
        c.batch.ctx_len.copy_(torch.tensor(lens, dtype=torch.int32))
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, qt.qtea_attention(c.cache, c.batch, q))


def test_attention_captured_on_a_stream_without_a_workspace(qt):
    """The first call of a stream under capture: no graph's workspace waits for another graph's replay."""
    c = Case(qt, "f16", [1, 1], [4000, 900], 8, 2, 128, 32, seed=8)
    q = torch.randn(2, 8, 128, device="cuda").half()
    ref = qt.qtea_attention(c.cache, c.batch, q)
    s = torch.cuda.Stream()
    outs, graphs = [torch.zeros_like(q) for _ in range(3)], []
    for out in outs[:2]:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            qt.qtea_attention(c.cache, c.batch, q, out=out)
            qt.qtea_attention(c.cache, c.batch, q, out=out)
        graphs.append(g)
    with torch.cuda.stream(s):
        qt.qtea_attention(c.cache, c.batch, q, out=outs[2])
    torch.cuda.synchronize()
    for g in reversed(graphs):
        g.replay()
        g.replay()
        torch.cuda.synchronize()
    assert all(torch.equal(out, ref) for out in outs)


@pytest.mark.parametrize("fmt", list(FMTS))
@pytest.mark.parametrize("rows", [1, 40, 150])
def test_attention_reads_no_partial_result_that_it_did_not_write(qt, fmt, rows):
    """Only the workspace's counters start as zeros: NaN in all the rest changes nothing."""
    c = Case(qt, fmt, [rows, 1], [3000, 700], 8, 2, 128, 64, seed=11)
    q = torch.randn(c.tokens, 8, 128, device="cuda").half()
    ws = torch.full((qt.attention_workspace().numel(),), 255, dtype=torch.uint8, device="cuda")
    ws[:16384] = 0
    ref = qt.qtea_attention(c.cache, c.batch, q)
    assert torch.isfinite(ref).all()
    assert torch.equal(qt.qtea_attention(c.cache, c.batch, q, workspace=ws), ref)


def test_attention_on_two_streams_with_their_own_workspaces(qt):
    c = Case(qt, "f16", [1, 1], [4000, 900], 8, 2, 128, 32, seed=7)
    q = [torch.randn(2, 8, 128, device="cuda").half() for _ in range(2)]
    ref = [qt.qtea_attention(c.cache, c.batch, x) for x in q]
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [torch.empty_like(x) for x in q]
    for s in streams:
        qt.attention_workspace(stream=s)
    torch.cuda.synchronize()
    for _ in range(20):
        for i, s in enumerate(streams):
            qt.qtea_attention(c.cache, c.batch, q[i], out=outs[i], stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, ref))


@pytest.mark.parametrize("op", ["append", "read", "attention", "norm"])
def test_outputs_on_another_stream_take_no_memory_in_use(qt, op):
    """What the current stream has still to read, though freed, is not an output of a call on another."""
    n = 12288  # 12 MB of fp16: a block of the allocator's own, taken again by what has its size
    cache = qt.KVCache.empty(n // 64, 64, 4, 128)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    batch = qt.KVBatch(i32([0, n]), i32([n]), i32([list(range(n // 64))]), n, n)
    rows = torch.randn(n, 4 * 128, device="cuda").half()
    weight, row_start = torch.ones(512, device="cuda").half(), i32([0, n])
    s = torch.cuda.Stream()
    calls = {"append": lambda **k: qt.qtea_kv_append(cache, batch, rows, rows, q=rows, stream=s,
                                                     **({"q_out": k["out"][0]} if k else {})),
             "read": lambda **k: qt.qtea_kv_read(cache, batch, row_start, n_rows=n, stream=s,
                                                 **(dict(zip(("k_out", "v_out"), k["out"])) if k else {})),
             "attention": lambda **k: qt.qtea_attention(cache, batch, rows.view(n, 4, 128), stream=s.cuda_stream,
                                                        **({"out": k["out"][0]} if k else {})),
             "norm": lambda **k: qt.qtea_norm(rows, weight, stream=s,
                                              **({"x": k["out"][0].view(n, 512)} if k else {}))}
    taken = [torch.empty(n, 4, 128, dtype=torch.float16, device="cuda") for _ in range(2)]
    copies = [torch.empty_like(t) for t in taken]
    calls["append"]()
    calls[op](out=taken)  # the kernels are loaded
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    for t in taken:
        t.fill_(7)
    torch.cuda.synchronize()
    torch.cuda._sleep(50_000_000)
    for t, copy in zip(taken, copies):
        copy.copy_(t)
    del t, taken
    out = calls[op]()
    torch.cuda.synchronize()
    assert all(bool((copy == 7).all()) for copy in copies) and out is not None


def test_offsets_past_32_bits(qt):
    """Pages more than 4 GB into the cache: written, read back and attended to as those at its start."""
    n_pages, heads, dim, page = 20000, 8, 128, 128  # 5.2 GB a side
    cache = qt.KVCache.empty(n_pages, page, heads, dim)
    x = torch.randn(200, heads * dim, device="cuda").half()
    q = torch.randn(1, 8, dim, device="cuda").half()
    q40 = torch.randn(40, 8, dim, device="cuda").half()
    got = []
    for ids in ([3, 4], [n_pages - 1, n_pages - 2]):
        make = lambda n: qt.KVBatch(torch.tensor([0, n], dtype=torch.int32, device="cuda"),  # noqa: E731
                                    torch.tensor([200], dtype=torch.int32, device="cuda"),
                                    torch.tensor([ids], dtype=torch.int32, device="cuda"), n, n)
        qt.qtea_kv_append(cache, make(200), x, 2 * x)
        k, v = qt.qtea_kv_read(cache, make(1), torch.tensor([0, 200], dtype=torch.int32, device="cuda"), n_rows=200)
        assert torch.equal(k.flatten(1), x) and torch.equal(v.flatten(1), 2 * x)
        got.append((qt.qtea_attention(cache, make(1), q), qt.qtea_attention(cache, make(40), q40)))
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])


def test_status_reports_a_timeout_once_and_clears(qt):
    n = qt.attention_workspace().numel()
    ws = torch.zeros(n, dtype=torch.uint8, device="cuda")
    ws.view(torch.int32)[0] = qt.QTEA_ERR_TIMEOUT  # as a kernel whose wait gave up would leave it
    ws.view(torch.int32)[70] = 3
    assert qt.qtea_attention_status(ws) == qt.QTEA_ERR_TIMEOUT
    assert qt.qtea_attention_status(ws) == qt.QTEA_OK and not ws.any()


def test_work_that_cannot_be_numbered_is_refused(qt):
    import ctypes
    from paper_2609_00224_gb300 import decoder as d
    c = Case(qt, "f16", [1], [5], 4, 2, 64, 16, seed=22)
    q, ws = torch.zeros(1, 4, 64, device="cuda").half(), qt.attention_workspace()
    for n_seqs, max_pages, tokens, want in [(1, (1 << 27) - 1, 100, qt.QTEA_ERR_UNSUPPORTED), (513, 1, 1, qt.QTEA_ERR_INVALID_ARG),
                                            (1, 1 << 27, 1, qt.QTEA_ERR_INVALID_ARG), (1, 0, 1, qt.QTEA_ERR_INVALID_ARG)]:
        b = d._Batch(c.batch.q_start.data_ptr(), c.batch.ctx_len.data_ptr(), c.batch.pages.data_ptr(), n_seqs, max_pages,
                     tokens, 1)
        assert qt.load().qtea_attention(c.cache.handle, ctypes.byref(b), q.data_ptr(), 256, 4, 1.0, 0, q.data_ptr(), 256,
                                        None, ws.data_ptr(), ws.numel(), None) == want


# ------------------------------------------------------------------------------- cache: write and read


def pools(c):
    return {s: c.t[s].cpu().numpy() for s in "kv"}, {s: None if c.ts[s] is None else c.ts[s].cpu().numpy() for s in "kv"}


def rotate32(x, pos, cos, sin):
    """The rotation in fp32, each product and sum rounded by itself."""
    at = np.clip(pos, 0, len(cos) - 1)
    c, s = cos[at][:, None], sin[at][:, None]
    h = x.shape[-1] // 2
    a, b = x[..., :h], x[..., h:]
    return np.concatenate((a * c - b * s, b * c + a * s), axis=-1)


@pytest.mark.parametrize("src", [torch.float32, torch.float16])
@pytest.mark.parametrize("fmt", list(FMTS))
@pytest.mark.parametrize("dim,page,hq,hkv", [(128, 16, 10, 2), (64, 64, 3, 3)])
@pytest.mark.parametrize("rotate", [False, True])
def test_append_codes_are_exact(qt, src, fmt, dim, page, hq, hkv, rotate):
    q_len, ctx = [3, 1, 40, 0, 2], [70, 1, 40, 5, 1]  # the last sequence's first token has no place
    c = Case(qt, fmt, q_len, ctx, hq, hkv, dim, page, seed=11)
    before, before_s = pools(c)
    rng = np.random.default_rng(12)
    # blocks of every size class: zeros, subnormal, tiny, ordinary, at and past the formats' ends
    mag = np.exp2(rng.integers(-30, 14, (c.tokens, hkv, dim // 32)))
    x = {n: rng.standard_normal((c.tokens, hkv, dim)) * np.repeat(mag, 32, -1) for n in "kv"}
    x["k"][0, 0, :32] = 0
    x["v"][1, 0, :32] = 6.0 * np.array([1, -1] * 16)
    x["v"][2, 0, 32:] = 5e4
    x["q"] = rng.standard_normal((c.tokens, hq, dim))
    x = {n: gpu(v.astype(np.float32)).to(src) for n, v in x.items()}
    f32 = {n: v.float().cpu().numpy() for n, v in x.items()}
    cos = sin = None
    pos = od.token_positions(q_len, ctx)
    if rotate:
        ang = rng.uniform(0, 6.28, (60, dim // 2))  # shorter than some positions: they use the last row
        cos, sin = np.cos(ang).astype(np.float32), np.sin(ang).astype(np.float32)
        f32["q"], f32["k"] = rotate32(f32["q"], pos, cos, sin), rotate32(f32["k"], pos, cos, sin)
    q_out = qt.qtea_kv_append(c.cache, c.batch, x["k"].flatten(1), x["v"].flatten(1), q=x["q"].flatten(1),
                              cos=None if cos is None else gpu(cos), sin=None if sin is None else gpu(sin))
    assert np.array_equal(q_out.cpu().numpy().view(np.uint16), f32["q"].astype(np.float16).view(np.uint16))
    after, after_s = pools(c)
    for s in "kv":
        want, want_s = before[s].copy(), None if before_s[s] is None else before_s[s].copy()
        codes, scale = od.encode(f32[s], c.fmt)
        t = 0
        for i, (n, m) in enumerate(zip(q_len, ctx)):
            for j in range(n):
                p = m - n + j
                if p >= 0:
                    at = (c.pages[i][p // page], slice(None), p % page)
                    want[at] = codes[t]
                    if want_s is not None:
                        want_s[at] = scale[t]
                t += 1
        kind = np.uint16 if c.fmt == od.F16 else np.uint8
        assert np.array_equal(after[s].view(kind), want.view(kind)), s
        assert want_s is None or np.array_equal(after_s[s], want_s)


@pytest.mark.parametrize("dim", [64, 128])
def test_append_norms_and_strided_sources(qt, dim):
    q_len, ctx = [5, 2], [9, 2]
    c = Case(qt, "f16", q_len, ctx, 4, 2, dim, 16, seed=13)
    rng = np.random.default_rng(14)
    qkv = gpu(rng.standard_normal((c.tokens, 8 * dim + 3)).astype(np.float32))  # odd row stride
    q, k, v = qkv[:, :4 * dim], qkv[:, 4 * dim:6 * dim], qkv[:, 6 * dim:8 * dim]
    wq, wk = ((1 + 0.3 * rng.standard_normal(dim)).astype(np.float16) for _ in range(2))
    ang = rng.uniform(0, 6.28, (20, dim // 2))
    cos, sin = np.cos(ang).astype(np.float32), np.sin(ang).astype(np.float32)
    got = qt.qtea_kv_append(c.cache, c.batch, k, v, q=q, cos=gpu(cos), sin=gpu(sin), q_norm=gpu(wq), k_norm=gpu(wk),
                            eps=1e-5)
    pos = od.token_positions(q_len, ctx)
    heads = lambda t, n: t.cpu().numpy().reshape(c.tokens, n, dim)
    ref_q = od.prepare_heads(heads(q, 4), pos, wq, cos, sin, 1e-5)
    ref_k = od.prepare_heads(heads(k, 2), pos, wk, cos, sin, 1e-5)

    def near(x, ref):
        big = np.abs(ref).max()
        assert np.all(np.abs(x - ref) <= 2.0 ** -11 * np.abs(ref) + 8 * 2.0 ** -24 * big + 2.0 ** -25)

    near(got.cpu().numpy().astype(np.float64), ref_q)
    after, _ = pools(c)
    t = 0
    for i, (n, m) in enumerate(zip(q_len, ctx)):
        for j in range(n):
            p = m - n + j
            at = (c.pages[i][p // 16], slice(None), p % 16)
            near(after["k"][at].astype(np.float64), ref_k[t])
            assert np.array_equal(after["v"][at], heads(v, 2)[t].astype(np.float16))
            t += 1


def test_append_non_finite_and_overflowing_sources(qt):
    for fmt, top in (("f16", 65504.0), ("fp8", 448.0 * 128), ("fp4", 6.0 * 2 ** 13)):
        c = Case(qt, fmt, [1], [1], 1, 1, 64, 16, seed=15)
        x = torch.zeros(1, 64, device="cuda")
        x[0, 3], x[0, 4], x[0, 5] = float("inf"), -1e30, float("nan")
        x[0, 40] = 1.5
        qt.qtea_kv_append(c.cache, c.batch, x, x)
        k, _ = qt.qtea_kv_read(c.cache, c.batch, torch.tensor([0, 1], dtype=torch.int32, device="cuda"), n_rows=1)
        k = k[0, 0].float().cpu()
        assert k[3] == top and k[4] == -top and k[40] == 1.5
        assert torch.isnan(k[5]) if fmt != "fp4" else k[5].abs() == top


def test_append_outside_the_cache_writes_nothing(qt):
    c = Case(qt, "fp8", [1, 1, 1, 4], [20, 20, 200, 20], 2, 2, 64, 16, seed=16)
    table = c.batch.pages.clone()
    table[0, 1], table[1, 1] = c.cache.n_pages, -1
    ctx = torch.tensor([20, 20, 1000, -3], dtype=torch.int32, device="cuda")  # past its table: its last place
    table[2] = -1
    b = qt.KVBatch(c.batch.q_start, ctx, table, c.tokens, 4)
    before = [t.clone() for t in (c.t["k"], c.t["v"], c.ts["k"], c.ts["v"])]
    x = torch.randn(c.tokens, 128, device="cuda")
    qt.qtea_kv_append(c.cache, b, x, x)
    assert all(torch.equal(a, t) for a, t in zip(before, (c.t["k"], c.t["v"], c.ts["k"], c.ts["v"])))


@pytest.mark.parametrize("fmt", list(FMTS))
@pytest.mark.parametrize("dim,page,hkv,ctx", [(128, 16, 2, [37, 0, 1, 64]), (64, 128, 5, [300, 2]), (64, 32, 1, [1])])
def test_read_back_is_exact(qt, fmt, dim, page, hkv, ctx):
    c = Case(qt, fmt, [1] * len(ctx), ctx, hkv, hkv, dim, page, seed=17)
    room = [n + (3 if i == 0 else 0) for i, n in enumerate(ctx)]  # the first has room for more: zeros
    start = np.concatenate(([2], 2 + np.cumsum(room))).astype(np.int32)
    k, v = (torch.full((int(start[-1]) + 2, hkv, dim), 7.0, dtype=torch.float16, device="cuda") for _ in range(2))
    qt.qtea_kv_read(c.cache, c.batch, gpu(start), k_out=k, v_out=v)
    for side, t in (("k", k), ("v", v)):
        t = t.cpu().numpy()
        assert np.all(t[:2] == 7) and np.all(t[start[-1]:] == 7)
        for s, n in enumerate(ctx):
            assert np.array_equal(t[start[s]:start[s] + n].astype(np.float64), c.seq[side][s])
            assert np.all(t[start[s] + n:start[s + 1]] == 0)
    only = torch.zeros_like(k)
    qt.qtea_kv_read(c.cache, c.batch, gpu(start), v_out=only)
    assert torch.equal(only[2:start[-1]], v[2:start[-1]])


# ------------------------------------------------------------------------------------------- norms


@pytest.mark.parametrize("h_type", [torch.float32, torch.float16])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 4096), (3, 5120), (2, 33), (700, 64), (1300, 1096), (5, 8200), (2, 16392),
                                       (1, 40001), (153, 2047)])
@pytest.mark.parametrize("form", ["x", "h", "post", "gate", "all", "all16"])
def test_norm(qt, h_type, rows, cols, form):
    rng = np.random.default_rng(rows * 7 + cols)
    h = gpu((3 * rng.standard_normal((rows, cols))).astype(np.float32)).to(h_type)
    w = gpu((1 + 0.2 * rng.standard_normal(cols)).astype(np.float16))
    kw, ref = {}, {}
    if form != "x":
        y_type = torch.float16 if form == "all16" else torch.float32
        y = rng.standard_normal((rows, cols))
        y[:, cols // 2] *= 100
        kw["y"] = gpu(y.astype(np.float32)).to(y_type)
        kw["res_scale"] = 0.7
        if form in ("post", "all", "all16"):
            kw["post_weight"] = gpu((1 + 0.2 * rng.standard_normal(cols)).astype(np.float16))
        if form in ("gate", "all", "all16"):
            shape = (rows, cols) if form == "all" else (cols,)
            kw["gate"] = gpu(rng.uniform(-1, 1, shape).astype(np.float16))
    want_x = form != "h"
    ref = {k: v.double().cpu().numpy() if hasattr(v, "cpu") else v for k, v in kw.items()}
    h_ref, x_ref = od.norm(h.double().cpu().numpy(), w.double().cpu().numpy() if want_x else None, eps=1e-5, **ref)
    if form != "x":
        kw["h_out"] = torch.full_like(h, 9.0)
    keep = h.clone()
    x = qt.qtea_norm(h, w if want_x else None, eps=1e-5, want_x=want_x, **kw)
    rel = 2 * (cols / 64 + 16) * 2.0 ** -24
    terms = np.abs(keep.double().cpu().numpy()) + np.abs(h_ref - keep.double().cpu().numpy())
    e_h = rel * terms
    if want_x:
        scale = np.abs(x_ref) / np.maximum(np.abs(h_ref), 1e-30)
        lim = 2.0 ** -11 * np.abs(x_ref) + scale * e_h + 2 * rel * np.abs(x_ref) + 2.0 ** -24
        assert np.all(np.abs(x.double().cpu().numpy() - x_ref) <= lim)
    if form != "x":
        got = kw["h_out"].double().cpu().numpy()
        lim = e_h + (2.0 ** -11 * np.abs(h_ref) + 2.0 ** -25 if h_type == torch.float16 else 0)
        assert np.all(np.abs(got - h_ref) <= lim)
        assert torch.equal(h, keep)
        qt.qtea_norm(h, w if want_x else None, eps=1e-5, want_x=want_x, **{**kw, "h_out": None})
        assert torch.equal(h, kw["h_out"])  # in place: the same


def test_norm_strided_and_misaligned_rows_agree_with_dense_ones(qt):
    for cols in (512, 4096):
        base = torch.randn(5, cols + 24, device="cuda")
        w = torch.rand(cols + 8, device="cuda").half()
        h, y = base[:, 8:8 + cols], torch.randn(5, 2 * cols, device="cuda")[:, cols:]
        ref_h = torch.empty(5, cols, device="cuda")
        ref = qt.qtea_norm(h.contiguous(), w[:cols], y=y.contiguous(), h_out=ref_h)
        out = torch.zeros(5, cols + 16, device="cuda").half()
        h_out = torch.zeros(5, cols + 8, device="cuda")
        qt.qtea_norm(h, w[:cols], y=y, h_out=h_out[:, :cols], x=out[:, 8:8 + cols])
        assert torch.equal(out[:, 8:8 + cols], ref) and torch.equal(h_out[:, :cols], ref_h)
        assert not out[:, :8].any() and not out[:, 8 + cols:].any() and not h_out[:, cols:].any()
        odd = base[:, 3:3 + cols]  # 4-byte aligned only
        got = qt.qtea_norm(odd, w[1:1 + cols].clone())
        want = od.norm(odd.double().cpu().numpy(), w[1:1 + cols].double().cpu().numpy())[1]
        lim = (2.0 ** -11 + 4 * (cols / 64 + 16) * 2.0 ** -24) * np.abs(want) + 2.0 ** -24
        assert np.all(np.abs(got.double().cpu().numpy() - want) <= lim)


# ---------------------------------------------------------------------------------------- refusals


def test_refusals(qt):
    c = Case(qt, "fp8", [1, 1], [20, 5], 4, 2, 64, 16, seed=20)
    q = torch.randn(2, 4, 64, device="cuda").half()
    out = torch.full_like(q, 7.0)
    lib, ws = qt.load(), qt.attention_workspace()
    bad = qt.QTEA_ERR_INVALID_ARG

    def att(kv=c.cache.handle, batch=c.batch._ref, qp=q.data_ptr(), q_ld=256, heads=4, window=0, o=out.data_ptr(),
            o_ld=256, lse=None, w=ws.data_ptr(), n=ws.numel()):
        return lib.qtea_attention(kv, batch, qp, q_ld, heads, 1.0, window, o, o_ld, lse, w, n, None)

    assert att(kv=None) == bad and att(batch=None) == bad and att(qp=None) == bad and att(o=None) == bad
    assert att(heads=3) == bad and att(heads=0) == bad and att(window=-1) == bad
    assert att(q_ld=254) == bad and att(q_ld=257) == bad and att(o_ld=255) == bad and att(qp=q.data_ptr() + 2) == bad
    assert att(w=None) == bad and att(n=ws.numel() - 1) == bad and att(w=ws.data_ptr() + 16) == bad
    assert att(lse=2) == bad
    assert att(heads=66 * 2, q_ld=66 * 2 * 64, o_ld=66 * 2 * 64) == qt.QTEA_ERR_UNSUPPORTED
    torch.cuda.synchronize()
    assert (out == 7.0).all()

    P, ok = c.cache.k_pages.data_ptr(), c.cache
    for args in [(P, P, None, P, 2, 16, 1, 64, 1), (P + 8, P, P, P, 2, 16, 1, 64, 1), (P, P, P, P + 4, 2, 16, 1, 64, 1),
                 (P, P, P, P, 0, 16, 1, 64, 1), (P, P, P, P, 2, 16, 0, 64, 1), (P, P, P, P, 2, 16, 1, 64, 3),
                 (P, P, P, P, 1 << 27, 16, 1, 64, 1), (P, P, P, P, 2, 16, 1025, 64, 1)]:
        with pytest.raises(qt.QteaError):
            import ctypes
            h = ctypes.c_void_p()
            rc = lib.qtea_kv_create(*args, ctypes.byref(h))
            assert rc == bad and not h.value
            raise qt.QteaError(rc, "qtea_kv_create")

    f = lambda *s, t=torch.float32: torch.zeros(*s, device="cuda", dtype=t)
    for call, kind in [
            (lambda: qt.KVCache(f(2, 1, 24, 64, t=torch.float16), f(2, 1, 24, 64, t=torch.float16)), qt.QteaError),
            (lambda: qt.KVCache(f(2, 1, 16, 80, t=torch.float16), f(2, 1, 16, 80, t=torch.float16)), qt.QteaError),
            (lambda: qt.KVCache(f(2, 1, 16, 64), f(2, 1, 16, 64)), TypeError),
            (lambda: qt.KVCache(c.t["k"], c.t["v"], fmt=qt.QTEA_KV_FP8), ValueError),
            (lambda: qt.KVCache(c.t["k"], c.t["v"], c.ts["k"], c.ts["v"][:1], fmt=qt.QTEA_KV_FP8), ValueError),
            (lambda: qt.KVBatch(c.batch.q_start[:2], c.batch.ctx_len, c.batch.pages, 2, 1), ValueError),
            (lambda: qt.KVBatch(c.batch.q_start.long(), c.batch.ctx_len, c.batch.pages, 2, 1), TypeError),
            (lambda: qt.KVBatch(c.batch.q_start.cpu(), c.batch.ctx_len, c.batch.pages, 2, 1), TypeError),
            (lambda: qt.qtea_attention(ok, c.batch, q.float()), TypeError),
            (lambda: qt.qtea_attention(ok, c.batch, q[:1]), ValueError),
            (lambda: qt.qtea_attention(ok, c.batch, q.transpose(1, 2).contiguous().transpose(1, 2)), ValueError),
            (lambda: qt.qtea_attention(ok, c.batch, q, out=out[:, :, :32]), ValueError),
            (lambda: qt.qtea_attention(ok, c.batch, q, lse=f(2, 3)), ValueError),
            (lambda: qt.qtea_attention(ok, qt.KVBatch(c.batch.q_start, c.batch.ctx_len, c.batch.pages, 2, 0), q),
             qt.QteaError),
            (lambda: qt.qtea_kv_append(ok, c.batch, f(2, 128), f(2, 128, t=torch.float16)), TypeError),
            (lambda: qt.qtea_kv_append(ok, c.batch, f(2, 64), f(2, 64)), ValueError),
            (lambda: qt.qtea_kv_append(ok, c.batch, f(2, 128), f(2, 128), q=f(2, 100)), ValueError),
            (lambda: qt.qtea_kv_append(ok, c.batch, f(2, 128), f(2, 128), cos=f(4, 32)), ValueError),
            (lambda: qt.qtea_kv_append(ok, c.batch, f(2, 128), f(2, 128), cos=f(4, 32), sin=f(5, 32)), ValueError),
            (lambda: qt.qtea_kv_append(ok, c.batch, f(2, 128), f(2, 128), cos=f(0, 32), sin=f(0, 32)), qt.QteaError),
            (lambda: qt.qtea_kv_read(ok, c.batch, c.batch.q_start), ValueError),
            (lambda: qt.qtea_kv_read(ok, c.batch, c.batch.q_start[:2], n_rows=4), ValueError),
            (lambda: qt.qtea_norm(f(2, 64), f(64, t=torch.float16), gate=f(64, t=torch.float16)), ValueError),
            (lambda: qt.qtea_norm(f(2, 64), f(64)), TypeError),
            (lambda: qt.qtea_norm(f(2, 64), None), ValueError),
            (lambda: qt.qtea_norm(f(2, 64), f(64, t=torch.float16), y=f(2, 65)), ValueError),
            (lambda: qt.qtea_norm(f(2, 64), f(64, t=torch.float16), y=f(2, 64), h_out=f(2, 64, t=torch.float16)),
             TypeError)]:
        with pytest.raises(kind):
            call()


def test_empty_calls_do_nothing(qt):
    c = Case(qt, "f16", [0, 0], [20, 0], 4, 2, 64, 16, seed=21)
    assert qt.qtea_attention(c.cache, c.batch, torch.zeros(0, 4, 64, device="cuda").half()).shape == (0, 4, 64)
    z = torch.zeros(0, 128, device="cuda")
    before = c.t["k"].clone().view(torch.int16)
    qt.qtea_kv_append(c.cache, c.batch, z, z)
    assert torch.equal(before, c.t["k"].view(torch.int16))
    k, v = qt.qtea_kv_read(c.cache, c.batch, torch.zeros(3, dtype=torch.int32, device="cuda"), n_rows=0)
    assert k.shape == v.shape == (0, 2, 64)
    assert qt.qtea_norm(torch.zeros(0, 64, device="cuda"), torch.ones(64, device="cuda").half()).shape == (0, 64)
