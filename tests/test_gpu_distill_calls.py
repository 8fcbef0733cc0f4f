"""Scoring with top alternatives and distillation: how they are called.  Graphs, streams, workspaces, places of outputs, batches with little or nothing in them, numbers that
are none, sizes at the ends of what is allowed, and the two of them together."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import distill_oracle as orc
from paper_2603_16435_amd import binding
from test_gpu_distill import Batch, DTYPES, U, check_distill, check_score, host, near, off_grid

pytestmark = pytest.mark.gpu
FIELDS = ("loss", "row_loss", "lse", "d_hidden", "d_weight", "stats")


def same(a, b, fields):
    for f in fields:
        x, y = getattr(a, f), getattr(b, f)
        assert torch.equal(x.view(torch.uint8) if x.dtype != torch.uint8 else x, y.view(torch.uint8)), f


def need(b, K, distill, chunk=0, bwd=True, dw=0):
    batch = binding.make_batch(b.hidden, b.weight, b.ids, b.mask, b.cu)
    n = C.c_size_t(0)
    if distill:
        binding._check(binding.lib().rl_distill_workspace_bytes(C.byref(batch), C.byref(binding.rl_distill_params(K, 0, 0, chunk, 1.0, 1.0, dw)), int(bwd), C.byref(n)))
    else:
        binding._check(binding.lib().rl_token_top_logprobs_workspace_bytes(C.byref(batch), C.byref(binding.rl_top_params(K, chunk, 1.0)), C.byref(n)))
    return n.value


SHAPES = [(50, 128, 3000, "bf16", 0), (300, 136, 2000, "bf16", 256), (20, 68, 1000, "f32", 0), (600, 100, 700, "f32", 256)]


@pytest.mark.parametrize("R,H,V,dtype,chunk", SHAPES)
def test_the_workspace_is_as_large_as_asked_and_its_contents_do_not_count(R, H, V, dtype, chunk):
    b = Batch(R, H, V, dtype, seed=1)
    ids, lp = b.teacher(9)
    for distill in (False, True):
        n = need(b, 9, distill, chunk)
        run = (lambda ws: b.distill(ids, lp, chunk_rows=chunk, workspace=ws)) if distill else (lambda ws: b.score(9, chunk_rows=chunk, workspace=ws))
        buf = torch.zeros(n + 8192, dtype=torch.uint8, device="cuda")
        at = -buf.data_ptr() % 256 + 2048
        res = []
        for fill in (0, 0xFF, 0x7F):
            buf.fill_(fill)
            res.append(run(buf[at:at + n]))
            assert bool((buf[:at] == fill).all()) and bool((buf[at + n:] == fill).all())
        for r in res[1:]:
            same(res[0], r, FIELDS if distill else ("logprob", "lse", "entropy", "top_ids", "top_logprob"))
        with pytest.raises(binding.RlError) as e:
            run(buf[at:at + n - 256])
        assert e.value.status == 5


@pytest.mark.parametrize("R,H,V,dtype,chunk", SHAPES)
def test_captured_and_replayed(R, H, V, dtype, chunk):
    """A graph of both calls, replayed on new inputs with eager work and synchronisations between, gives what the eager calls give."""
    b, others = Batch(R, H, V, dtype, seed=2), [Batch(R, H, V, dtype, seed=20 + i) for i in range(3)]
    ids, lp = b.teacher(9)
    lists = [o.teacher(9) for o in others]
    score = lambda x: x.score(9, chunk_rows=chunk)
    learn = lambda x, i, l: x.distill(i, l, chunk_rows=chunk, d_weight_dtype=DTYPES[dtype])
    want = [(score(o), learn(o, *l)) for o, l in zip(others, lists)]
    score(b), learn(b, ids, lp)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        got = (score(b), learn(b, ids, lp))
    for _ in range(2):
        for o, l, w in zip(others, lists, want):
            for dst, src in ((b.hidden, o.hidden), (b.weight, o.weight), (b.ids, o.ids), (b.mask, o.mask), (b.cu, o.cu), (ids, l[0]), (lp, l[1])):
                dst.copy_(src)
            graph.replay()
            torch.cuda.synchronize()
            same(got[0], w[0], ("logprob", "lse", "entropy", "top_ids", "top_logprob"))
            same(got[1], w[1], FIELDS)
            same(learn(o, *l), w[1], FIELDS)


def test_two_streams_at_once():
    a, b = Batch(200, 256, 9000, "bf16", seed=3), Batch(60, 512, 4000, "bf16", seed=4)
    ta, tb = a.teacher(20), b.teacher(20)
    want = [a.distill(*ta), b.distill(*tb), a.score(20), b.score(20)]
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    got = []
    for _ in range(5):
        with torch.cuda.stream(s1):
            x = a.distill(*ta), a.score(20)
        with torch.cuda.stream(s2):
            y = b.distill(*tb), b.score(20)
        got.append((x[0], y[0], x[1], y[1]))
    torch.cuda.synchronize()
    for g in got:
        for w, r in zip(want[:2], g[:2]):
            same(w, r, FIELDS)
        for w, r in zip(want[2:], g[2:]):
            same(w, r, ("logprob", "lse", "entropy", "top_ids", "top_logprob"))


@pytest.mark.parametrize("dtype,H,V", [("bf16", 128, 5000), ("bf16", 264, 33000), ("f32", 68, 3000)])
def test_a_row_does_not_depend_on_the_batch(dtype, H, V):
    """Chunk sizes, and (bf16) the number of rows scored together, change no bit; neither does running again."""
    b = Batch(300, H, V, dtype, seed=5, masked=0.0, B=1)
    want = b.score(17)
    fields = ("logprob", "lse", "entropy", "top_ids", "top_logprob")
    same(want, b.score(17), fields)
    same(want, b.score(17, chunk_rows=256), fields)
    same(want, b.score(17, chunk_rows=100000), fields)
    for n in ((1, 64, 65, 128, 129) if dtype == "bf16" else (65, 100, 256)):
        part = binding.rl_token_top_logprobs(b.hidden[:n].contiguous(), b.weight, b.ids[:n].contiguous(), b.mask[:n].contiguous(), 17)
        for f in fields:
            assert torch.equal(getattr(part, f), getattr(want, f)[:n]), (n, f)
    ids, lp = b.teacher(17)
    same(b.distill(ids, lp), b.distill(ids, lp), FIELDS)
    one, two = b.distill(ids, lp), b.distill(ids, lp, chunk_rows=256)
    same(one, two, ("row_loss", "lse", "stats"))                 # (dX is cut along the vocabulary by the rows of a chunk: another order of its sums)


@pytest.mark.parametrize("R,H,V,dtype,chunk", SHAPES)
def test_hidden_makes_room_for_its_gradient(R, H, V, dtype, chunk):
    b = Batch(R, H, V, dtype, seed=6)
    ids, lp = b.teacher(12)
    want = b.distill(ids, lp, chunk_rows=chunk)
    x = b.hidden.clone()
    got = binding.rl_distill_loss_fwd_bwd(x, b.weight, ids, lp, b.mask, b.cu, chunk_rows=chunk, d_hidden=x)
    assert got.d_hidden.data_ptr() == x.data_ptr()
    same(want, got, FIELDS)


@pytest.mark.parametrize("R,H,V,dtype,chunk", SHAPES)
@pytest.mark.parametrize("off", [1, 3])
def test_outputs_start_anywhere_and_end_where_they_end(R, H, V, dtype, chunk, off):
    """Through the C ABI: gradients at any element of a buffer, guards around every output, outputs that are not wanted."""
    b = Batch(R, H, V, dtype, seed=7)
    K = 9
    ids, lp = b.teacher(K)
    L, batch = binding.lib(), binding.make_batch(b.hidden, b.weight, b.ids, b.mask, b.cu)
    dw = 1 if dtype == "bf16" else 0
    want, top = b.distill(ids, lp, chunk_rows=chunk, d_weight_dtype=DTYPES[dtype]), b.score(K, chunk_rows=chunk)
    guarded = {}

    def place(name, t, shift):
        g = torch.full((t.numel() + 64,), 7, dtype=t.dtype, device="cuda")
        guarded[name] = (g, shift, t)
        return g[shift:].data_ptr()

    ws = torch.empty(need(b, K, True, chunk, dw=dw) + 256, dtype=torch.uint8, device="cuda")
    ws = ws[-ws.data_ptr() % 256:]
    out = binding.rl_distill_outputs(*[place(f, getattr(want, f), off if f.startswith("d_") else 16) for f in ("loss", "row_loss", "lse", "d_hidden", "d_weight", "stats")])
    prm = binding.rl_distill_params(K, 0, 0, chunk, 1.0, 1.0, dw)
    binding._check(L.rl_distill_loss_fwd_bwd(C.byref(batch), ids.data_ptr(), lp.data_ptr(), C.byref(prm), C.byref(out), ws.data_ptr(), ws.numel(), None))
    tops = ("logprob", "lse", "entropy", "top_ids", "top_logprob")
    tout = binding.rl_top_outputs(*[place("t_" + f, getattr(top, f), 16 + off) for f in tops])
    binding._check(L.rl_token_top_logprobs(C.byref(batch), C.byref(binding.rl_top_params(K, chunk, 0.0)), C.byref(tout), ws.data_ptr(), ws.numel(), None))
    torch.cuda.synchronize()
    for name, (g, shift, t) in guarded.items():
        n = t.numel()
        assert torch.equal(g[shift:shift + n].view(torch.uint8), t.flatten().view(torch.uint8)), name
        assert bool((g[:shift] == 7).all()) and bool((g[shift + n:] == 7).all()), name
    # one output at a time
    for f in tops:
        t = torch.empty_like(getattr(top, f))
        one = binding.rl_top_outputs(**{f: t.data_ptr()})
        binding._check(L.rl_token_top_logprobs(C.byref(batch), C.byref(binding.rl_top_params(K, chunk, 1.0)), C.byref(one), ws.data_ptr(), ws.numel(), None))
        assert torch.equal(t, getattr(top, f)), f
    loss = torch.empty(1, device="cuda")
    binding._check(L.rl_distill_loss_fwd_bwd(C.byref(batch), ids.data_ptr(), lp.data_ptr(), C.byref(prm), C.byref(binding.rl_distill_outputs(loss=loss.data_ptr())),
                                             ws.data_ptr(), ws.numel(), None))
    assert torch.equal(loss, want.loss)
    alone = b.distill(ids, lp, chunk_rows=chunk, backward=False)
    same(alone, want, ("loss", "row_loss", "lse", "stats"))
    assert alone.d_hidden is None and alone.d_weight is None


@pytest.mark.parametrize("R,H,V,dtype,chunk", SHAPES)
def test_nothing_counts(R, H, V, dtype, chunk):
    b = Batch(R, H, V, dtype, seed=8)
    ids, lp = b.teacher(5)
    b.mask.zero_()
    b.hidden.fill_(float("nan"))
    r, t = b.distill(ids, lp, chunk_rows=chunk, d_weight_dtype=DTYPES[dtype]), b.score(5, chunk_rows=chunk)
    for x in (r.loss, r.row_loss, r.lse, r.d_hidden, r.d_weight, r.stats, t.logprob, t.lse, t.entropy, t.top_logprob):
        assert not x.any()
    assert bool((t.top_ids == -1).all())


@pytest.mark.parametrize("dtype,H,V", [("bf16", 128, 3000), ("f32", 68, 1000)])
@pytest.mark.parametrize("R", [40, 200])
def test_sequences_lists_and_masks_of_every_kind(dtype, H, V, R):
    """Offsets that alternate, dip and leave rows out, many sequences without a row, any non-zero mask, lists of which nothing is left."""
    for cu in ([0, 5, 5, 3, 20, R], [0, 1, 2, 2, R // 2], [3, 10, R - 1], [0, R, 0, R], [0] * 500 + [R] + [R] * 600, [0, R + 1, R]):
        b = Batch(R, H, V, dtype, seed=9, cu=cu)
        ids, lp = b.teacher(6)
        b.mask *= 255
        ids[R // 2:R // 2 + 5] = -1
        lp[3] = -float("inf")
        for rest in ("bucket", "renormalise"):
            check_distill(b, b.distill(ids, lp, rest=rest, d_weight_dtype=DTYPES[dtype]), ids, lp, rest, 1.0, "sequence")
        check_score(b, b.score(6), 6, 1.0)


@pytest.mark.parametrize("dtype,H,V,R", [("bf16", 128, 3000, 40), ("bf16", 128, 3000, 200), ("f32", 68, 1000, 20), ("f32", 68, 1000, 200)])
def test_what_is_no_number_stays_in_its_row(dtype, H, V, R):
    b = Batch(R, H, V, dtype, seed=10, masked=0.3)
    ids, lp = b.teacher(6)
    b.mask[7], b.mask[8], b.mask[9] = 1, 0, 1
    ids[7, 0] = ids[9, 0] = 1
    lp[9, 0] = float("nan")
    want, top = b.distill(ids, lp, rest="renormalise"), b.score(6)
    b.hidden[7], b.hidden[8] = float("nan"), float("inf")
    got, t = b.distill(ids, lp, rest="renormalise"), b.score(6)
    others = torch.arange(R, device="cuda") != 7
    for f in ("logprob", "lse", "entropy", "top_ids", "top_logprob"):
        assert torch.equal(getattr(t, f)[others], getattr(top, f)[others]), f
    assert t.lse[7].isnan() and t.entropy[7].isnan() and bool((t.top_ids[7] == -1).all()) and bool(t.top_logprob[7].isnan().all())
    clean = others & (torch.arange(R, device="cuda") != 9)
    assert torch.equal(got.row_loss[clean], want.row_loss[clean]) and torch.equal(got.d_hidden[clean], want.d_hidden[clean])
    assert got.row_loss[7].isnan() and got.row_loss[9].isnan() and want.row_loss[9].isnan() and got.loss.isnan()
    assert not got.row_loss[8].any() and not got.d_hidden[8].any()
    # a row without a list has no part in it, whatever its logits
    ids[7], ids[9] = -1, -1
    r = b.distill(ids, lp)
    assert r.row_loss[7] == 0 and not r.d_hidden[7].any() and bool(r.loss.isfinite())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tau", [0.01, 100.0])
@pytest.mark.parametrize("R", [20, 100])
def test_sharp_and_flat(dtype, tau, R):
    """Rows whose largest logit has all of the probability (what the others have is far below f32's smallest number), and rows that are nearly uniform: the bucket's logarithm and
    gradient are those of the definition.  Logits are whole multiples of 2^-8 or so, and the differences that are scaled reach 1000: an exponential is off by 2 u d of itself, d <= 2000."""
    b = Batch(R, 64, 2000, dtype, seed=11)
    ids, lp = b.teacher(4, wild=False)
    lp = torch.where(ids >= 0, torch.log(torch.tensor([0.4, 0.3, 0.1, 0.05], device="cuda")).expand(R, 4), lp).contiguous()
    r = b.distill(ids, lp, temperature=tau, d_weight_dtype=DTYPES[dtype])
    want = orc.distill(host(b.hidden), host(b.weight), host(ids), host(lp), host(b.mask), host(b.cu), "bucket", tau)
    big = max(1.0, np.abs(want["row_loss"]).max())
    assert bool(r.row_loss.isfinite().all()) and (tau > 1 or big > 200)
    near(r.row_loss, want["row_loss"], 64 * U * (1 + big), "row_loss")
    near(r.lse, want["lse"], 64 * U * (1 + np.abs(want["lse"])), "lse")
    x, w, ds = np.abs(host(b.hidden).astype(np.float64)), np.abs(host(b.weight).astype(np.float64)), np.abs(want["dS"])
    err = 4096 * U * want["gross"] + (2.0 ** -8 if dtype == "bf16" else U) * ds + 1e-37
    half = 2.0 ** -8 if dtype == "bf16" else U
    near(r.d_hidden, want["d_hidden"], err @ w + 2100 * U * (ds @ w) + half * (np.abs(want["d_hidden"]) + err @ w), "d_hidden")
    near(r.d_weight, want["d_weight"], err.T @ x + (R + 64) * U * (ds.T @ x) + half * (np.abs(want["d_weight"]) + err.T @ x), "d_weight")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_largest_vocabulary(dtype):
    b = Batch(9, 8, 524288, dtype, seed=12, masked=0.0)
    check_score(b, b.score(128), 128, 1.0)
    ids, lp = b.teacher(128)
    check_distill(b, b.distill(ids, lp, d_weight_dtype=DTYPES[dtype]), ids, lp, "bucket", 1.0, "sequence")


def test_a_list_that_names_every_token():
    b = Batch(30, 64, 100, "bf16", seed=13)
    ids, lp = b.teacher(128, wild=False)
    for rest in ("bucket", "renormalise"):
        check_distill(b, b.distill(ids, lp, rest=rest, d_weight_dtype=torch.bfloat16), ids, lp, rest, 1.0, "sequence")


def test_offsets_past_32_bits():
    """Logits of one chunk past 2^32 elements, outputs past 2^31: the rows that count are those of small calls."""
    R, H, V, K = 32768, 64, 140000, 3
    g = torch.Generator(device="cuda").manual_seed(1)
    w = (torch.randn(V, H, generator=g, device="cuda") * 0.15).bfloat16()
    x = torch.randn(R, H, generator=g, device="cuda").bfloat16()
    mask, ids = torch.ones(R, dtype=torch.uint8, device="cuda"), torch.zeros(R, dtype=torch.int32, device="cuda")
    big = binding.rl_token_top_logprobs(x, w, ids, mask, K, chunk_rows=R)
    for at in (0, 30683, R - 200):
        part = binding.rl_token_top_logprobs(x[at:at + 200].contiguous(), w, ids[at:at + 200].contiguous(), mask[at:at + 200].contiguous(), K)
        for f in ("logprob", "lse", "entropy", "top_ids", "top_logprob"):
            assert torch.equal(getattr(part, f), getattr(big, f)[at:at + 200]), f
    del big
    R, H, V, K = 17_000_000, 8, 300, 128
    x, w = torch.zeros(R, H, dtype=torch.bfloat16, device="cuda"), torch.randn(V, H, generator=g, device="cuda").bfloat16()
    mask = torch.zeros(R, dtype=torch.uint8, device="cuda")
    on = torch.tensor([0, 16_777_216, R - 1], device="cuda")
    mask[on], x[on] = 1, torch.randn(3, H, generator=g, device="cuda").bfloat16()
    big = binding.rl_token_top_logprobs(x, w, None, mask, K)
    part = binding.rl_token_top_logprobs(x[on].contiguous(), w, None, mask[on].contiguous(), K)
    assert torch.equal(big.top_ids[on], part.top_ids) and torch.equal(big.top_logprob[on], part.top_logprob)
    assert bool((big.top_ids[16_777_000:16_777_216] == -1).all()) and not big.top_logprob[16_777_217:R - 1].any()
    d = binding.rl_distill_loss_fwd_bwd(x, w, big.top_ids, big.top_logprob, mask, temperature=2.0)
    e = binding.rl_distill_loss_fwd_bwd(x[on].contiguous(), w, part.top_ids, part.top_logprob, mask[on].contiguous(), temperature=2.0)
    assert torch.equal(d.row_loss[on], e.row_loss) and torch.equal(d.d_hidden[on], e.d_hidden) and d.stats_dict() == e.stats_dict()


def test_gradient_by_differences():
    """f32: the loss of the kernel itself, in steps of the hidden states and the weight."""
    b = Batch(10, 16, 150, "f32", seed=14, masked=0.2)
    ids, lp = b.teacher(8)
    for rest, tau in (("bucket", 1.0), ("renormalise", 1.5)):
        r = b.distill(ids, lp, rest=rest, temperature=tau, aggregation="token")
        f = lambda x, w: orc.distill(x, w, host(ids), host(lp), host(b.mask), host(b.cu), rest, tau, "token")["loss"]
        x, w = host(b.hidden).astype(np.float64), host(b.weight).astype(np.float64)
        h, g = 1e-5, np.random.default_rng(3)
        for _ in range(6):                                       # along random directions, of the oracle's loss in 64 bits: h^2 and 1e-16 / h are far below
            dx, dw = g.normal(size=x.shape), g.normal(size=w.shape)
            slope = (f(x + h * dx, w + h * dw) - f(x - h * dx, w - h * dw)) / (2 * h)
            got = (host(r.d_hidden) * dx).sum() + (host(r.d_weight) * dw).sum()
            size = (np.abs(host(r.d_hidden)) * np.abs(dx)).sum() + (np.abs(host(r.d_weight)) * np.abs(dw)).sum()
            assert abs(slope - got) <= 2.0 ** -12 * size
        loss = binding.rl_distill_loss_fwd_bwd(b.hidden, b.weight, ids, lp, b.mask, b.cu, rest=rest, temperature=tau, aggregation="token", backward=False).loss
        assert torch.equal(loss, r.loss)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_teacher_and_a_student(dtype):
    """The two calls as they are used: a teacher's lists, a student that learns from them; one that has the teacher's weights has nothing to learn, and its gradient is rounding."""
    t = Batch(90, 128, 4000, dtype, seed=15)
    s = Batch(90, 128, 4000, dtype, seed=16)
    s.mask, s.cu = t.mask, t.cu
    top = t.score(32, 1.3)
    r = s.distill(top.top_ids, top.top_logprob, temperature=1.3, d_weight_dtype=DTYPES[dtype])
    check_distill(s, r, top.top_ids, top.top_logprob, "bucket", 1.3, "sequence")
    again = t.distill(top.top_ids, top.top_logprob, temperature=1.3)
    assert again.row_loss.abs().max() < 2.0 ** -17 and again.loss.abs() < 2.0 ** -17 and r.loss > 0.1
    assert again.d_hidden.float().norm() < 2.0 ** -14 * r.d_hidden.float().norm()
    scaled = s.distill(top.top_ids, top.top_logprob, temperature=1.3, scale=-2.0, d_weight_dtype=DTYPES[dtype])
    assert torch.equal(scaled.loss, -2 * r.loss)
    # (the matrix unit's sums are not mirrored to the bit by a sign: its inner additions cut off, they do not round)
    check_distill(s, scaled, top.top_ids, top.top_logprob, "bucket", 1.3, "sequence", -2.0)
    twice = s.distill(top.top_ids, top.top_logprob, temperature=1.3, scale=2.0, d_weight_dtype=DTYPES[dtype])
    assert torch.equal(twice.loss, 2 * r.loss) and torch.equal(twice.d_hidden, 2 * r.d_hidden) and torch.equal(twice.d_weight, 2 * r.d_weight)


def test_binding_refusals():
    b = Batch(8, 64, 300, "bf16", seed=17)
    ids, lp = b.teacher(4)
    for bad in (lambda: b.score(301), lambda: b.score(0), lambda: b.score(129), lambda: b.score(4, tau=-1.0), lambda: b.distill(ids, lp, rest=5), lambda: b.distill(ids, lp, chunk_rows=-1),
                lambda: binding.rl_token_top_logprobs(b.hidden, b.weight, b.ids, b.mask, 3, workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(binding.RlError):
            bad()
    for bad in (lambda: b.distill(ids.long(), lp), lambda: b.distill(ids, lp.double()), lambda: b.distill(ids[:, :2], lp[:, :2]), lambda: b.distill(ids, lp[:4]), lambda: b.distill(ids, lp, scale=0.0),
                lambda: b.distill(ids, lp, d_weight_dtype=torch.float16), lambda: b.distill(ids, lp, d_hidden=torch.empty(8, 64, device="cuda")), lambda: b.score(3, ids=b.ids.cpu()),
                lambda: binding.rl_token_top_logprobs(b.hidden.t(), b.weight, None, b.mask, 3), lambda: b.score(3, workspace=torch.empty(10, device="cuda"))):
        with pytest.raises(ValueError):
            bad()
