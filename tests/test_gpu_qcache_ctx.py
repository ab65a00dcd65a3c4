"""Contexts with 8-bit K/V through the C ABI, against the 64-bit decoder over the 8-bit cache's reference.

Tolerances.  What the device computes differs from the reference by the path's own rounding (1e-4 for fp32
models, 3e-2 for bf16 ones, as in the other context tests) and by the codes that rounding sends to
the neighbour.  With a relative error r of the keys and values, about r / 2^-4 of the codes flip, each by a
whole step where rounding costs step / sqrt(12), so the flips move the logits by sqrt(12 * 16 r) of what the
rounding to 8 bits does (delta, the reference's own difference from fp64 K/V): r of 2^-20 and
2^-11 gives 1/74 and 0.31; the tests allow 1/20 and 1.
"""
import numpy as np
import pytest

from paper_2508_10259_amd import workload as W
import oracle.decoder as D
from gpu_util import ForcedRef, Pair, gpu_new_tokens, log, small_spec
from qcache_ref import QuantRow

pytestmark = pytest.mark.gpu

PATH = {"f32": 1e-4, "bf16": 3e-2}
FLIPS = {"f32": 1 / 20, "bf16": 1.0}


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def _prefixes(spec, seed, lens):
    return [W.Prefix(W.make_observation(spec, seed, 0, b, n - min(4, n - 1)),
                     np.arange(min(4, n - 1), dtype=np.int32) * 5 % 40) for b, n in enumerate(lens)]


def _forced(seed, B, A):
    import torch
    f = np.random.default_rng(seed).integers(0, 256, (B, A)).astype(np.int32)
    return f, torch.from_numpy(f).cuda()


class Row:
    """A row's references over 8-bit and over fp64 K/V, and the check of a step's logits."""

    def __init__(self, pair, prefix, cap, select=0):
        self.pair, self.cap, self.q = pair, cap, QuantRow(pair.p, cap, select)
        self.q.commit(prefix)
        self.plain = ForcedRef(pair.p, prefix)

    def step(self, new, fed, got, dtype):
        new = None if new is None else self.pair.obs_f64(new)
        z, z0 = self.q.step(new, fed), self.plain.step(new, fed)
        delta, err = np.abs(z - z0).max(), np.abs(got - z)
        tol = PATH[dtype] + FLIPS[dtype] * delta
        log(f"   max error {err.max():.2e} (tolerance {tol:.2e}, 8-bit K/V move the logits by {delta:.2e})")
        assert err.max() <= tol
        return err, np.abs(z - z0)


@pytest.mark.parametrize("dtype,B,d,H,F,paged", [
    ("f32", 3, 256, 4, 512, False), ("f32", 2, 256, 2, 512, True), ("bf16", 1, 256, 4, 512, False),
    ("bf16", 5, 512, 4, 1024, True), ("bf16", 12, 512, 8, 1536, False), ("bf16", 70, 256, 4, 512, False)])
def test_steps_over_8_bit_contexts(dtype, B, d, H, F, paged):
    import torch
    from paper_2508_10259_amd.runtime import DeviceContext
    spec = small_spec(dtype, 2, d, H, F)
    pair = Pair(spec, seed=61)
    lens = [int(x) for x in np.random.default_rng(B + d).integers(40, 190, size=B)]
    lens[0], lens[-1] = 1, 64
    pre = _prefixes(spec, 61, lens)
    packed, plens = pair.dev.pack_prefixes(pre)
    cap, A = 256, 5
    ctx = DeviceContext(pair.dev, B, cap, n_pages=B * cap // 64 if paged else None, qcache=True)
    assert not ctx.persistent_decode
    ctx.build(packed, plens)
    rows = sorted({0, B // 2, B - 1})
    f64 = pair.prefixes_f64(pre)
    refs = {b: Row(pair, f64[b], cap) for b in rows}
    for s in range(3):
        news = [W.make_observation(spec, 61, 20 + s, b, (b + s) % 4) if (b + s) % 4 else None for b in range(B)]
        fed, forced = _forced(s, B, A)
        nt, nl = gpu_new_tokens(spec, news)
        _, z = ctx.step(A, nt, nl if nt is not None else None, forced=forced)
        torch.cuda.synchronize()
        z = z.cpu().numpy()
        for b in rows:
            refs[b].step(news[b], fed[b], z[b], dtype)
        if s == 0:  # new tokens without a step, and one row rebuilt alone
            more = [W.make_observation(spec, 61, 40, b, 1 + b % 3) for b in range(B)]
            nt, nl = gpu_new_tokens(spec, more)
            ctx.append(nt, nl)
            for b in rows:
                x = pair.obs_f64(more[b])
                refs[b].q.commit(x)
                refs[b].plain.step(x, [0])
            p1 = _prefixes(spec, 62, [77])
            ctx.invalidate_rows([B // 2])
            pk, pl = pair.dev.pack_prefixes(p1)
            ctx.build_rows([B // 2], pk, pl)
            refs[B // 2] = Row(pair, pair.prefixes_f64(p1)[0], cap)
    ctx.close()


def test_selected_pages_of_a_decode():
    """fp32, three pages of up to six: the reference's choices have a gap that rounding does not close."""
    import torch
    from paper_2508_10259_amd.runtime import DeviceContext
    spec = small_spec("f32", 2, 256, 4, 512)
    pair = Pair(spec, seed=65)
    B, cap, A = 2, 384, 4
    pre = _prefixes(spec, 63, [330, 200])
    packed, plens = pair.dev.pack_prefixes(pre)
    ctx = DeviceContext(pair.dev, B, cap, qcache=True)
    ctx.build(packed, plens)
    f64 = pair.prefixes_f64(pre)
    fed, forced = _forced(5, B, A)
    for n in (3, 0, 2, 6, 100):
        ctx.select_pages(n)
        _, z = ctx.step(A, forced=forced)
        torch.cuda.synchronize()
        z = z.cpu().numpy()
        for b in range(B):
            r = Row(pair, f64[b], cap, n if n < 6 else 0)
            r.step(None, fed[b], z[b], "f32")
            log(f"n={n} row {b}: relative gap {r.q.margin:.1e}")
    ctx.close()


def test_selected_pages_that_no_rounding_exchanges():
    """fp32, two and three pages of up to six, with the gap between chosen and other pages held to what rounding can do.

    A score is a sum of whole numbers.  The device's queries and keys are off by about 2^-20 of a head's largest: a
    query's 64 elements of up to 2^7 turn to the neighbouring number with a probability of some 2^-12 each, a
    page's bounds (a code's neighbour, e4m3 steps being 2^-4) with less.  One such turn moves a score by 127 at most
    (the largest element of a query; bounds are at most 112), so three at once, of which there are none in most runs, stay
    below 381."""
    import torch
    from paper_2508_10259_amd.runtime import DeviceContext
    spec = small_spec("f32", 2, 256, 4, 512)
    pair = Pair(spec, seed=65)
    B, cap, A = 2, 384, 2
    pre = _prefixes(spec, 297, [330, 200])
    packed, plens = pair.dev.pack_prefixes(pre)
    ctx = DeviceContext(pair.dev, B, cap, qcache=True)
    ctx.build(packed, plens)
    f64 = pair.prefixes_f64(pre)
    fed, forced = _forced(5, B, A)
    for n in (3, 2):
        ctx.select_pages(n)
        _, z = ctx.step(A, forced=forced)
        torch.cuda.synchronize()
        for b in range(B):
            r, full = Row(pair, f64[b], cap, n), QuantRow(pair.p, cap)
            full.commit(f64[b])
            err = r.step(None, fed[b], z[b].cpu().numpy(), "f32")[0]
            assert r.q.units > 3 * 127
            # and over all pages the logits are others, by far more than the device is off
            want, over_all = z[b].cpu().numpy().astype(np.float64), full.step(None, fed[b])
            assert np.abs(over_all - want).max() > 10 * err.max()
    ctx.close()


def test_rows_away_on_the_host_come_back_as_they_were():
    import torch
    from paper_2508_10259_amd import capi
    from paper_2508_10259_amd.runtime import DeviceContext
    for dtype, B, d, H, paged in (("bf16", 5, 256, 4, True), ("f32", 3, 256, 2, False)):
        spec = small_spec(dtype, 2, d, H, 512)
        pair = Pair(spec, seed=41)
        lens = [int(x) for x in np.random.default_rng(B).integers(20, 180, size=B)]
        packed, plens = pair.dev.pack_prefixes(_prefixes(spec, 41, lens))
        kw = dict(qcache=True, n_pages=B * 4 if paged else None)
        ctx, twin, plain = DeviceContext(pair.dev, B, 256, **kw), DeviceContext(pair.dev, B, 256, **kw), \
            DeviceContext(pair.dev, B, 256)
        for c in (ctx, twin, plain):
            c.build(packed, plens)
        _, forced = _forced(1, B, 4)
        ctx.step(4, forced=forced), twin.step(4, forced=forced)
        away = [1, B - 1]
        size = [ctx.row_host_bytes(lens[r]) for r in away]
        pages = [-(-lens[r] // 64) for r in away]
        assert size == [256 + 2 * n * H * (130 * (d // H) + 16) + 8 * d for n in pages]
        bufs = [torch.empty(n, dtype=torch.uint8).pin_memory() for n in size]
        ctx.offload_rows(away, bufs)
        if paged:  # another row takes the freed pages meanwhile
            for c in (ctx, twin):
                c.invalidate_rows([0])
                p0, l0 = pair.dev.pack_prefixes(_prefixes(spec, 42, [lens[0] + 60]))
                c.build_rows([0], p0, l0)
        torch.cuda.synchronize()
        plain.invalidate_rows([1])
        with pytest.raises(capi.AmsError) as e:  # an image of 8-bit pages is none of an fp16 context
            plain.reload_rows([1], bufs[:1])
        assert e.value.status == capi.AMS_EINVAL
        ctx.reload_rows(away, bufs)
        a, b = ctx.step(4, forced=forced)[1], twin.step(4, forced=forced)[1]
        torch.cuda.synchronize()
        assert torch.equal(a, b)
        for c in (ctx, twin, plain):
            c.close()


def test_shared_prefix_pages():
    import torch
    from paper_2508_10259_amd.runtime import DeviceContext
    spec = small_spec("f32", 2, 256, 4, 512)
    pair = Pair(spec, seed=33)
    B, cap, A = 4, 256, 3
    scene = W.random_gaussian((150, spec.d_model), 33, 500, dtype="f32")
    pre = [W.Prefix(np.concatenate([scene, W.make_observation(spec, 33, 1, b, 20 + 15 * b)]), np.zeros(0, np.int32)) for b in range(B)]
    packed, plens = pair.dev.pack_prefixes(pre)
    ctx = DeviceContext(pair.dev, B, cap, share_prefix=True, qcache=True)
    ctx.build(packed, plens)
    assert int((ctx.pages()[1] == B).sum()) == 2  # both full pages of the scene
    fed, forced = _forced(2, B, A)
    f64 = pair.prefixes_f64(pre)
    refs = [Row(pair, f64[b], cap) for b in range(B)]
    for s in range(2):
        news = [W.make_observation(spec, 33, 50 + s, b, 3) for b in range(B)]
        nt, nl = gpu_new_tokens(spec, news)
        _, z = ctx.step(A, nt, nl, forced=forced)
        torch.cuda.synchronize()
        for b in range(B):
            refs[b].step(news[b], fed[b], z.cpu().numpy()[b], "f32")
    ctx.close()


@pytest.mark.parametrize("dtype,n_select", [("f32", 0), ("bf16", 0), ("f32", 40)])
def test_a_decode_over_rows_in_pieces(dtype, n_select):
    """Rows long enough to be cut, and selections too: the pieces' sums are joined into the decode's output and its
    rounding errors.  40 of row 0's 41 pages are chosen, with a gap above two turns of a whole number."""
    import torch
    from paper_2508_10259_amd.runtime import DeviceContext
    spec = small_spec(dtype, 1, 128, 2, 256)
    pair = Pair(spec, seed=81)
    lens, cap, A, seed = [2600, 30, 1150], 4096, 4, 217
    pre = _prefixes(spec, seed, lens)
    packed, plens = pair.dev.pack_prefixes(pre)
    ctx = DeviceContext(pair.dev, 3, cap, qcache=True)
    ctx.build(packed, plens)
    ctx.select_pages(n_select)
    f64 = pair.prefixes_f64(pre)
    for s in range(2):
        fed, forced = _forced(s, 3, A)
        news = [W.make_observation(spec, seed, 20 + s, b, n) for b, n in enumerate((5, 1, 2))]
        nt, nl = gpu_new_tokens(spec, news)
        _, z = ctx.step(A, nt, nl, forced=forced)
        torch.cuda.synchronize()
        if s == 0:
            refs = [Row(pair, f64[b], cap, n_select) for b in range(3)]
        for b in range(3):
            refs[b].step(news[b], fed[b], z[b].cpu().numpy(), dtype)
    assert refs[0].q.units > 2 * 127
    ctx.close()


@pytest.mark.parametrize("dtype,B,share", [("bf16", 3, False), ("f32", 70, False), ("bf16", 70, True)])
def test_replayed_steps_give_what_new_ones_give(dtype, B, share):
    """Steps into the same buffers (one captured graph, replayed) and into new ones, over page ends, changed selections and rows
    that leave for the host: the same bits."""
    import torch
    from paper_2508_10259_amd.runtime import DeviceContext
    spec = small_spec(dtype, 2, 256, 4, 512)
    pair = Pair(spec, seed=91)
    lens = [int(x) for x in np.random.default_rng(B).integers(100, 300, size=B)]
    scene = W.random_gaussian((90, spec.d_model), 91, 500, dtype=dtype)
    pre = [W.Prefix(np.concatenate([scene, W.make_observation(spec, 91, 0, b, n - 90)]), np.zeros(0, np.int32))
           for b, n in enumerate(lens)]
    packed, plens = pair.dev.pack_prefixes(pre)
    kept, fresh = (DeviceContext(pair.dev, B, 512, share_prefix=share, qcache=True) for _ in range(2))
    for c in (kept, fresh):
        c.build(packed, plens)
    A = 3
    tok = torch.empty(B, A, dtype=torch.int32, device="cuda")
    logits = torch.empty(B, A, spec.n_bins, device="cuda")
    forced = torch.empty(B, A, dtype=torch.int32, device="cuda")
    now = list(lens)
    for s in range(8):
        forced.copy_(_forced(s, B, A)[1])
        n_new = [(7 * b + 5 * s) % 23 for b in range(B)]
        news = [W.make_observation(spec, 91, 20 + s, b, n) if n else None for b, n in enumerate(n_new)]
        nt, nl = gpu_new_tokens(spec, news)
        now = [x + n for x, n in zip(now, n_new)]
        for c in (kept, fresh):
            c.select_pages((0, 2, 0, 4, 3, 2, 0, 9)[s])
        if s == 5:
            row = B // 2
            for c in (kept, fresh):
                buf = torch.empty(c.row_host_bytes(now[row] - n_new[row]), dtype=torch.uint8).pin_memory()
                c.offload_rows([row], [buf])
                c.reload_rows([row], [buf])
        kept.step(A, nt, nl, tokens=tok, logits=logits, forced=forced)
        t, z = fresh.step(A, nt, nl, forced=forced.clone())
        torch.cuda.synchronize()
        assert torch.equal(z, logits) and torch.equal(t, tok), s
        assert bool(torch.isfinite(z).all())
    for c in (kept, fresh):
        c.close()


def test_flow_over_8_bit_contexts():
    import torch
    from paper_2508_10259_amd.runtime import DeviceContext, DeviceFlowHead
    spec = small_spec("f32", 2, 256, 4, 512)
    pair = Pair(spec, seed=71)
    lens, T, a, steps = [100, 61], 5, 7, 3
    pre = _prefixes(spec, 71, lens)
    packed, plens = pair.dev.pack_prefixes(pre)
    ctx = DeviceContext(pair.dev, 2, 128, qcache=True)
    ctx.build(packed, plens)
    rng = np.random.default_rng(7)
    w = [(rng.normal(size=s) * 0.1).astype(np.float32) for s in ((256, a), (256,), (a, 256))]
    head = DeviceFlowHead(spec, *w, T)
    x0 = rng.normal(size=(2, T, a)).astype(np.float32)
    x = ctx.flow(head, torch.from_numpy(x0.copy()).cuda(), 0.1, steps).cpu().numpy()
    w = [v.astype(np.float64) for v in w]
    for b, prefix in enumerate(pair.prefixes_f64(pre)):
        want = {}
        for kind in ("q", "plain"):
            row = QuantRow(pair.p, 128)
            row.commit(prefix)
            past = D.forward(pair.p, prefix)[1]
            y, dt = x0[b].astype(np.float64), 0.9 / steps
            for k in range(steps):
                e = y @ w[0].T + (0.1 + k * dt) * w[1]
                h = row.forward(e, lens[b]) if kind == "q" else D.forward(pair.p, e, start=lens[b], past=past)[0]
                y = y + dt * (h / np.sqrt(np.mean(h * h, -1, keepdims=True) + pair.p.cfg.rms_eps)) @ w[2].T
            want[kind] = y
        delta, err = np.abs(want["q"] - want["plain"]).max(), np.abs(x[b] - want["q"]).max()
        log(f"flow row {b}: error {err:.2e}, 8-bit K/V move the latent by {delta:.2e}")
        assert err <= 1e-4 + delta / 20
    ctx.close()


def test_selecting_needs_an_8_bit_context():
    from paper_2508_10259_amd import capi
    from paper_2508_10259_amd.runtime import DeviceContext
    spec = small_spec("bf16", 2, 256, 4, 512)
    pair = Pair(spec, seed=1)
    plain, ctx = DeviceContext(pair.dev, 2, 128), DeviceContext(pair.dev, 2, 128, qcache=True)
    for c, n in ((plain, 2), (ctx, -1)):
        with pytest.raises(capi.AmsError) as e:
            c.select_pages(n)
        assert e.value.status == capi.AMS_EINVAL
    plain.close()
    ctx.close()
