"""The head's losses and gradients on the GPU against their definition in float64, at
the sizes and masks where tiles, strips, pieces and lists end (bounds: head_common)."""
import math

import pytest
import torch

from paper_2608_16188_amd import vmoe_head as H

from .gpu_common import say
from .head_common import W1, W2, Case, Data
from .train_common import close, same_bits

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    torch.cuda.set_device(0)
    yield
    torch.cuda.synchronize()
    torch.cuda.empty_cache()


CASES = {
    "one_row": Case(1, 64, 10),
    "one_class": Case(5, 8, 1, k=1, t=2.0),
    "two_classes_f32": Case(9, 16, 2, k=2, t=0.5, dtype="f32"),
    "narrow": Case(33, 8, 100, k=3),
    # waves whose strips hold no class, at scales that are no powers of two
    **{f"few_classes_t{t}": Case(n, 16, 10, k=2, t=t, dtype=dt, labels=lab)
       for t, n, dt, lab in ((3.0, 5, "bf16", True), (0.7, 70, "bf16", True),
                             (1.5, 70, "f32", False), (5.3, 300, "f32", True),
                             (0.11, 9, "f32", False), (11.0, 90, "bf16", False))},
    "tile_edge_below": Case(255, 72, 255, ignored=0.2),
    "tile_edge": Case(256, 64, 256, weighted=True),
    "tile_edge_above": Case(257, 192, 257, k=5, t=2.0),
    "tile_edge_f32": Case(128, 32, 128, dtype="f32"),
    "past_tile_f32": Case(129, 40, 129, k=4, t=3.0, dtype="f32", ignored=0.3),
    "odd_classes": Case(300, 128, 1003, k=17, t=2.0, ignored=0.4, missing=0.3, weighted=True),
    "odd_classes_f32": Case(300, 136, 1003, k=17, t=2.0, dtype="f32", ignored=0.4, missing=0.3,
                            weighted=True),
    "no_bias": Case(100, 96, 777, bias=False),
    "no_bias_f32": Case(100, 96, 777, bias=False, dtype="f32"),
    "teacher_alone": Case(130, 64, 513, k=64, t=1.5, labels=False),
    "teacher_alone_t1": Case(130, 64, 513, k=63, labels=False, missing=0.9),
    "teacher_t1": Case(70, 320, 900, k=65),
    "teacher_cold": Case(64, 64, 300, k=10, t=0.25),
    "teacher_hot": Case(64, 64, 300, k=10, t=50.0, dtype="f32"),
    "longest_list": Case(40, 64, 999, k=256, t=2.0, missing=0.2),
    "longest_list_f32": Case(40, 64, 999, k=256, t=2.0, dtype="f32", labels=False),
    "list_of_all": Case(50, 48, 10, k=10, t=2.0),
    "nearly_all_out": Case(1500, 64, 700, ignored=0.995),
    "all_out": Case(300, 64, 700, k=4, ignored=1.0),
    "all_out_f32": Case(30, 64, 70, k=4, ignored=1.0, dtype="f32"),
    "empty": Case(0, 64, 700, k=4),
    "summed": Case(200, 64, 300, k=4, t=2.0, reduction=H.VMOE_REDUCE_SUM, weighted=True,
                   ignored=0.1),
    "few_rows_at_most": Case(64, 72, 1001, k=5, t=2.0, weighted=True, missing=0.2),
    "few_rows_at_most_f32": Case(64, 72, 1001, k=5, t=2.0, dtype="f32", ignored=0.3),
    "few_rows_passed": Case(65, 72, 1001, k=5, t=2.0, weighted=True, missing=0.2),
    "few_rows_passed_f32": Case(65, 72, 1001, k=5, t=2.0, dtype="f32", ignored=0.3),
    "row_blocks_of_1024": Case(70001, 16, 33, k=2, t=2.0, ignored=0.4, weighted=True),
    "row_blocks_of_1024_f32": Case(66000, 8, 17, dtype="f32", ignored=0.7),
    "mark_blocks": Case(2100, 64, 90, k=2, ignored=0.5, weighted=True),
    "wide": Case(20, 4096, 500),
    "wide_f32": Case(20, 2056, 500, dtype="f32", k=3, t=2.0),
    "many_classes_few_rows": Case(3, 64, 30001, k=8, t=2.0),
    "many_rows_few_classes": Case(9000, 64, 17),
    "many_rows_few_classes_f32": Case(9000, 64, 17, dtype="f32"),
    # more logits than the kernels of few take: tiles, and z formed twice
    "tiles_below": Case(1279, 72, 3583, ignored=0.2),
    "tiles_even": Case(1280, 64, 3584, weighted=True),
    "tiles_even_taught": Case(1280, 64, 3584, k=3, t=2.0),
    "tiles_above": Case(1281, 192, 3585, k=5, t=2.0),
    "tiles_odd": Case(1300, 128, 4003, k=17, t=2.0, ignored=0.4, missing=0.3, weighted=True),
    "tiles_no_bias": Case(1100, 96, 4100, bias=False),
    "tiles_teacher_alone": Case(1290, 64, 3841, k=64, t=1.5, labels=False),
    "tiles_teacher_alone_t1": Case(1290, 64, 3841, k=63, labels=False, missing=0.9),
    "tiles_teacher_t1": Case(1300, 320, 3700, k=65),
    "tiles_longest_list": Case(1281, 64, 3999, k=256, t=2.0, missing=0.2),
    "tiles_nearly_all_out": Case(2100, 64, 3000, k=3, ignored=0.995),
    "tiles_all_out": Case(1300, 64, 4000, k=4, ignored=1.0),
    "tiles_summed": Case(1200, 64, 4000, k=4, t=2.0, reduction=H.VMOE_REDUCE_SUM, weighted=True,
                         ignored=0.1),
    "tiles_one_class": Case(131100, 8, 1, k=1, t=3.0),
    "tiles_few_classes_t0.7": Case(131100, 16, 10, k=2, t=0.7),
    "tiles_few_classes_t5.3_f32": Case(50000, 16, 10, k=2, t=5.3, dtype="f32"),
    "tiles_below_f32": Case(1087, 40, 1663, dtype="f32", ignored=0.1),
    "tiles_odd_f32": Case(1000, 136, 2003, k=17, t=2.0, dtype="f32", ignored=0.4, missing=0.3,
                          weighted=True),
    "tiles_longest_list_f32": Case(1000, 64, 2003, k=256, t=2.0, dtype="f32", labels=False),
    "tiles_all_out_f32": Case(1000, 64, 2003, k=4, dtype="f32", ignored=1.0),
    # f32 tiles whose z is kept
    "kept_f32": Case(1088, 192, 1664, dtype="f32", weighted=True),
    "kept_odd_f32": Case(1000, 200, 2003, k=17, t=2.0, dtype="f32", ignored=0.4, missing=0.3,
                         weighted=True),
    "kept_teacher_alone_f32": Case(1089, 256, 1665, k=100, t=3.0, dtype="f32", labels=False,
                                   bias=False),
    "kept_all_out_f32": Case(1000, 200, 2003, k=4, dtype="f32", ignored=1.0),
    "narrow_tiles": Case(600, 192, 4000, k=2),
    "long": Case(5000, 256, 5001, weighted=True, ignored=0.1),
}


def check(c, data=None, **kw):
    data = data or Data(c)
    got = data.run(**kw)
    ref, bound = data.reference()
    for k in got:
        close(k, got[k], ref[k], bound[k])
    return data, got


@pytest.mark.parametrize("name", CASES)
def test_against_float64(name):
    say("head loss", name, CASES[name])
    check(CASES[name])


@pytest.mark.parametrize("dtype, n, d, v", [
    ("bf16", 8192, 32, 70001), ("f32", 4100, 32, 66001),
    # as many rows as dx needs no ranges of classes for
    ("bf16", 70000, 16, 9000), ("f32", 66000, 8, 9000)])
def test_several_pieces_of_the_classes(dtype, n, d, v):
    say("head loss pieces", dtype, n, d, v)
    c = Case(n, d, v, k=3, t=2.0, dtype=dtype, ignored=0.3)
    assert n * v * (2 if dtype == "bf16" else 4) > 2 ** 30
    assert H.vmoe_head_loss_bwd_workspace_bytes(c.shape()) < n * v * 4
    check(c)
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_gradient_against_differences(dtype):
    """Directional derivatives of the float64 objective in x, weight and bias."""
    c = Case(40, 48, 90, k=7, t=2.0, dtype=dtype, weighted=True, ignored=0.2, missing=0.2)
    d = Data(c)
    got = d.run()
    _, bound = d.reference()
    x, w, b = (t.double() for t in (d.x, d.weight, d.bias))
    rw, label, there, taught = d.masks()
    g = torch.Generator(device="cuda").manual_seed(5)
    y = torch.where(label, d.labels, 0).long()
    yt = torch.where(there, d.idx, 0).long()
    t = torch.where(there, d.logits.double() / c.t, -1e30)
    q = torch.softmax(torch.where(taught[:, None], t, 0.0), 1) * there

    def objective(x, w, b):
        z = torch.mm(x, w.T) + b
        a = -(torch.log_softmax(z, 1).gather(1, y[:, None])[:, 0])
        kd = -(q * torch.log_softmax(z / c.t, 1).gather(1, yt)).sum(1) * c.t ** 2
        return W1 * (rw * label * a).sum() / (rw * label).sum() + \
            W2 * (rw * taught * kd).sum() / (rw * taught).sum()

    for name, at in (("dx", x), ("dweight", w), ("dbias", b)):
        along = torch.randn(at.shape, dtype=torch.float64, device="cuda", generator=g)
        move = [torch.zeros_like(t) for t in (x, w, b)]
        move[("dx", "dweight", "dbias").index(name)] = 1e-5 * along
        slope = (objective(*(p + m for p, m in zip((x, w, b), move))) -
                 objective(*(p - m for p, m in zip((x, w, b), move)))) / 2e-5
        have = got[name].double()
        # differences of values about 3 at steps of 1e-5: 3 eps / 1e-5, and a third
        # derivative at 1e-10
        allowed = float((bound[name] * along.abs()).sum()) + 1e-9 * float(along.abs().sum())
        assert abs(float((have * along).sum() - slope)) <= allowed, name


@pytest.mark.parametrize("want", [("dx",), ("dweight",), ("dbias",), ("dweight", "dbias"),
                                  ("dx", "dbias"), ()])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_gradients_that_are_not_wanted(want, dtype):
    d = Data(Case(150, 64, 333, k=4, t=2.0, dtype=dtype, ignored=0.2))
    full, part = d.run(), d.run(want=want, row_losses=False)
    assert set(part) == {"losses", *want}
    ref, bound = d.reference()
    for k in part:
        close(k, part[k], ref[k], bound[k])
        if k != "dbias":  # whose own product may be cut otherwise
            assert same_bits(part[k], full[k]), k


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_weights_of_the_losses(dtype):
    d = Data(Case(120, 64, 200, k=6, t=2.0, dtype=dtype, ignored=0.1))
    for w1, w2 in ((1.0, 0.0), (0.0, 1.0), (-0.5, 2.0), (0.0, 0.0)):
        got = d.run(w1=w1, w2=w2)
        ref, bound = d.reference(w1=w1, w2=w2)
        for k in got:
            close(k, got[k], ref[k], bound[k])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n, v", [(40, 200), (300, 200), (1300, 4000)])
@pytest.mark.parametrize("w1, w2", [(0.5, -0.5), (-1.0, 0.25), (0.0, 1.0), (0.0, 0.0)])
@pytest.mark.parametrize("temperature", [1.0, 2.0])
def test_signs_of_the_losses(dtype, n, v, w1, w2, temperature):
    """At temperature 1 with opposite weights the two softmaxes cancel, the targets stay."""
    d = Data(Case(n, 64, v, k=3, t=temperature, dtype=dtype, weighted=True, ignored=0.2))
    got = d.run(w1=w1, w2=w2)
    ref, bound = d.reference(w1, w2)
    for k in got:
        close(k, got[k], ref[k], bound[k])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n, v, reduction", [(40, 200, 0), (300, 200, 0), (300, 200, 1),
                                             (1300, 4000, 0), (1300, 4000, 1)])
def test_rows_of_negative_weight(dtype, n, v, reduction):
    c = Case(n, 64, v, k=3, t=2.0, dtype=dtype, reduction=reduction)
    d = Data(c)
    g = torch.Generator(device="cuda").manual_seed(9)
    d.row_weight = torch.randn(n, device="cuda", generator=g) + 0.5
    check(c, d)
    label = Data(Case(n, 64, v, dtype=dtype, reduction=reduction))
    label.row_weight = d.row_weight
    check(label.case, label)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_weight_of_a_loss_that_is_not_there(dtype):
    """However large it is, it moves nothing."""
    for kw in (dict(), dict(k=3, labels=False)):
        d = Data(Case(100, 64, 300, dtype=dtype, reduction=H.VMOE_REDUCE_SUM, **kw))
        big = dict(w1=1.0, w2=1e30) if d.case.labels else dict(w1=1e30, w2=1.0)
        a, b = d.run(w1=1.0, w2=1.0), d.run(**big)
        for k in a:
            assert same_bits(a[k], b[k]), k


@pytest.mark.parametrize("n", [40, 70])
def test_weights_beyond_2_gib(n):
    """Offsets past 32 bits in the head's weight and its gradient, and several pieces."""
    d, v = 1024, 1100003
    assert v * d * 2 > 2 ** 31
    c = Case(n, d, v, k=2, t=2.0, bias=False)
    data = Data(c)
    data.labels[:4] = torch.tensor([v - 1, v - 2, 0, v - 300], dtype=torch.int32)
    say("head loss beyond 2 GiB", c)
    got = data.run(want=("dx", "dweight"))
    ref, bound = data.reference()
    for k in ("losses", "row_losses", "dx"):
        close(k, got[k], ref[k], bound[k])
    for rows in (slice(0, 300), slice(v // 2, v // 2 + 300), slice(v - 300, v)):
        close("dweight", got["dweight"][rows], ref["dweight"][rows], bound["dweight"][rows])
    torch.cuda.empty_cache()


@pytest.mark.parametrize("c", [Case(90, 64, 200, k=6, t=2.0), Case(1300, 64, 4000, k=6, t=2.0),
                               Case(1000, 192, 2003, k=6, t=2.0, dtype="f32")])
def test_several_backwards_of_one_forward(c):
    d = Data(c)
    s = d.case.shape()
    first = d.run()
    before = d.saved.clone()
    ws = torch.full((H.vmoe_head_loss_bwd_workspace_bytes(s),), 0x7F, dtype=torch.uint8,
                    device="cuda")
    dx = torch.empty_like(first["dx"])
    for w1, w2 in ((1.0, 0.0), (W1, W2)):
        H.vmoe_head_loss_bwd(s, d.weight, d.saved, w1, w2, dx, None, None, ws)
    assert same_bits(dx, first["dx"])
    assert torch.equal(d.saved, before)


@pytest.mark.parametrize("name", ["odd_classes", "odd_classes_f32", "long", "mark_blocks",
                                  "many_rows_few_classes", "tiles_odd", "tiles_odd_f32",
                                  "kept_odd_f32"])
def test_same_bits_every_time(name):
    d = Data(CASES[name])
    a, b = d.run(), d.run(spoil=False)
    for k in a:
        assert same_bits(a[k], b[k]), k


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("temperature", [1.0, 0.25, 3.0])
def test_teachers_logits_at_their_limits(dtype, temperature):
    """-infinity is no entry, the type's lowest value is one; a list of nothing else
    counts evenly; a sure teacher is a label."""
    c = Case(8, 64, 50, k=5, t=temperature, dtype=dtype)
    d = Data(c)
    low = torch.finfo(torch.float32).min
    d.idx = torch.arange(40, device="cuda", dtype=torch.int32).view(8, 5)
    d.logits[0] = -math.inf
    d.logits[1] = low
    d.logits[2, :4] = low
    d.logits[3, 1:] = -math.inf
    d.logits[4] = 0.0
    d.logits[5] = torch.tensor([1e30, 0.0, -1e30, 5.0, low], device="cuda")
    d.logits[6] = -1e-30
    d.idx[7] = 3  # one class five times
    _, got = check(c, d)
    assert float(got["row_losses"][0, 1]) == 0.0
    assert (got["losses"][3] == 7).all()


def test_a_nan_logit_of_an_entry_is_not_hidden():
    d = Data(Case(4, 64, 50, k=3))
    d.logits[2, 1] = float("nan")
    got = d.run(spoil=False)
    assert torch.isnan(got["row_losses"][2, 1]) and torch.isfinite(got["row_losses"][[0, 1, 3]]).all()
    assert torch.isnan(got["losses"][1]) and torch.isfinite(got["losses"][0])
    assert torch.isfinite(got["dx"][[0, 1, 3]]).all() and torch.isnan(got["dx"][2]).any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_weights_that_cancel(dtype):
    """A mean over weights whose sum is 0 is 0, and so is its gradient."""
    c = Case(6, 64, 40, dtype=dtype)
    d = Data(c)
    d.row_weight = torch.tensor([1.0, -1.0, 2.0, -2.0, 0.5, -0.5], device="cuda")
    got = d.run()
    assert got["losses"].tolist() == [0.0, 0.0, 0.0, 0.0]
    for k in ("dx", "dweight", "dbias"):
        assert (got[k] == 0).all(), k
    assert (got["row_losses"][:, 0] > 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [40, 200, 6400])
@pytest.mark.parametrize("t", [1.0, 1.7])
@pytest.mark.parametrize("lowest", [False, True])
def test_classes_masked_by_the_bias(dtype, n, t, lowest):
    """-infinity, or the type's lowest value, at classes that are not to be there, whole
    strips of them too: as a head over the others. An entry of such a class that has
    no share of its list (exp(-200) is 0 in f32) takes no part."""
    v = 700
    c = Case(n, 64, v, k=4, t=t, dtype=dtype)
    d = Data(c)
    g = torch.Generator(device="cuda").manual_seed(3)
    keep = torch.rand(v, device="cuda", generator=g) < 0.6
    keep[256:520] = False
    kept = torch.nonzero(keep)[:, 0]
    pick = lambda *s: kept[torch.randint(0, len(kept), s, device="cuda",  # noqa: E731
                                         generator=g)].to(torch.int32)
    d.labels, d.idx = pick(n), pick(n, 4)
    d.idx[::2, 3] = 300
    d.logits[::2, 3] = -200.0 * t
    mask = torch.finfo(d.bias.dtype).min if lowest else -math.inf
    d.bias = torch.where(keep, d.bias, mask)
    got = d.run()
    to = torch.full((v,), -1, dtype=torch.int32, device="cuda")
    to[kept] = torch.arange(len(kept), dtype=torch.int32, device="cuda")
    few = Data(Case(n, 64, len(kept), k=4, t=t, dtype=dtype))
    few.x, few.weight, few.bias = d.x, d.weight[kept], d.bias[kept]
    few.labels, few.idx, few.logits = to[d.labels.long()], to[d.idx.long()], d.logits
    ref, bound = few.reference()
    # (the bounds' counts of strips and of sums over classes are of 700 here)
    more = 1.0 + (v + 80) / (len(kept) + 80)
    for k in ("losses", "row_losses", "dx"):
        close(k, got[k], ref[k], more * bound[k])
    for k in ("dweight", "dbias"):
        close(k, got[k][kept], ref[k], more * bound[k])
        assert (got[k][~keep] == 0).all(), k


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shift", [-300.0, 300.0])
@pytest.mark.parametrize("n, v", [(70, 130), (1300, 4000)])
def test_large_logits(dtype, shift, n, v):
    """Logits far from 0 and rows that are certain."""
    c = Case(n, 64, v, k=4, t=2.0, dtype=dtype)
    d = Data(c)
    d.bias = (d.bias.float() + shift).to(d.bias.dtype)
    d.x = (4 * d.x.float()).to(d.x.dtype)
    check(c, d)


def test_perfect_rows_have_small_losses():
    """A row whose label has all the mass: the loss is 0 to the logits' rounding."""
    c = Case(16, 64, 300, dtype="f32")
    d = Data(c)
    d.x = 60 * d.weight[d.labels.long()]
    _, got = check(c, d)
    assert float(got["row_losses"][:, 0].abs().max()) < 1e-4


def test_on_another_stream_and_handle():
    d = Data(CASES["odd_classes"])
    want = d.run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for stream in (side, side.cuda_stream):
        got = d.run(stream=stream)
        for k in want:
            assert same_bits(got[k], want[k]), k


def test_streams_side_by_side():
    """Two heads at once, each with its own buffers."""
    ds = [Data(CASES[k]) for k in ("odd_classes", "tile_edge_above", "tiles_odd", "kept_odd_f32")]
    want = [d.run() for d in ds]
    streams = [torch.cuda.Stream() for _ in ds]
    out = []
    for d, st in zip(ds, streams):
        c, s = d.case, d.case.shape()
        new = lambda *sh, dt=d.x.dtype: torch.empty(*sh, dtype=dt, device="cuda")  # noqa: E731
        u8 = lambda k: new(max(k, 16), dt=torch.uint8)  # noqa: E731
        o = dict(losses=new(4, dt=torch.float32), row_losses=new(c.n, 2, dt=torch.float32),
                 dx=new(c.n, c.d), dweight=new(c.v, c.d), dbias=new(c.v))
        bufs = (u8(H.vmoe_head_loss_saved_bytes(s)), u8(H.vmoe_head_loss_fwd_workspace_bytes(s)),
                u8(H.vmoe_head_loss_bwd_workspace_bytes(s)))
        out.append((d, st, s, o, bufs))
    torch.cuda.synchronize()
    for _ in range(5):
        for d, st, s, o, (saved, fw, bw) in out:
            H.vmoe_head_loss_fwd(s, d.x, d.weight, d.bias, d.labels, d.idx, d.logits,
                                 d.row_weight, o["losses"], o["row_losses"], saved, fw, st)
            H.vmoe_head_loss_bwd(s, d.weight, saved, W1, W2, o["dx"], o["dweight"], o["dbias"],
                                 bw, st)
    torch.cuda.synchronize()
    for (d, _, _, o, _), w in zip(out, want):
        for k in w:
            assert same_bits(o[k], w[k]), k


@pytest.mark.parametrize("dtype, n, d_model, v", [
    ("bf16", 400, 64, 600), ("f32", 400, 64, 600), ("bf16", 1300, 64, 4000),
    ("f32", 1000, 64, 2003), ("f32", 1000, 192, 2003)])
def test_captured_and_replayed(dtype, n, d_model, v):
    """One graph of forward and backward, replayed on other inputs (another number of
    live rows among them), with eager work in between."""
    c = Case(n, d_model, v, k=4, t=2.0, dtype=dtype, ignored=0.3, weighted=True)
    s, act = c.shape(), torch.bfloat16 if dtype == "bf16" else torch.float32
    d = Data(c)
    new = lambda *sh, dt=act: torch.empty(*sh, dtype=dt, device="cuda")  # noqa: E731
    o = dict(losses=new(4, dt=torch.float32), row_losses=new(c.n, 2, dt=torch.float32),
             dx=new(c.n, c.d), dweight=new(c.v, c.d), dbias=new(c.v))
    saved, fw, bw = (new(k, dt=torch.uint8) for k in (
        H.vmoe_head_loss_saved_bytes(s), H.vmoe_head_loss_fwd_workspace_bytes(s),
        H.vmoe_head_loss_bwd_workspace_bytes(s)))

    def step():
        H.vmoe_head_loss_fwd(s, d.x, d.weight, d.bias, d.labels, d.idx, d.logits, d.row_weight,
                             o["losses"], o["row_losses"], saved, fw)
        H.vmoe_head_loss_bwd(s, d.weight, saved, W1, W2, o["dx"], o["dweight"], o["dbias"], bw)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k, ignored in enumerate((0.3, 0.9, 0.0, 1.0, 0.5)):
        e = Data(Case(n, d_model, v, k=4, t=2.0, dtype=dtype, ignored=ignored, weighted=True,
                      seed=10 + k))
        for a in ("x", "weight", "bias", "labels", "idx", "logits", "row_weight"):
            getattr(d, a).copy_(getattr(e, a))
        for t in (saved, fw, bw):
            t.fill_(0xFF)
        graph.replay()
        torch.cuda.synchronize()
        want = e.run()
        for name in want:
            assert same_bits(o[name], want[name]), (k, name)
