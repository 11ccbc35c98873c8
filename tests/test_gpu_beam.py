"""GPU parity of beam search's step and of the states' reordering.

Places are compared exactly with an order formed in 64 bits on the CPU; random inputs leave gaps between
candidates far above the 2^-22 that a sum of exponentials in fp32 may be off, and equal logits within
a beam, or equal beams, are equal on both sides.  Scores: that sum, and half a step of the output."""
import math

import pytest
import torch

import paper_1810_09958_amd as isam

pytestmark = pytest.mark.gpu


def reference(logits, scores, width, finished=None, end=-1):
    b, n, V = logits.shape
    l, s = logits.cpu().double(), scores.cpu().double()
    total = torch.full((b, n, V), -math.inf, dtype=torch.float64)
    for i in range(b):
        for j in range(n):
            row, sc = l[i, j], float(s[i, j])
            if finished is not None and bool(finished[i, j]):
                if sc == sc:
                    total[i, j, end] = sc
            elif sc == sc and sc != -math.inf and not row.isnan().any() and row.max() != -math.inf and row.max() != math.inf:
                total[i, j] = sc + (row - torch.logsumexp(row, 0))
    flat = total.view(b, n * V)
    best, at = flat.sort(dim=1, descending=True, stable=True)
    best, at = best[:, :width], at[:, :width]
    parent, token = at // V, at % V
    done = token == end
    if finished is not None:
        done |= finished.cpu().bool().gather(1, parent)
    return best, parent, token, done


def compare(logits, scores, width=None, finished=None, end=-1):
    w = logits.shape[1] if width is None else width
    want = reference(logits, scores, w, finished, end)
    got = isam.beam_step(logits, scores, width=width, finished=finished, end=end)
    torch.cuda.synchronize()
    assert torch.equal(got[1].cpu().long(), want[1]), (got[1], want[1])
    assert torch.equal(got[2].cpu().long(), want[2])
    assert torch.equal(got[3].cpu(), want[3])
    a, r = got[0].cpu().double(), want[0]
    inf = r == -math.inf
    assert torch.equal(a[inf], r[inf])
    assert ((a - r)[~inf].abs() <= 2.0 ** -22 + 2.0 ** -24 * r[~inf].abs()).all()
    return got


def inputs(b, n, V, dtype, seed=0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn((b, n, V), generator=g) * 3).to(dtype).cuda(), (torch.rand((b, n), generator=g) * -20).cuda()


DTYPES = pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])


@DTYPES
@pytest.mark.parametrize("V", [1, 2, 3, 7, 8, 64, 255, 256, 257, 1000, 4095, 4096, 4097, 9001, 50000])
def test_vocabularies(V, dtype):
    compare(*inputs(3, 4, V, dtype, seed=V))
    if V > 8:
        compare(*inputs(2, 1, V, dtype, seed=V), width=8)


@DTYPES
@pytest.mark.parametrize("n,w", [(1, 1), (1, 5), (2, 2), (3, 7), (8, 8), (16, 16), (16, 3), (64, 64), (5, 64)])
def test_beams(n, w, dtype):
    compare(*inputs(4, n, 700, dtype, seed=n), width=w)
    compare(*inputs(2, n, 9000, dtype, seed=w), width=w)


@DTYPES
def test_finished_beams(dtype):
    for seed in range(6):
        logits, scores = inputs(5, 4, 300, dtype, seed)
        g = torch.Generator().manual_seed(seed)
        fin = (torch.rand((5, 4), generator=g) < 0.5).cuda()
        fin[0] = True                                     # all of a text's beams: the rest of the candidates have -inf
        fin[1] = False
        for end in (0, 2, 299):
            compare(logits, scores, finished=fin, end=end)
            compare(logits, scores, finished=fin, end=end, width=9)
    compare(logits[..., :3].contiguous(), scores, finished=fin, end=1, width=12)


@DTYPES
def test_ties_and_masks(dtype):
    # equal logits, equal beams: the lowest place; both zeros are equal
    logits = torch.zeros((2, 3, 5000), device="cuda", dtype=dtype)
    logits[..., ::2] = -0.0
    scores = torch.zeros((2, 3), device="cuda")
    compare(logits, scores, width=20)
    scores[:, 1:] = -math.inf                             # a first step: one beam stands for all
    compare(logits, scores, width=20)
    # masked tokens, a beam with nothing left, all beams with nothing left
    logits, scores = inputs(3, 3, 40, dtype, 1)
    logits[0, :, 5:] = -math.inf
    logits[1, 1] = -math.inf
    logits[2] = -math.inf
    compare(logits, scores, width=30)
    logits, scores = inputs(2, 3, 6000, dtype, 2)
    logits[0, :, 100:5900] = torch.finfo(dtype).min       # the type's lowest value is a value
    logits[1, 0, 17] = float("nan")
    logits[1, 1, 5003] = math.inf
    scores[0, 2] = float("nan")
    compare(logits, scores, width=40)


@DTYPES
def test_large_and_small_logits(dtype):
    logits, scores = inputs(2, 4, 3000, dtype, 3)
    compare(logits * 100, scores)
    compare(logits * 0.001 + 500, scores)


@DTYPES
def test_strides(dtype):
    # logits as the last rows of a larger tensor, off 16 bytes, and beams outside of texts
    logits, scores = inputs(3, 4, 601, dtype, 4)
    wide = torch.full((3, 4, 640), 1e4, device="cuda", dtype=dtype)
    wide[..., 3:604] = logits
    compare(wide[..., 3:604], scores)
    turned = logits.transpose(0, 1).contiguous().transpose(0, 1)
    compare(turned, scores)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.int32, torch.uint8, torch.int64])
@pytest.mark.parametrize("shape,dim", [((2, 6, 40), 1), ((6, 7), 0), ((3, 2, 6, 1), 2), ((6,), 0), ((2, 6, 5000), 1), ((6, 3, 4), 0)])
def test_reorder(shape, dim, dtype):
    g = torch.Generator().manual_seed(dim)
    s = torch.randint(0, 100, shape, generator=g).to(dtype).cuda()
    for w in (1, 3, 5):
        p = torch.randint(0, 3, (2, w), generator=g).int().cuda()
        got = isam.beam_reorder(s, p, dim=dim)
        rows = (p.cpu().long() + torch.arange(2)[:, None] * 3).reshape(-1)
        assert torch.equal(got.cpu(), s.cpu().index_select(dim, rows))
    p = torch.tensor([[0, -1], [3, 2]], dtype=torch.int32, device="cuda")   # outside: zeros
    got = isam.beam_reorder(s, p, dim=dim).cpu()
    assert (got.select(dim, 1) == 0).all() and (got.select(dim, 2) == 0).all()
    assert torch.equal(got.select(dim, 3), s.cpu().select(dim, 5))


def test_streams_repeats_and_graph_replays():
    logits, scores = inputs(3, 4, 9000, torch.float32, 5)
    state = torch.randn((2, 12, 33), device="cuda")
    out = dict(scores_out=torch.empty((3, 4), device="cuda"), parent=torch.empty((3, 4), device="cuda", dtype=torch.int32),
               token=torch.empty((3, 4), device="cuda", dtype=torch.int32), finished_out=torch.empty((3, 4), device="cuda", dtype=torch.bool),
               workspace=torch.empty(isam.beam_step_workspace_size(3, 4, 9000, 4, isam.ISAM_F32), device="cuda", dtype=torch.uint8))
    moved = torch.empty_like(state)

    def step():
        isam.beam_step(logits, scores, end=2, **out)
        isam.beam_reorder(state, out["parent"], dim=1, out=moved)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(3):
        logits.copy_(inputs(3, 4, 9000, torch.float32, 10 + i)[0])
        want = compare(logits, scores, end=2)
        other = isam.beam_reorder(state, want[1], dim=1)
        for _ in range(2):
            graph.replay()
            torch.cuda.synchronize()
            for a, b in zip((out["scores_out"], out["parent"], out["token"], out["finished_out"], moved), (*want, other)):
                assert torch.equal(a, b)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = isam.beam_step(logits, scores, end=2)
    torch.cuda.current_stream().wait_stream(s)
    for a, b in zip(got, want):
        assert torch.equal(a, b)


def test_refusals():
    logits, scores = inputs(2, 3, 50, torch.float32)
    fin = torch.zeros((2, 3), device="cuda", dtype=torch.bool)
    with pytest.raises(ValueError):
        isam.beam_step(logits[0], scores)
    with pytest.raises(ValueError):
        isam.beam_step(logits, scores[:, :2])
    with pytest.raises(TypeError):
        isam.beam_step(logits, scores.double())
    with pytest.raises(TypeError):
        isam.beam_step(logits.half(), scores)
    with pytest.raises(TypeError):
        isam.beam_step(logits, scores, finished=fin.float(), end=1)
    with pytest.raises(ValueError):
        isam.beam_step(logits.cpu(), scores.cpu())
    for kw in (dict(width=65), dict(width=0), dict(end=50), dict(finished=fin), dict(width=200)):
        with pytest.raises((isam.IsamError, RuntimeError)):
            isam.beam_step(logits, scores, **kw)
    with pytest.raises(isam.IsamError) as e:
        isam.beam_step(logits, scores, workspace=torch.empty(16, device="cuda", dtype=torch.uint8))
    assert e.value.status == 3
    p = torch.zeros((2, 3), device="cuda", dtype=torch.int32)
    state = torch.zeros((4, 6, 5), device="cuda")
    for bad in (lambda: isam.beam_reorder(state, p, dim=2), lambda: isam.beam_reorder(state.transpose(0, 1), p),
                lambda: isam.beam_reorder(state, p[0], dim=1), lambda: isam.beam_reorder(state, p, dim=3),
                lambda: isam.beam_reorder(state, p, dim=1, out=torch.zeros((4, 5, 5), device="cuda"))):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(TypeError):
        isam.beam_reorder(state, p.long(), dim=1)
    with pytest.raises(isam.IsamError):
        isam.beam_reorder(state, p, dim=1, out=state)


@DTYPES
@pytest.mark.parametrize("width", [1, 4, 16, 17, 64])
def test_equal_logits_and_nan_of_all_bits(width, dtype):
    """More equal values than the candidates' list holds: the lowest places; a row of NaN with every bit set has no
    candidates."""
    logits = torch.zeros((2, 3, 9000), dtype=dtype, device="cuda")
    scores = torch.tensor([[-1.0, -2.0, -2.0], [0.0, 0.0, -1.0]], device="cuda")
    compare(logits, scores, width=width)
    logits[:, :, 4000:] = 1.0
    compare(logits, scores, width=width)
    bits = logits.view(torch.int16 if dtype is torch.bfloat16 else torch.int32)
    bits[0, 0] = -1
    bits[1, :2] = -1
    compare(logits, scores, width=width)


@DTYPES
def test_one_beam_far_ahead(dtype):
    """The best all come from one beam's parts, whose lists have to be followed to their ends."""
    logits, scores = inputs(2, 16, 20000, dtype, seed=5)
    scores[0, 3] += 100
    scores[1, 15] += 100
    for width in (2, 16, 64):
        compare(logits, scores, width=width)


@DTYPES
@pytest.mark.parametrize("width", [1, 4, 16, 17, 64])
@pytest.mark.parametrize("V", [4096, 9000])
def test_nan_before_finite_values(V, width, dtype):
    """NaN of both signs in the first values that most threads of a workgroup hold, finite ones behind: the row has no
    candidates, and its neighbours keep theirs."""
    logits, scores = inputs(2, 4, V, dtype, seed=V)
    bits = logits.view(torch.int16 if dtype is torch.bfloat16 else torch.int32)
    low, high = (-64, 0x7fc0) if dtype is torch.bfloat16 else (-4194304, 0x7fc00000)     # NaN below -inf and above inf by their bits
    rising = torch.arange(V, device="cuda", dtype=torch.float32).to(dtype)
    for b, i, first in ((0, 0, low), (0, 2, high), (1, 3, low)):
        logits[b, i] = rising
        bits[b, i, :1024] = low
        bits[b, i, 0:2048:8] = first
        bits[b, i, 1:2048:8] = first
        logits[b, i, 96:104] = 2.0                        # one thread that has a value among them
    compare(logits, scores, width=width)


@DTYPES
@pytest.mark.parametrize("width", [1, 4, 16, 17, 64])
@pytest.mark.parametrize("V", [4097, 8193, 12000])
def test_nan_among_masked_logits(V, width, dtype):
    """A NaN whose neighbours are all -inf, or the row's last logit: the beam has no candidates."""
    logits, scores = inputs(2, 4, V, dtype, seed=V)
    scores[:, 1:3] += 50                                  # the beams with a NaN would win
    logits[0, 1, V - 1] = float("nan")
    logits[1, 2, V - 1] = -float("nan")
    compare(logits, scores, width=width)
    logits, scores = inputs(2, 4, V, dtype, seed=V)
    scores[:, 1:3] += 50
    logits[:, :, 4096:] = -math.inf                       # a part masked to -inf, with and without a NaN in it
    for b, i, at in ((0, 1, 4096), (0, 2, V - 1), (1, 1, (4096 + V) // 2)):
        logits[b, i, at] = float("nan")
    compare(logits, scores, width=width)


@DTYPES
@pytest.mark.parametrize("V", [300, 5000, 20000])
def test_beams_closer_than_fp32_tells(V, dtype):
    """Two beams whose best candidates differ by no more than half a step of an fp32 score below 4 (2^-23), and by more than
    64 bits leave unsure: the order is that of 64 bits."""
    logits, scores = inputs(200, 2, V, dtype, seed=V + 1)
    l = logits.cpu().double()
    best = l.max(-1).values - torch.logsumexp(l, -1)
    scores[:, 0] = 0.0
    scores[:, 1] = (best[:, 0] - best[:, 1]).float().cuda()          # the nearest fp32 to a tie
    gap = (best[:, 0] - best[:, 1] - scores[:, 1].cpu().double()).abs()
    assert (gap <= 2.0 ** -23).all() and (gap > 2.0 ** -44).sum() >= 180
    keep = gap > 2.0 ** -44
    compare(logits[keep.cuda()].contiguous(), scores[keep.cuda()].contiguous())


@DTYPES
@pytest.mark.parametrize("width", [1, 2, 16, 17, 64])
@pytest.mark.parametrize("V", [100, 5000, 9000])
def test_unequal_logits_of_equal_values(V, width, dtype):
    """Scores beside which 64 bits tell no logits apart: the lowest places, in texts whose other beam is finished too."""
    logits, scores = inputs(3, 2, V, dtype, seed=V)
    scores[:] = torch.finfo(torch.float32).min
    compare(logits, scores, width=width)
    scores[1, 0] = -1.0
    scores[2, 1] = -2.0
    fin = torch.zeros((3, 2), dtype=torch.bool, device="cuda")
    fin[1, 0] = fin[2, 1] = True
    compare(logits, scores, width=width, finished=fin, end=7)
    logits, scores = inputs(3, 2, V, dtype, seed=V)
    compare(logits * 2.0 ** -100, scores, width=width)               # (the same beside an ordinary score)
    logits[:, :, ::5] = -math.inf
    compare(logits * 2.0 ** -100, scores, width=width)


@pytest.mark.parametrize("width", [1, 5, 16, 17, 40, 64])
@pytest.mark.parametrize("V", [600, 9000, 30000])
def test_classes_of_equal_values(V, width):
    """Some candidates ahead, then many of one value with unequal logits in every part: steps of 2^31 of the values, the
    logits' classes 2^36 and 2^37 with digits from 2^14 to 2^20 behind."""
    g = torch.Generator().manual_seed(V + width)
    logits = torch.full((2, 3, V), 2.0 ** 36) + torch.randint(0, 64, (2, 3, V), generator=g) * 2.0 ** 14
    for b in range(2):
        for i in range(3):
            at = torch.randperm(V, generator=g)[:5]
            logits[b, i, at] = 2.0 ** 37 + torch.randint(0, 32, (5,), generator=g) * 2.0 ** 15
            logits[b, i, torch.rand(V, generator=g) < 0.3] = -(2.0 ** 36)
    scores = torch.full((2, 3), -(2.0 ** 83))
    scores[1, 1:] = -(2.0 ** 84)
    compare(logits.cuda(), scores.cuda(), width=width)


@DTYPES
def test_no_texts(dtype):
    # a batch of none goes through the step and the reordering alike
    got = isam.beam_step(torch.empty((0, 3, 50), device="cuda", dtype=dtype), torch.empty((0, 3), device="cuda"), width=4, end=2)
    assert [tuple(t.shape) for t in got] == [(0, 4)] * 4
    assert isam.beam_reorder(torch.empty((2, 0, 5), device="cuda", dtype=dtype), got[1], dim=1).shape == (2, 0, 5)
    out = torch.empty((0, 7), device="cuda", dtype=dtype)
    assert isam.beam_reorder(torch.empty((0, 7), device="cuda", dtype=dtype), got[1], out=out) is out
    with pytest.raises(ValueError):
        isam.beam_reorder(torch.empty((2, 6, 5), device="cuda", dtype=dtype), got[1], dim=1)
