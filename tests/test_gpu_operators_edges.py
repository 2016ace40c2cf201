"""Calls of the operators at which workspaces, pieces or types are at their limits; bounds as in test_gpu_operators.py."""
import os
import subprocess
import sys

import pytest

from test_gpu_operators import TINY, U, _close, _gen, _int4_weights, _xent_case, _xent_check

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def B():
    from paper_2507_20055_b200 import binding
    return binding


def _unaligned(t):
    """The same matrix in memory that starts one element behind a 16-byte boundary."""
    import torch
    flat = torch.empty(t.numel() + 1, dtype=t.dtype, device=t.device)
    view = flat[1:].view(t.shape)
    view.copy_(t)
    return view


@pytest.mark.parametrize("kind,rows,features,classes", [("bfloat16", 3500, 4096, 32768), ("float16", 3329, 2048, 32768), ("bfloat16", 300, 4096, 12000)])
def test_xent_copied_weights_in_pieces_of_narrow_tiles(B, kind, rows, features, classes):
    """Weights that TMA cannot read in place go through a copy of a few thousand classes, whose tiles leave more pairs than
    one tiling of all classes."""
    x, w, y, b = _xent_case(kind, rows, features, classes, True, 0.0, seed=17)
    op = B.LinearCrossEntropy(rows, features, classes, dtype=x.dtype)
    w = _unaligned(w)
    assert w.data_ptr() % 16 == 2
    _xent_check(B, op, x, w, y, b)
    # rows that do not count leave the number of slots as it is
    y[::3] = -100
    _xent_check(B, op, x, w, y, b)


@pytest.mark.parametrize("rows,features,classes,aligned", [(3072, 64, 44544, True), (546, 3600, 12750, False)])
def test_xent_last_piece_with_a_tile_behind_the_bias(B, rows, features, classes, aligned):
    x, w, y, b = _xent_case("bfloat16", rows, features, classes, True, 0.2, seed=23)
    _xent_check(B, B.LinearCrossEntropy(rows, features, classes, dtype=x.dtype), x, w if aligned else _unaligned(w), y, b)


def test_xent_in_several_pieces_under_the_checking_build():
    """Every plain store of the piecewise calls is looked up in the table of the buffers that they may write."""
    if os.environ.get("CERT_EXPECT_CHECKED") == "1":
        pytest.skip("already a run of the checking build")
    from paper_2507_20055_b200 import build
    env = dict(os.environ, CERT_LIB=build.build_checked(), CERT_EXPECT_CHECKED="1")
    run = subprocess.run([sys.executable, "-m", "pytest", os.path.join("tests", "test_gpu_operators.py"), os.path.join("tests", "test_gpu_operators_edges.py"),
                          "-q", "-x", "-m", "gpu", "-k", "xent_in_several_pieces or xent_copied_weights or xent_last_piece"], cwd=ROOT, env=env, capture_output=True,
                         text=True, timeout=900)
    assert run.returncode == 0, run.stdout[-3000:] + run.stderr[-2000:]
    assert " passed" in run.stdout


def test_int4_weights_are_laid_out_when_the_constructor_returns(B):
    """The product reads them ahead of the wait for the kernel in front of it, on whatever stream: nothing may be under way."""
    import torch
    codes = torch.randint(0, 256, (4096, 2048), device="cuda", dtype=torch.uint8)
    scales = torch.full((4096, 64), 0.01, dtype=torch.bfloat16, device="cuda")
    big = torch.randn(8192, 8192, device="cuda")
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for _ in range(20):
            big @ big                                      # some 300 ms in front of the layout
        op = B.Int4Weight(codes, scales, 4096, 64)
        assert side.query()
    x = torch.randn(1, 4096, device="cuda").to(torch.bfloat16)
    first = op.matvec(x)
    torch.cuda.synchronize()
    assert bool((op.matvec(x) == first).all()) and op.last_status() == 0


@pytest.mark.parametrize("kind", ["float16", "bfloat16"])
@pytest.mark.parametrize("group", [32, 64, 128, 256])
@pytest.mark.parametrize("zeros", [False, True])
def test_int4_inputs_of_one_sign(B, kind, group, zeros):
    """Inputs as a ReLU leaves them, and constant ones: what an accumulator loses goes one way.  It holds sums of weights times x
    and nothing larger: group / 16 products, truncated, then one addition per group, per warp and for the scale's power of two, all
    relative to the sum of the products' magnitudes; bfloat16 x is off by 2^-40 of the row's largest value at most."""
    import torch
    for m, n, k in ((1, 512, 4096), (4, 512, 8192), (13, 500, 4096), (16, 100, 1000)):
        codes, scales, zp, w = _int4_weights(kind, n, k, group, zeros, seed=group + m)
        op = B.Int4Weight(codes, scales, k, group, zeros=zp)
        for x in (torch.randn(m, k, generator=_gen(m), device="cuda").relu(), torch.full((m, k), 3.0, device="cuda")):
            x = x.to(scales.dtype)
            want, terms = x.double() @ w.t(), x.double() @ w.abs().t()
            bound = terms * ((group / 16 + 2) * 2.0 ** -23 + (scales.shape[1] + 20) * 2.0 ** -24)
            bound = bound + 2.0 ** -39 * x.double().amax(1, keepdim=True) * w.abs().sum(1)[None]
            _close(op.matvec(x), want, 1.01 * bound + 1.01 * U[kind] * want.abs() + TINY[kind], "y")
    assert op.last_status() == 0


@pytest.mark.parametrize("kind", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("zeros", [False, True])
def test_int4_quantize_hides_no_value_that_is_not_finite(B, kind, zeros):
    import torch
    w = (torch.randn(6, 200, generator=_gen(3), device="cuda") * 0.1).to(getattr(torch, kind))
    want = B.int4_quantize(w, 64, zeros)
    for bad in (float("nan"), float("inf"), -float("inf")):
        v = w.clone()
        v[1, 70], v[3, 199], v[5] = bad, bad, bad
        codes, scales, zp = B.int4_quantize(v, 64, zeros)
        hit = torch.zeros(6, 4, dtype=torch.bool, device="cuda")
        hit[1, 1] = hit[3, 3] = True
        hit[5] = True
        assert bool(torch.isnan(scales[hit]).all()) and bool((scales[~hit] == want[1][~hit]).all())
        back = B.Int4Weight(codes, scales, 200, 64, zeros=zp)
        assert bool((torch.isnan(back.dequantize()) == hit.repeat_interleave(64, 1)[:, :200]).all())
        kept = ~hit.repeat_interleave(64, 1)[:, :200:2]
        assert bool((codes[kept] == want[0][kept]).all())
        y = back.matvec(torch.ones(2, 200, device="cuda").to(w.dtype), relu=True)
        assert bool((torch.isnan(y) == hit.any(1)[None]).all())


@pytest.mark.parametrize("in_place", [True, False])
def test_clip_follows_the_gradients_of_parameters(B, in_place):
    """With torch's default zero_grad the gradients are new tensors every step: parameters stand for the ones of the day."""
    import math
    import torch
    torch.manual_seed(5)
    params = [torch.nn.Parameter(torch.randn(s, device="cuda")) for s in ((300, 70), (70,), (5000,))]
    params.append(torch.nn.Parameter(torch.randn(9, device="cuda").to(torch.bfloat16)))
    unused = torch.nn.Parameter(torch.randn(11, device="cuda"))
    plain = torch.randn(40, device="cuda")                 # a buffer among them stays what it is
    out = None if in_place else [torch.full_like(p.data, 7.0) for p in (*params, unused)] + [torch.empty_like(plain)]
    x, held, op = torch.randn(20, 300, device="cuda"), [], None
    for step in range(4):
        for p in params:
            p.grad = None
        held.append([torch.empty(1 << (8 + step), device="cuda")])            # so that addresses differ
        ((x @ params[0] + params[1]).square().sum() + (step + 1) * params[2].sum() + params[3].float().square().sum()).backward()
        held[-1] += [p.grad for p in params]
        if op is None:
            op = B.GradClipper([*params, unused, plain], out=out)
        before = [p.grad.double() for p in params] + [plain.double()]
        data = [p.detach().clone() for p in (*params, unused)]
        norm = float(op.clip(1.0))
        want = math.sqrt(sum(float((g ** 2).sum()) for g in before))
        assert abs(norm - want) <= 2.0 ** -19 * want
        got = [p.grad for p in params] + [plain] if in_place else [op.out[i] for i in (0, 1, 2, 3, 5)]
        for g, o in zip(before, got):
            kind = str(o.dtype).replace("torch.", "")
            _close(o, g / (want + 1e-6), (g / (want + 1e-6)).abs() * (U[kind] + 2.0 ** -18) + TINY[kind], kind)
        assert all(bool((a == b.detach()).all()) for a, b in zip(data, (*params, unused)))
        if out is not None:
            assert bool((out[4] == 7.0).all())
        assert op.check_guards() == 0 and op.last_status() == 0
    # kept buffers: the list stays
    handle = op._h
    for p in params:
        p.grad.mul_(3.0)
    op.clip(1.0)
    assert op._h is handle


@pytest.mark.parametrize("kind", ["float32", "bfloat16"])
def test_the_first_cuda_call_of_a_host_thread(B, kind):
    """A new thread has no context before its first launch, and the tensor maps of a call are made before that."""
    import threading
    import torch
    cases = [_xent_case(kind, rows, 256, 3000, True, 0.2, seed=rows) for rows in (500, 130)]
    op = B.LinearCrossEntropy(500, 256, 3000, dtype=cases[0][0].dtype)
    want = [[t.clone() for t in op.loss_and_grad(x, w, y, bias=b)] for x, w, y, b in cases]       # (and memory to hand out again)
    torch.cuda.synchronize()
    for (x, w, y, b), alone in zip(cases, want):
        got = []

        def call():
            try:
                got.extend(op.loss_and_grad(x, w, y, bias=b))
            except Exception as e:
                got.append(e)
        thread = threading.Thread(target=call)
        thread.start()
        thread.join()
        assert not isinstance(got[0], Exception), got[0]
        assert all(bool((g == r).all()) for g, r in zip(got, alone))


def test_host_threads_share_a_handle_on_one_stream(B):
    """Two threads call one object with different sizes: every result is the one of the call alone, to the bit."""
    import threading
    import torch
    cases = [_xent_case("bfloat16", rows, 256, 3000, True, 0.2, seed=rows) for rows in (500, 130)]
    op = B.LinearCrossEntropy(500, 256, 3000, dtype=torch.bfloat16)
    alone = [[t.clone() for t in op.loss_and_grad(x, w, y, bias=b)] for x, w, y, b in cases]
    grads = [torch.randn(n, generator=_gen(n), device="cuda") for n in (100000, 77, 3000)]
    clip = B.GradClipper(grads, out=[torch.empty_like(t) for t in grads])
    norm = float(clip.clip(1.0))
    torch.cuda.synchronize()
    wrong, stream = [], torch.cuda.current_stream()

    def calls(i):
        try:
            with torch.cuda.stream(stream):
                for _ in range(200):
                    x, w, y, b = cases[i]
                    got = op.loss_and_grad(x, w, y, bias=b)
                    if not all(bool((g == r).all()) for g, r in zip(got, alone[i])) or float(clip.clip(1.0)) != norm:
                        wrong.append(i)
        except Exception as e:
            wrong.append(e)
    threads = [threading.Thread(target=calls, args=(i,)) for i in (0, 1)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert wrong == [] and op.last_status() == 0 and op.check_guards() == 0 and clip.check_guards() == 0


def _rounded_dz(x, w, y):
    """float64 probabilities minus one at the target, rounded to the type as the gradient products get them (float16: times 2^14)."""
    import torch
    p = torch.softmax(x.double() @ w.double().t(), 1)
    p[torch.arange(len(y), device="cuda"), y] -= 1
    scale = 2.0 ** 14 if x.dtype == torch.float16 else 1.0
    return (p * scale).to(x.dtype).double() / scale


# accumulators of at most 4096 terms, 256 products of 16, each truncated by at most 2^-23 of what is there
LONG_SUMS = 256 * 2.0 ** -23


@pytest.mark.parametrize("kind", ["float16", "bfloat16"])
def test_xent_many_rows_of_one_sign(B, kind):
    """dW over 262144 rows of inputs behind a ReLU: truncation goes one way, so it must show in the mean error no more than
    accumulators of a bounded length let it (the roundings of the result are as often up as down)."""
    import torch
    rows, features, classes = 262144, 512, 8192
    x = torch.randn(rows, features, generator=_gen(1), device="cuda").relu().to(getattr(torch, kind))
    w = (torch.randn(classes, features, generator=_gen(2), device="cuda") / features ** 0.5).to(x.dtype)
    y = torch.randint(0, classes, (rows,), generator=_gen(3), device="cuda")
    op = B.LinearCrossEntropy(rows, features, classes, dtype=x.dtype)
    dw = op.loss_and_grad(x, w, y, reduction="sum")[2].double()
    assert op.last_status() == 0 and op.check_guards() == 0
    want, terms = torch.zeros_like(dw), torch.zeros_like(dw)
    for a in range(0, rows, 8192):
        dz, xs = _rounded_dz(x[a:a + 8192], w, y[a:a + 8192]), x[a:a + 8192].double()
        want += dz.t() @ xs
        terms += dz.abs().t() @ xs
    assert abs(float((dw - want).mean())) <= LONG_SUMS * float(terms.mean())


@pytest.mark.parametrize("kind,features", [("float16", 16384), ("bfloat16", 32768)])
def test_xent_many_features_of_one_sign(B, kind, features):
    """Inputs and weights that are all positive: the probabilities' logits are the losses', whose accumulators have 1024 terms."""
    import torch
    rows, classes = 512, 4096
    x = torch.randn(rows, features, generator=_gen(1), device="cuda").relu().to(getattr(torch, kind))
    w = (torch.rand(classes, features, generator=_gen(2), device="cuda") * (100.0 / features)).to(x.dtype)
    y = torch.randint(0, classes, (rows,), generator=_gen(3), device="cuda")
    op = B.LinearCrossEntropy(rows, features, classes, dtype=x.dtype)
    dx = op.loss_and_grad(x, w, y, reduction="sum")[1].double()
    assert op.last_status() == 0 and op.check_guards() == 0
    dz = _rounded_dz(x, w, y)
    logit = float((x.double() @ w.double().t()).max()) * (64 * 2.0 ** -23 + features / 1024 * 2.0 ** -24)
    bound = (2 * logit + LONG_SUMS) * float((dz.abs() @ w.double()).mean())
    assert abs(float((dx - dz @ w.double()).mean())) <= bound


@pytest.mark.parametrize("kind", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("classes", [10, 40, 200, 700])
def test_xent_every_class_masked_by_the_lowest_value(B, kind, classes):
    """The type's lowest value as a mask in every class swallows the logits: equal ones, so every class has the same probability,
    whichever path the number of classes takes.  -infinity beside it leaves the others equal."""
    import math
    import torch
    x, w, y, b = _xent_case(kind, 70, 64, classes, True, 0.0, seed=classes)
    if kind == "float16":                                  # (-65504 swallows no logit in float32)
        x = x * 0
    low = torch.full_like(b, torch.finfo(b.dtype).min)
    op = B.LinearCrossEntropy(70, 64, classes, dtype=x.dtype)
    for gone in (0, classes // 2):
        low[classes - gone:] = -float("inf")
        y = y % (classes - gone)
        loss, dx, dw, db = op.loss_and_grad(x, w, y, bias=low)
        # 2^x, the sum and the logarithm as in the other tests
        assert abs(float(loss) - math.log(classes - gone)) <= 2.0 ** -19 * (1 + math.log(classes))
        p = torch.zeros(70, classes, dtype=torch.float64, device="cuda")
        p[:, :classes - gone] = 1.0 / (classes - gone)
        p[torch.arange(70, device="cuda"), y] -= 1
        ep = p.abs() * (U[kind] + 2.0 ** -18) + (2.0 ** -38 if kind == "float16" else 0.0)
        want = p.sum(0) / 70
        _close(db, want, 1.01 * ep.sum(0) / 70 + 2 * U[kind] * want.abs() + 2.0 ** -20 * p.abs().sum(0) / 70 + TINY[kind], "db")
        want, terms = p.t() @ x.double() / 70, p.abs().t() @ x.double().abs() / 70
        _close(dw, want, 1.01 * ep.t() @ x.double().abs() / 70 + 2.0 ** -18 * terms + 2 * U[kind] * want.abs() + TINY[kind], "dw")
        want, terms = p @ w.double() / 70, p.abs() @ w.double().abs() / 70
        _close(dx, want, 1.01 * ep @ w.double().abs() / 70 + 2.0 ** -16 * terms + 2 * U[kind] * want.abs() + TINY[kind], "dx")
    assert op.last_status() == 0 and op.check_guards() == 0
