"""The residual junction where it is easily wrong: ties, values that are not finite, results in the place of inputs, the ends of
the range of magnitudes.  Statements, tolerances and random problems are those of test_gpu_residual.py."""
import numpy as np
import pytest
import torch

import paper_2302_06058_b200 as bm
import test_gpu_residual as R
from test_gpu_residual import TYPES, Problem

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("alpha", [1.7, 0.3, 1.0])
@pytest.mark.parametrize("stream", TYPES)
@pytest.mark.parametrize("T,C", [(24, 4096), (31, 96), (3, 16384)])
def test_the_scaled_stream_is_a_product_of_its_own(T, C, stream, alpha):
    """alpha x is rounded to fp32 before the branch is added.  A decimal alpha has an fp32 neighbour beside it; the rounding takes the
    neighbour's excess off again where alpha x has few bits, so that x' lies on a tie where alpha x + y does, and goes to the even side
    (in one fused step the excess decides every tie the same way)."""
    q = Problem(T, C, 0, 2, stream, scale=False, alpha=alpha)
    f = q.forward()
    want = (q.d["x"].float() * q.alpha + q.d["y"].float()).to(q.dt)
    assert torch.equal(f["xo"], want)
    q.check_forward(f)


@pytest.mark.parametrize("T,C", [(1, 8224), (2, 16384), (150, 12288), (230, 8224), (400, 16384)])
@pytest.mark.parametrize("stream", TYPES)
@pytest.mark.parametrize("post,pre,span", [(1, 1, 0), (2, 2, 1), (0, 2, 7), (1, 0, 0)])
def test_a_wait_of_a_cluster_that_runs_out(T, C, stream, post, pre, span):
    """A warp of every row gives up, at its first meeting or a later one; the others run out of time (a millisecond) one after the other.
    The call ends and reports it, every result is NaN or what it is otherwise, and the next call is as if nothing had been."""
    q = Problem(T, C, post, pre, stream, span=span, p=0.1)
    f = q.forward()
    g = q.backward(f)
    q.check_forward(f)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")

    def either(got, want, where):
        """Whether there are NaN in `got`, where it may not differ from `want` in another way."""
        lost = False
        for k in want:
            if k != "ws":
                nan = torch.isnan(got[k])
                assert bool((nan | (got[k] == want[k])).all()), (k, where)
                lost |= bool(nan.any())
        return lost

    def run(backward, *limits):
        """Results of a pass; with limits: of one with a wait that ends early, reported in `status`."""
        out = q.gradients() if backward else q.outputs()
        bufs = {**q.d, **out, "status_word": status}
        if backward:
            bufs.update({k: f[k] for k in ("xo", "stats_post", "stats_pre") if k in f})
        else:
            bufs.pop("dxo"), bufs.pop("dn")
        a = q.args({k: v for k, v in bufs.items() if backward or k[0] != "d"})
        status.zero_()
        if limits:
            bm.bimask_debug_residual_give_up(a, backward, *limits)
        else:
            (bm.bimask_residual_norm_bwd if backward else bm.bimask_residual_norm_fwd)(a)
        torch.cuda.synchronize()
        return out

    for backward, want in ((False, f), (True, g)):
        for limits in ((2000000, 0, 0), (2000000, 9, 0), (1000000, 4, 1), (1000000, 11, 2), (1000000, 0, 1)):
            lost = either(run(backward, *limits), want, limits)
            assert lost == (int(status.item()) == bm.binding.BIMASK_ETIMEOUT) and (lost or limits[2] > 0), limits
        for limits in ((0,), (200,), (1 << 31, -1, 3)):          # whoever is late by itself; nobody
            lost = either(run(backward, *limits), want, limits)
            assert int(status.item()) != 0 if lost else limits[0] <= 200 or int(status.item()) == 0, limits
            assert not (lost and limits[0] > 200), limits
        assert not either(run(backward), want, None) and int(status.item()) == 0


@pytest.mark.parametrize("T,C,spans", [(45, 288, (0, 1, 9, 45, 50)), (700, 384, (0, 1, 197)), (37, 1152, (0, 1, 5)), (6, 5120, (0, 1, 4)), (5, 16384, (0, 1, 2))])
@pytest.mark.parametrize("stream", TYPES)
def test_a_dropped_element_counts_as_zero_in_every_gradient(T, C, spans, stream):
    """Whatever a dropped element of y was, the gradients are bit for bit those with a zero in its place, as the results are."""
    for span in spans:
        for pre in (0, 1, 2):
            q = Problem(T, C, 0, pre, stream, span=span, p=0.3)
            dropped = torch.from_numpy(q.m == 0).cuda()
            zeros = q.d["y"].masked_fill(dropped, 0.0)
            odd = torch.tensor([float("inf"), float("nan"), -float("inf"), 3e38], device="cuda", dtype=torch.bfloat16).repeat(T * C // 4).view(T, C)
            seen = []
            for y in (zeros, torch.where(dropped, odd, zeros)):
                q.d["y"] = y
                f = q.forward()
                seen.append({**f, **q.backward(f)})
            for k in seen[0]:
                if k != "ws":
                    assert bool(torch.isfinite(seen[1][k]).all()) and torch.equal(seen[0][k], seen[1][k]), (k, span, pre)


@pytest.mark.parametrize("T,C,pitch", [(50, 320, None), (23, 160, 480), (700, 1152, None), (301, 4096, None), (5, 8192, 16384), (9, 16384, None)])
@pytest.mark.parametrize("stream", TYPES)
def test_the_gradient_of_a_gate_in_its_place(T, C, pitch, stream):
    for post, pre, span in ((1, 1, 1), (0, 2, 1), (2, 2, 1), (0, 1, 3), (1, 0, T)):
        q = Problem(T, C, post, pre, stream, span=span, p=0.1, pitch=pitch)
        f = q.forward()
        g = q.backward(f)
        q.check_backward(g, f)
        if pitch:
            q.d["gate"] = q.wide.clone()[:, :C]
        i = q.backward(f, dgate=q.d["gate"])
        assert all(torch.equal(i[k], g[k]) for k in g if k != "ws"), (post, pre, span)


def test_a_counter_lives_as_long_as_what_was_made_with_it():
    """A counter that nobody else holds, and tensors made after it that would take its place."""
    x = torch.ones(64, 64, device="cuda", dtype=torch.bfloat16)
    y, want = torch.empty_like(x), torch.empty_like(x)
    bm.bimask_dropout(x, bm.TYPE_BF16, 64, 64, bm.make_dropout(0.5, 3, 12), want)
    drop = bm.make_dropout(0.5, 3, 5, torch.full((1,), 7, dtype=torch.int64, device="cuda"))
    others = [torch.full((1,), 1000 + i, dtype=torch.int64, device="cuda") for i in range(8)]
    bm.bimask_dropout(x, bm.TYPE_BF16, 64, 64, drop, y)
    assert torch.equal(y, want)
    bufs = {"x": torch.zeros_like(x), "y": x, "xo": y}
    args = bm.make_residual_args(64, 64, bufs, drop=bm.make_dropout(0.5, 3, 5, torch.full((1,), 7, dtype=torch.int64, device="cuda")))
    others += [torch.full((1,), 2000 + i, dtype=torch.int64, device="cuda") for i in range(8)]
    bm.bimask_residual_norm_fwd(args)
    assert torch.equal(y, want) and len(others) == 16


@pytest.mark.parametrize("T,C", [(5, 32), (3, 384), (4, 4096), (3, 5120), (3, 16384)])
@pytest.mark.parametrize("stream", TYPES)
@pytest.mark.parametrize("size,eps", [(1e18, 1e-5), (2e-18, 0.0)])
def test_rows_at_the_ends_of_the_range(T, C, stream, size, eps, monkeypatch):
    """Rows of which every value is within a factor of two of the largest magnitude that the norms take, and of the smallest with eps 0."""
    monkeypatch.setattr(R, "EPS", (eps, eps))
    rng = np.random.default_rng(C)
    for post, pre in ((0, 1), (0, 2), (1, 1), (2, 2), (1, 0)):
        q = Problem(T, C, post, pre, stream, scale=False)
        for k, s in (("x", 0.7 if post == 0 else 1.0), ("y", 0.3 if post == 0 else 1.0)):
            v = torch.from_numpy(rng.uniform(0.5, 1.0, (T, C)) * rng.choice((-1.0, 1.0), (T, C)) * size * s)
            t = (v * 0.99).float().to(q.d[k].dtype)                        # 0.99: a rounding up stays in the range
            q.d[k], q.h[k] = t.cuda(), t.double().numpy()
        f = q.forward()
        q.check_forward(f)
        q.check_backward(q.backward(f), f)


def test_every_form_in_one_process_sets_its_limit_once():
    """Forward and backward passes in all forms that differ in their kernel: stream, gate, norms with and without means, one row or two
    per step, clusters.  Going through them again sets no shared-memory limit any more."""
    def every_form():
        for stream in TYPES:
            for T, C in ((9, 256), (9, 1152), (9, 2304), (5, 16384)):
                for span in (0, 1, 3):
                    for post, pre, bias in ((0, 1, False), (0, 2, True), (1, 1, False), (2, 2, True), (1, 1, True)):
                        q = Problem(T, C, post, pre, stream, span=span, bias=bias)
                        q.backward(q.forward())
    every_form()
    n = bm.bimask_debug_limits_set()
    assert n > 64
    every_form()
    assert bm.bimask_debug_limits_set() == n
