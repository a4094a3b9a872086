"""Buffers of the runners across batches that grow, without a GPU: what a recorded
step was recorded with lives on; without a recording, outgrown buffers are freed."""

import gc
import weakref

import pytest

G = pytest.importorskip("paper_2102_10424_amd.gist",
                        reason="libgist.so not built (python -m paper_2102_10424_amd.build)")


class Batch:
    """The sizes of a mini-batch: all that allocating for it asks."""

    def __init__(self, n, nnz):
        self.n, self.nnz = n, nnz

    def rows(self, l):
        return self.n


class Ctx:
    def __init__(self, captures):
        self.captures = captures


def held(run):
    """Every tensor a step of the runner works on."""
    ts = [run.ws, run.loss_ws, run.dlogits] + run.dH + run.agg + [h for h in run.H if h is not None]
    return [weakref.ref(t) for t in ts + (run.alpha or [])]


@pytest.mark.parametrize("kind", ["gcn", "sage", "gat"])
def test_buffers_of_a_recorded_step_live_on(kind):
    from paper_2102_10424_amd import step as S
    run = S.SubGCN(Ctx(1), kind, [8, 24, 5], 16, device="cpu", input_grad=True)
    run.prepare(Batch(16, 60))
    refs = held(run)
    for n in (17, 18, 19, 200, 201, 5000):
        run.prepare(Batch(n, 5 * n))
        refs += held(run)
    gc.collect()
    assert all(r() is not None for r in refs)
    assert run.n_cap >= 5000 and run.dH[0].shape == (run.n_cap, 8)
    # capacities at least double: what is kept adds up to less than what is in use
    for name in ("H", "agg"):
        caps = sorted({k[("H", "agg").index(name)][1].shape[0] for k in run._kept if len(k) == 5})
        assert sum(caps) < run.n_cap


@pytest.mark.parametrize("kind", ["gcn", "gat"])
def test_buffers_are_freed_without_a_recording(kind):
    from paper_2102_10424_amd import step as S
    run = S.SubGCN(Ctx(0), kind, [8, 24, 5], 16, device="cpu")
    run.prepare(Batch(16, 60))
    refs = held(run)
    run.prepare(Batch(3000, 20000))
    gc.collect()
    assert run.n_cap == 3000 and run.dlogits.shape == (3000, 5)
    assert not any(r() is not None for r in refs)


def test_workspace_of_a_recorded_batched_step_lives_on():
    from paper_2102_10424_amd import step as S
    run = S.SubGCNBatch(Ctx(1), "gcn", [8, 24, 5], 2, 6000, device="cpu")
    sizes = [run._workspace(n).numel() for n in (10,)]
    ws = weakref.ref(run.ws)
    for n in (500, 6000):
        sizes.append(run._workspace(n).numel())
    gc.collect()
    assert sizes == sorted(sizes) and ws() is not None


def test_log_probs_buffers_double():
    """Batches that grow one row at a time: few sets of buffers are kept, of fewer rows
    together than the one in use."""
    from paper_2102_10424_amd import step as S
    run = S.SubGCN(Ctx(1), "gcn", [8, 24, 5], 16, device="cpu")
    for n in range(1, 600):
        p = run._log_probs_buffers(n, 3)
        assert p["n"] >= n and p["logp"].shape[0] == p["n"] and p["top_idx"].shape == (p["n"], 3)
    kept = [k["n"] for k in run._kept if k is not None]
    assert sum(kept) < p["n"] and len(kept) <= 6
