"""dk_seq_reorder: what every slot holds afterwards, to the bit, and that slots grow apart."""
import numpy as np
import pytest
import torch

import oracle
from gpu_util import Mirror, to_dev
from test_gpu_shared import bounds
from paper_2605_26289_amd import binding as dk
from paper_2605_26289_amd import workloads as wl

pytestmark = pytest.mark.gpu

SHAPES = [(8, 2, 128, "bf16"), (8, 2, 64, "bf16"), (7, 1, 64, "f32"), (3, 3, 128, "f32")]


class Beams(Mirror):
    def __init__(self, shape, n, prompt, granule=16, seed=0, cells=40000):
        super().__init__(wl.Shape(*shape), n + 1, cells, granule, seed)
        self.prompt = self.acquire()
        if prompt:
            self.append([self.prompt], [prompt])
        self.slots = [self.acquire() for _ in range(n)]
        for s in self.slots:
            if prompt:
                self.alias(self.prompt, s, prompt)

    def reorder(self, parents, slots=None):
        self.pool.reorder(self.slots if slots is None else slots, parents)
        self.model.reorder(self.slots if slots is None else slots, parents)

    def check(self):
        for s in [self.prompt] + self.slots:
            if self.pool.length(s):
                self.check_gather(s)
            assert self.pool.length(s) == len(self.model.seqs[s])


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("granule", [16, 5, 256])
def test_a_beam_search(shape, granule):
    b = Beams(shape, 5, 37, granule)
    rng = np.random.default_rng(1)
    b.reorder([0, 0, 0, 0, 0])
    for step in range(40):
        b.append(b.slots, [1] * 5)
        b.reorder(rng.integers(0, 5, size=5).tolist())
        if step % 8 == 0:
            b.check()
    b.check()
    for s in b.slots:  # short chains, few runs of cells
        runs, depth = dk.seq_stats(b.pool.handle, s)
        assert runs <= 4 + 40 // granule and depth <= 4 + 40 // granule
    for s in [b.prompt] + b.slots:
        b.pool.release(s)
    assert dk.pool_stats(b.pool.handle)[0] == 0


@pytest.mark.parametrize("parents", [[0, 1, 2, 3], [3, 2, 1, 0], [1, 1, 1, 1], [1, 2, 3, 0], [2, 2, 0, 0]])
def test_maps_of_parents(parents):
    b = Beams(SHAPES[0], 4, 0)
    b.append(b.slots, [21, 3, 48, 0])
    b.reorder(parents)
    b.check()
    b.append(b.slots, [2, 1, 3, 40])  # they grow apart
    b.check()
    b.reorder(parents[:2] if max(parents[:2]) < 2 else [1, 0], b.slots[:2])  # some of them
    b.check()


def test_many_copies_in_one_call():
    """More than the arguments of one launch hold."""
    b = Beams((2, 1, 64, "bf16"), 400, 0, granule=16, cells=16 * 1000)
    b.append(b.slots[:1], [23])
    b.reorder([0] * 400)
    for s in b.slots[:3] + b.slots[-3:]:
        b.check_gather(s)
    b.append(b.slots, [1] * 400)
    b.check()


def test_no_cells_leaves_all_as_it_was():
    b = Beams(SHAPES[0], 4, 0, granule=16, cells=16 * 5)
    b.append(b.slots, [17, 9, 0, 0])  # three of five granules
    with pytest.raises(dk.DeltaKVError) as e:
        b.pool.reorder(b.slots, [0, 0, 0, 0])
    assert e.value.name == "NO_CELLS"
    b.check()
    b.reorder([0, 0, 0, 1])
    b.check()


def test_a_beam_step_of_all_operators():
    """Selection, reordering, append and attention as a search would use them, against the oracle, for some steps."""
    shape = (8, 2, 128, "bf16")
    beams, requests, vocab, prompt = 4, 2, 1504, 300
    b = Beams(shape, beams * requests, 0, granule=32, seed=3)
    rng = np.random.default_rng(4)
    for r in range(requests):
        s = b.slots[r * beams]
        b.append([s], [prompt + 40 * r])
        for t in b.slots[r * beams + 1:(r + 1) * beams]:
            b.alias(s, t, prompt + 40 * r)
    scores = np.full(beams * requests, -np.inf, dtype=np.float32)
    scores[::beams] = 0.0
    cu_rows = torch.tensor([0, beams, 2 * beams], dtype=torch.int32, device="cuda")
    out = [torch.empty((requests, beams), dtype=t, device="cuda") for t in (torch.int32, torch.int32, torch.float32)]
    ws = torch.empty(dk.beam_workspace_bytes(beams * requests, vocab, dk.BF16, beams), dtype=torch.uint8, device="cuda")
    cu = np.arange(beams * requests + 1, dtype=np.int32)
    for step in range(6):
        logits = wl.normal(rng, (beams * requests, vocab), "bf16")
        dk.beam_select(requests, beams * requests, cu_rows, to_dev(logits, "bf16"), dk.BF16, vocab, vocab, torch.from_numpy(scores).cuda(), beams,
                       *out, ws)
        want = oracle.beam_select(logits, scores, [0, beams, 2 * beams], beams)
        rows = out[0].cpu().numpy()
        assert np.array_equal(rows, want[0]) and np.array_equal(out[1].cpu().numpy(), want[1])
        scores = out[2].cpu().numpy().reshape(-1)
        b.reorder(rows.reshape(-1).tolist())
        b.append(b.slots, [1] * len(b.slots))
        q = wl.normal(rng, (len(b.slots), 8, 128), "bf16")
        lse = torch.empty((len(b.slots), 8), dtype=torch.float32, device="cuda")
        got = b.pool.shared_attend(b.slots, cu, to_dev(q, "bf16"), b.shape.scale, lse=lse)
        torch.cuda.synchronize()
        for i, s in enumerate(b.slots):
            k, v = b.cache(s)
            ref = oracle.scored_attend(q[i:i + 1], k, v, len(k) - 1, b.shape.scale)
            tol, ltol = bounds(ref, "bf16", len(k), 128)
            assert (np.abs(got[i:i + 1].float().cpu().numpy() - ref[0]) <= tol).all()
            assert (np.abs(lse[i:i + 1].cpu().numpy() - ref[1]) <= ltol).all()
