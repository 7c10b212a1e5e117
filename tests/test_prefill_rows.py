"""Rows that a scheduled batch hands to the norm and rotation: tensors that do not hold a chunk's rows are refused in front of the launch."""
import numpy as np
import pytest
import torch

from paper_2401_11181_amd import prefill, synth, tetri

HQ, HKV, D, C = 4, 2, 64, 64


class Recorder:
    def __init__(self, *a, **k):
        self.calls = []

    def tetri_qk_norm_rope(self, *args):
        self.calls.append(args)


@pytest.fixture
def session(monkeypatch):
    monkeypatch.setattr(tetri, "Tetri", Recorder)
    w = synth.small("rows", [70, 33], C, HQ, HKV, D, seed=6)
    s = prefill.ChunkedPrefill(w.prompt_lens, None, C, HQ, HKV, D, w.num_pages, synth.place_pages(w), device="cpu")
    assert [sum(n for _, _, n in s.chunk_segments(c)) for c in range(s.n_chunks)] == [64, 39]
    return s


def call(s, c, rows, out_rows=None, q=None, k=None, q_out=None, k_out=None):
    def zeros(n, width):
        return torch.zeros((n, width), dtype=torch.bfloat16)
    out_rows = rows if out_rows is None else out_rows
    s.qk_norm_rope(c, zeros(rows, HQ * D) if q is None else q, zeros(rows, HKV * D) if k is None else k, None, None, 1e-6, tetri.Rope(np.ones(8)),
                   zeros(out_rows, HQ * D).view(-1, HQ, D) if q_out is None else q_out, zeros(out_rows, HKV * D) if k_out is None else k_out)


def test_the_real_rows_are_enough(session):
    """Padding rows are neither read nor written: tensors need not have them."""
    call(session, 0, 64)
    call(session, 1, 64)
    call(session, 1, 39)
    rows = torch.zeros((39, (HQ + 2 * HKV) * D), dtype=torch.bfloat16)
    call(session, 1, 39, q=rows[:, :HQ * D], k=rows[:, HQ * D:(HQ + HKV) * D])
    call(session, 1, 39, q=rows, k=rows[:, HQ * D:])                 # (wider than they need be)
    assert [a[12] for a in session.handle.calls] == [C] * 5


@pytest.mark.parametrize("change", [
    dict(rows=38), dict(q=torch.zeros((38, HQ * D))), dict(k=torch.zeros((38, HKV * D))), dict(q=torch.zeros((64, HQ * D - 8))),
    dict(k=torch.zeros((64, HKV * D - 8))), dict(out_rows=38), dict(q_out=torch.zeros((38, HQ, D))), dict(k_out=torch.zeros((39, HKV * D - 1))),
    dict(q_out=torch.zeros((64, 2 * HQ * D))[:, ::2]), dict(k_out=torch.zeros((HKV * D, 64)).T)], ids=lambda c: "-".join(c))
def test_too_few_rows_are_refused(session, change):
    with pytest.raises(ValueError):
        call(session, 1, **{"rows": 39, **change})
    assert not session.handle.calls


@pytest.mark.parametrize("change", ["replaced", "written"])
def test_metadata_of_ones_own_may_have_a_whole_chunk_of_rows(session, change):
    if change == "replaced":
        cu, ctx, bt, S = session.meta[1]
        session.meta[1] = (cu.clone(), ctx, bt, S)
    else:
        session.meta[1][0][-1] = 64
    with pytest.raises(ValueError):
        call(session, 1, 39)
    call(session, 1, 64)
    assert len(session.handle.calls) == 1
