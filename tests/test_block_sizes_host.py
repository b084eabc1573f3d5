"""Workspaces of the calls beside the attention over the whole range of sizes that the shapes allow (no GPU, no call)."""
import pytest


@pytest.fixture(scope="module")
def L():
    from paper_2404_02882_amd import lasp
    return lasp


MOST = 2 ** 31 - 1


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [8, 64, 72, 4104])
def test_recurrence_scratch_grows_with_the_length(L, dtype, D):
    """Tiles of the same kind: from 16384 tokens on the scratch only grows, up to the longest sequence that is allowed."""
    lengths = [16384, 16385, 1 << 20, (1 << 20) + 1, 1 << 30] + [MOST - k for k in (4096, 1024, 512, 256, 128, 64, 2, 1, 0)]
    sizes = [L.rec_scratch_bytes(L.make_rec_shape(1, n, D, dtype)) for n in lengths]
    assert all(a <= b for a, b in zip(sizes, sizes[1:])), list(zip(lengths, sizes))
    # 12 bytes a channel and tile, of 1024 tokens at most
    assert sizes[-1] >= MOST // 1024 * D * 12


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,C", [(MOST, 8), (MOST, 2048), (1, 16384), (MOST, 16384)])
def test_norm_scratch_stays_small(L, dtype, rows, C):
    """One partial row of C floats for every workgroup and sum, of at most ten workgroups a CU."""
    assert 0 < L.addnorm_scratch_bytes(L.make_rows(rows, C, dtype)) <= 2 * 4 * 256 * 10 * C
    assert 0 < L.gatenorm_scratch_bytes(L.make_gate_shape(1, 1, rows, C, dtype)) <= 4 * 256 * 10 * C


def test_recurrence_sequence_refuses_short_lists_first():
    """Before any of its calls: the first would refuse these tensors for lying on the host."""
    import torch
    from paper_2404_02882_amd import sequence
    seq = sequence.RecurrenceSequence(1, 16, 8, torch.float32, T=2, device="cpu")
    full, short = [torch.zeros(1, 8, 8)] * 2, [torch.zeros(1, 8, 8)]
    for i in range(3):
        args = [full] * 3
        args[i] = short
        with pytest.raises(ValueError, match="1 tensors for 2 sub-sequences"):
            seq.forward(*args)
    with pytest.raises(ValueError, match="lens: 1 tensors"):
        seq.forward(full, full, full, lens=[torch.zeros(1, dtype=torch.int32)])
    for i in range(1, 6):       # (x is not read)
        args = [None] + [full] * 5
        args[i] = short
        with pytest.raises(ValueError, match="1 tensors for 2 sub-sequences"):
            seq.backward(*args)
    with pytest.raises(ValueError, match="GPU"):
        seq.forward(full, full, full)
