"""Calls beside the sparse decode at the limits of what their arguments may be."""
import pytest
import torch

from tests.test_gpu_attention import DEV, _randn

pytestmark = pytest.mark.gpu


def test_evict_between_neighbours_in_one_piece_of_memory():
    """Inputs and outputs that touch, in one buffer, in every order: no byte is in common."""
    import paper_2502_12216_amd as T
    hkv, n, m = 2, 200, 50
    src = T.RaggedBatch([n], hkv, hkv)
    keep = torch.tensor([m], dtype=torch.int32, device=DEV)
    K, V = _randn(1, hkv, n, 128), _randn(2, hkv, n, 128)
    weights, positions = torch.rand(hkv, n, device=DEV), torch.arange(n, dtype=torch.int32, device=DEV).repeat(hkv, 1) + 7
    inputs, results = [K, V, weights, positions], []
    shapes = [((hkv, m, 128), torch.bfloat16)] * 2 + [((hkv, m), torch.float32), ((hkv, m), torch.int32)]
    for turn in range(3):
        if turn == 0:
            arrays = inputs + [torch.zeros(s, dtype=d, device=DEV) for s, d in shapes]
        else:
            sizes = [x.numel() * x.element_size() for x in inputs] + [torch.Size(s).numel() * d.itemsize for s, d in shapes]
            order = list(range(8)) if turn == 1 else [4, 0, 5, 1, 6, 2, 7, 3]
            buf, at, arrays = torch.zeros(sum(sizes), dtype=torch.uint8, device=DEV), 0, [None] * 8
            for i in order:
                piece = buf[at:at + sizes[i]]
                arrays[i] = (piece.view(inputs[i].dtype).view(inputs[i].shape) if i < 4 else
                             piece.view(shapes[i - 4][1]).view(shapes[i - 4][0]))
                at += sizes[i]
            for x, y in zip(arrays, inputs):
                x.copy_(y)
        k, v, w, p, ko, vo, wo, po = arrays
        T.CacheEvictor(src, T.RaggedBatch([0], hkv, hkv, capacities=[m]), 10)(
            k, v, w, keep, ko, vo, wo, po, positions=p, newest=torch.tensor([n + 6], dtype=torch.int32, device=DEV))
        torch.cuda.synchronize()
        results.append([x.clone() for x in arrays])
    for other in results[1:]:
        for x, y in zip(results[0], other):
            assert torch.equal(x, y)


def test_evict_of_nothing_into_nothing():
    """Empty sequences into spans without rows: only the lengths are written."""
    import paper_2502_12216_amd as T
    src, dest = T.RaggedBatch([0, 0], 4, 2), T.RaggedBatch([0, 0], 4, 2, capacities=[0, 0])
    dest.seq_len.fill_(9)
    rows = torch.zeros(2, 0, 128, dtype=torch.bfloat16, device=DEV)
    sums, pos = torch.zeros(2, 0, device=DEV), torch.zeros(2, 0, dtype=torch.int32, device=DEV)
    T.CacheEvictor(src, dest, 3)(rows, rows, sums, torch.tensor([4, 0], dtype=torch.int32, device=DEV), rows, rows, sums, pos)
    torch.cuda.synchronize()
    assert dest.seq_len.tolist() == [0, 0]


def test_append_off_its_alignment_leaves_the_cache():
    import paper_2502_12216_amd as T
    c = T.EvictingCache(8, 2, 1, 16, recent=4)
    k = _randn(1, 1, 2, 128)
    c.append(k, k)
    state = [x.clone() for x in (c.K, c.V, c.weights, c.positions, c.newest, c.batch.seq_len)]
    off = torch.zeros(2 * 128 + 1, dtype=torch.bfloat16, device=DEV)[1:].view(1, 2, 128)
    for bad in ((off, k), (k, off)):
        with pytest.raises(T.TacticError, match="16-byte"):
            c.append(*bad)
    torch.cuda.synchronize()
    for x, y in zip((c.K, c.V, c.weights, c.positions, c.newest, c.batch.seq_len), state):
        assert torch.equal(x, y)
    assert c.batch.seq_lens == [1]


def test_sparse_decoder_takes_a_workspace_of_one_piece_only():
    import paper_2502_12216_amd as T
    batch = T.RaggedBatch([900, 300], 8, 2)
    size = T.SparseDecoder(batch, [20, 10]).workspace.numel()
    whole = torch.zeros(2 * size, dtype=torch.uint8, device=DEV)
    assert T.SparseDecoder(batch, [20, 10], workspace=whole).workspace is whole
    for bad in (torch.zeros(1, dtype=torch.uint8, device=DEV).expand(size), whole[::2], whole[:size - 1]):
        got = T.SparseDecoder(batch, [20, 10], workspace=bad).workspace
        assert got is not bad and got.is_contiguous() and got.numel() == size


@pytest.mark.parametrize("lens", [[0, 50, 1], [0, 0, 70]])
def test_evicting_cache_of_empty_prompts(lens):
    """Sequences that start from nothing beside others, through prompt, eviction, insertion and decode."""
    import paper_2502_12216_amd as T
    from tests import attention_ref as R
    from tests.test_gpu_evict import _loop
    _loop(T.EvictingCache(8, 2, 3, 8, recent=3, cap=30.0, slopes=R.slopes(8)), lens, 8, 2, 12)
