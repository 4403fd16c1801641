"""A captured pass over one token of each sequence goes on when a sequence takes a new page: the batch's tensors keep their shapes."""
import pytest
import torch

from paper_2506_17870_b200.attention import PageTable


def test_shapes_stay_past_the_end_of_a_page():
    t = PageTable(20, 16, device="cpu", positions=100)
    a, b = t.add(), t.add()
    t.extend([a, b], [15, 30])
    shapes = None
    for n in range(70):
        x = t.extend([a, b], [1, 1])
        now = [v.shape for v in x if isinstance(v, torch.Tensor)]
        shapes = shapes or now
        assert now == shapes and x.table.shape == (2, 7)
        for i, length in enumerate((16 + n, 31 + n)):
            held = -(-length // 16)
            assert bool((x.table[i, :held] >= 0).all()) and bool((x.table[i, held:] == -1).all())
            assert x.slots[i] == x.table[i, (length - 1) // 16] * 16 + (length - 1) % 16
    assert PageTable(3, 16, device="cpu", positions=1000).columns == 3                # no more than there are pages
    assert PageTable(0, 16, device="cpu", positions=0).columns == 1


@pytest.mark.gpu
@pytest.mark.parametrize("kind", [torch.bfloat16, torch.float8_e4m3fn, torch.int8])
def test_a_graph_follows_sequences_into_new_pages(kind):
    from test_gpu_attention_block import make
    stack, table = make(kind=kind)
    x = torch.randn(2, 120, 256, device="cuda", dtype=torch.bfloat16)
    ids = [table.add(), table.add()]
    stack.serve(x[:, :14].reshape(-1, 256), table.extend(ids, [14, 14]))
    batch, stream = table.extend(ids, [1, 1]), x[:, 14].clone()
    stack.serve(stream, batch)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = stack.serve(stream, batch)
    for t in range(15, 85):                                                           # over the ends of five pages
        new = table.extend(ids, [1, 1])
        stream.copy_(x[:, t])
        for old, now in zip((batch.positions, batch.slots, batch.lengths, batch.table), (new.positions, new.slots, new.lengths, new.table)):
            old.copy_(now)
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        assert torch.equal(got, stack.serve(stream, new))
