"""Rows that are one: torch leaves the stride of a dimension of one element open, the library wants a row's length at least."""
import pytest
import torch


def views(heads, hd, dtype=torch.float32):
    """[1, heads, head_dim], heads back to back, with strides of the first dimension that are less than a row, more, and odd."""
    flat = torch.arange(4 * heads * hd).to(dtype)
    return [flat[:heads * hd].view(heads, 1, hd).transpose(0, 1), flat.as_strided((1, heads, hd), (1, hd, 1)), flat.as_strided((1, heads, hd), (0, hd, 1)),
            flat.as_strided((1, heads, hd), (3 * heads * hd + 2, hd, 1)), flat[:heads * hd].view(1, heads, hd)]


@pytest.mark.parametrize("heads,hd", [(4, 32), (1, 64), (28, 128)])
def test_the_stride_of_a_single_row_is_its_length(heads, hd):
    import paper_2507_17307_amd as P
    for t in views(heads, hd):
        assert P.binding._rows("x", t, -1) == (t.data_ptr(), heads * hd), t.stride()
        k, v = torch.zeros(1, heads, 16, hd, dtype=torch.bfloat16), torch.zeros(1, heads, hd, 16, dtype=torch.bfloat16)
        c = P.PagedCache(k, v, torch.zeros(1, 1, dtype=torch.int32))
        assert P.binding._paged_rows("q", t, c, 1, heads, torch.float32) == (t.data_ptr(), heads * hd), t.stride()


def test_the_stride_of_a_single_head_is_open_too():
    import paper_2507_17307_amd as P
    flat = torch.arange(1024.0)
    k, v = torch.zeros(1, 1, 16, 32, dtype=torch.bfloat16), torch.zeros(1, 1, 32, 16, dtype=torch.bfloat16)
    c = P.PagedCache(k, v, torch.zeros(1, 1, dtype=torch.int32))
    for head_stride in (0, 1, 32, 100):
        t = flat.as_strided((3, 1, 32), (64, head_stride, 1))
        assert P.binding._rows("x", t, -1) == (t.data_ptr(), 64)
        assert P.binding._paged_rows("k", t, c, 3, 1, torch.float32) == (t.data_ptr(), 64)
    with pytest.raises(ValueError):
        P.binding._rows("x", flat.as_strided((3, 2, 32), (128, 64, 1)), -1)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_decode_step_of_transposed_views(dtype):
    """One token: q, k, v and the outputs as [heads, 1, head_dim] tensors seen as rows, against the same as rows."""
    import paper_2507_17307_amd as P
    g = torch.Generator().manual_seed(73)
    nq, nkv, hd = 8, 2, 64
    got = []
    x = torch.randn(nq + 2 * nkv, 1, hd, generator=g).to(dtype).cuda()
    table, one = torch.tensor([[1, 0]], dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    pos = torch.full((1,), 17, dtype=torch.int32, device="cuda")
    pages = torch.randn(2, 2, nkv, 16, hd, generator=g).to(torch.bfloat16).cuda()
    f, _ = P.rs_rope_frequencies(hd, 1e4)
    r = P.Rope(f.cuda())
    for turned in (True, False):
        k, v = pages[0].clone(), pages[1].clone().view(2, nkv, hd, 16)
        c = P.PagedCache(k, v, table)

        def rows(t):
            return t.transpose(0, 1) if turned else t.transpose(0, 1).reshape(1, -1).view(1, -1, hd)
        turn, q, out = (torch.empty(nq, 1, hd, dtype=dtype, device="cuda") for _ in range(3))
        turn, q, out = (rows(t) for t in (turn, q, out))
        P.rs_rope_rows(r, pos, rows(x[:nq]), turn)
        P.rs_paged_append(c, 1, 1, one, None, pos, r, rows(x[:nq]), rows(x[nq:nq + nkv]), rows(x[nq + nkv:]), q)
        scratch = torch.empty(P.rs_paged_attention_scratch_bytes(c, 1, 1, nq), dtype=torch.uint8, device="cuda")
        P.rs_paged_attention(c, 1, 1, one, None, pos, q, 0.125, 0, out, None, scratch)
        torch.cuda.synchronize()
        got.append((turn.clone(), q.clone(), out.clone(), k, v))
    assert all(torch.equal(a, b) for a, b in zip(*got))
