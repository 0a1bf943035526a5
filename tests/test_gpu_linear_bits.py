"""Results are the same bits wherever sizes, types, pitch, alignment, working memory and offsets are: with operands at other addresses, other garbage in
the working memory, on another stream."""
import ctypes as C

import pytest
import torch

from paper_2501_10054_amd import tardis as T

pytestmark = pytest.mark.gpu
DEV = "cuda"
ALIGN = 16


def elsewhere(t, pitch=None):
    """The same values at another address of the same remainder by 16, behind and before NaNs, rows `pitch` apart."""
    n, k = t.reshape(-1, t.shape[-1]).shape
    pitch = pitch or k
    size = t.element_size()
    store = torch.full((n * pitch * size + 4096,), 255, dtype=torch.uint8, device=DEV)
    lead = (t.data_ptr() - store.data_ptr()) % ALIGN + 1024
    out = store[lead:lead + n * pitch * size].view(t.dtype).view(n, pitch)[:, :k]
    out.copy_(t.reshape(n, k))
    assert (out.data_ptr() - t.data_ptr()) % ALIGN == 0 and out.data_ptr() != t.data_ptr()
    return out if pitch != k else out.view(t.shape)


# (ranges of K that are joined, aligned copies, staged rows, large tiles, short rows)
@pytest.mark.parametrize("n,n_in,n_out,gap", [(8, 16384, 256, 0), (333, 11008, 1024, 0), (600, 1001, 2048, 0), (40, 129, 96, 3), (2048, 512, 4096, 8), (600, 64, 1000, 0)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("memory", ["all", "none"])
def test_linear(n, n_in, n_out, gap, dtype, memory):
    gen = torch.Generator(device=DEV).manual_seed(n)
    x = torch.randn(n, n_in + gap, device=DEV, generator=gen).to(dtype)[:, :n_in]
    W, r = torch.randn(n_out, n_in, device=DEV, generator=gen).to(dtype), torch.randn(n, n_out, device=DEV, generator=gen)
    code = T.F32 if dtype == torch.float32 else T.BF16

    def call(x, W, stream):
        y, need = torch.empty(n, n_out, device=DEV), C.c_int64()
        desc = T.tardis_linear_desc(n_in, n_out, code, T.F32, T.ACT["gelu_tanh"], 0, W.data_ptr(), None)
        assert T.lib().tardis_linear_workspace(desc, x.data_ptr(), n, x.stride(0), need) == T.OK
        size = need.value if memory == "all" else 0
        work = torch.full((max(size, 1),), 255, dtype=torch.uint8, device=DEV)
        torch.cuda.synchronize()
        assert T.lib().tardis_linear(desc, x.data_ptr(), n, x.stride(0), r.data_ptr(), y.data_ptr(), work.data_ptr() if size else None, size, stream.cuda_stream) == T.OK
        torch.cuda.synchronize()
        return y

    want = call(x, W, torch.cuda.current_stream())
    assert torch.isfinite(want).all()
    for stream in (torch.cuda.current_stream(), torch.cuda.Stream()):
        assert torch.equal(call(elsewhere(x, n_in + gap), elsewhere(W), stream), want)


@pytest.mark.parametrize("n_in", [512, 511])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_groups(n_in, dtype):
    gen = torch.Generator(device=DEV).manual_seed(n_in)
    for rows, n_out, experts in ((64, 192, 8), (3000, 2048, 5), (400, 96, 130)):
        x = torch.randn(rows, n_in, device=DEV, generator=gen).to(dtype)
        W = torch.randn(experts, n_out, n_in, device=DEV, generator=gen).to(dtype)
        cuts = torch.randint(0, rows + 1, (experts - 1,), device=DEV, generator=gen).sort().values
        offsets = torch.cat([cuts.new_zeros(1), cuts, cuts.new_full((1,), rows)]).int()
        order = torch.randperm(rows, device=DEV, generator=gen).int()
        want = T.tardis_grouped_linear(x, W, offsets, order=order)
        assert torch.equal(T.tardis_grouped_linear(elsewhere(x), elsewhere(W), offsets.clone(), order=order.clone()), want)
