"""Extents at the edges of what the training-step operators take: on the CPU what
is refused or only described, on the GPU what runs."""

import pytest

torch = pytest.importorskip("torch")

from tests.test_training_refusals import BASE, UNSUPPORTED, L, mat, ref  # noqa: F401


def test_more_channels_than_the_norm_counts(L):  # noqa: F811
    """(No memory is behind these matrices: what passes the checks of extents is
    refused for its addresses, or for want of a device.)"""
    lib = L.load_library()

    def both(cols):
        x, w = mat(L, rows=1, cols=cols), L.LmTensor(BASE, 1, cols, 0)
        return (lib.lm_rmsnorm(ref(x), None, None, 1e-6, None, ref(x), None, None, None),
                lib.lm_rmsnorm_grad(ref(x), ref(x), None, BASE, None, None, ref(x), ref(w), BASE, 1 << 40, None))

    for cols in (0x7FFFFF00, 0x7FFFFC01, (1 << 31) - 65535):
        assert both(cols) == (UNSUPPORTED, UNSUPPORTED)
    assert UNSUPPORTED not in both((1 << 31) - 65536)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,cols", [(torch.float32, (1 << 29) + 37), (torch.bfloat16, (1 << 30) + 37)])
def test_rows_of_more_than_2_31_bytes_off_16_byte_boundaries(dtype, cols):
    """The middle row of three, whose first element is on no such boundary, has
    the codes of the same row by itself, which is; and reads back the same."""
    from paper_2605_19811_gb300 import training as T
    some = torch.randn((1 << 20) + 7, device="cuda").to(dtype)
    x = some.repeat(-(-3 * cols // some.numel()))[:3 * cols].view(3, cols)
    assert x[1].data_ptr() % 16 != 0
    all_three, alone = T.checkpoint8(x, "i8"), T.checkpoint8(x[1].clone(), "i8")
    assert torch.equal(all_three.scales[:, 1], alone.scales[:, 0])
    assert torch.equal(all_three.codes[1, :cols], alone.codes[0, :cols])
    x.zero_()
    all_three.unpack(out=x)
    assert torch.equal(x[1], alone.unpack(dtype)[0])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows", [1, 5, 70001])
def test_norm_of_no_channels(rows, dtype):
    """A sum over nothing is zero: rstd = 1 / sqrt(eps)."""
    from paper_2605_19811_gb300 import training as T
    torch.full((rows,), 7.0, device="cuda")                # what a new rstd would be found to hold
    x = torch.empty(rows, 0, device="cuda", dtype=dtype)
    o = T.rmsnorm(x, torch.empty(0, device="cuda", dtype=dtype), residual=x, eps=1e-4, checkpoint="i8")
    assert o.y.shape == o.h.shape == (rows, 0) and o.rstd.shape == (rows,) and o.checkpoint.rows == rows
    assert float((o.rstd - 100.0).abs().max()) <= 100.0 * 2.0 ** -22
    dx, dw = T.rmsnorm_grad(x, x, o.rstd, torch.empty(0, device="cuda", dtype=dtype))
    assert dx.shape == (rows, 0) and dw.shape == (0,)


def test_empty_tensors_fold():
    from paper_2605_19811_gb300 import training as T
    for shape, want in (((2, 3, 0), (6, 0)), ((0, 3, 8), (0, 8)), ((2, 0, 8), (0, 8)), ((0, 3, 0), (0, 0)), ((0,), (1, 0))):
        m = T._matrix(torch.zeros(shape), "x")
        assert (m.rows, m.cols) == want
    m = T._matrix(torch.zeros(2, 3, 16)[:, :, :8], "x")
    assert (m.rows, m.cols, m.ld) == (6, 8, 16)
    m = T._matrix(torch.zeros(2, 0, 16)[:, :, :8], "x")
    assert (m.rows, m.cols) == (0, 8)


@pytest.mark.gpu
def test_norm_of_no_channels_over_two_leading_dimensions():
    from paper_2605_19811_gb300 import training as T
    o = T.rmsnorm(torch.empty(2, 3, 0, device="cuda"), eps=1.0)
    assert o.y.shape == (2, 3, 0) and bool((o.rstd == torch.ones(2, 3, device="cuda")).all())


def test_one_row_of_a_wider_checkpoint():
    """A view of one row has the pitch of its buffer, as a view of several has."""
    from paper_2605_19811_gb300 import training as T
    codes, scales = torch.zeros(4, 64, dtype=torch.uint8), torch.zeros(1, 4)
    for rows in (1, 2, 4):
        d = T.Checkpoint8(codes[:rows, :20], scales, 20, "i8").desc()
        assert (d.rows, d.cols, d.ld_codes) == (rows, 20, 64)
    assert T.Checkpoint8(torch.zeros(64, dtype=torch.uint8)[None], scales, 20, "i8").desc().ld_codes == 64
    assert T.Checkpoint8(torch.zeros(1, dtype=torch.uint8).expand(1, 1).expand(1, 1), scales, 1, "i8").desc().ld_codes == 1


@pytest.mark.gpu
def test_one_row_of_a_wider_checkpoint_is_used():
    from paper_2605_19811_gb300 import training as T
    whole = T.checkpoint8(torch.randn(3, 64, device="cuda"), "e4m3")
    for rows in (1, 2):
        part = T.Checkpoint8(whole.codes[:rows, :20], whole.scales, 20, "e4m3")
        assert torch.equal(part.unpack(), whole.unpack()[:rows, :20])
        dy = torch.randn(rows, 7, device="cuda")
        assert torch.equal(T.linear_wgrad8(dy, part, dtype=torch.float32),
                           T.linear_wgrad8(dy, T.Checkpoint8(whole.codes[:rows], whole.scales, 64, "e4m3"), dtype=torch.float32)[:, :20])


@pytest.mark.gpu
def test_a_target_beyond_the_vocabulary_and_no_weight_on_log_p():
    """logp is NaN there; the gradient of a loss without logp is not."""
    from paper_2605_19811_gb300 import training as T
    z = torch.randn(4, 900, device="cuda")
    y = torch.tensor([3, 900, 1 << 40, -1], device="cuda")
    gh, gz, gl = (torch.randn(4, device="cuda") for _ in range(3))
    o = T.token_logprob(z, y, g_entropy=gh, g_lse=gz)
    assert o.logp.isnan().tolist() == [False, True, True, False]
    want = T.token_logprob(z, None, g_entropy=gh, g_lse=gz).dlogits
    assert torch.equal(o.dlogits, want)
    assert torch.equal(T.token_logprob_grad(z, y, o.lse, o.entropy, None, gh, gz),
                       T.token_logprob_grad(z, None, o.lse, o.entropy, None, gh, gz))
    d = T.token_logprob(z, y, g_logp=gl).dlogits
    assert d.isnan().all(dim=1).tolist() == [False, True, True, False]
