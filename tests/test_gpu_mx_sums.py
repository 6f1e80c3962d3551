"""GPU tests of how products of 4-bit operands are summed, above all where they are cut along K: sums that fp32 holds
exactly, and random ones against a bound that tells fp32 from fewer bits (the companion on the CPU checks that it does)."""
import numpy as np
import pytest

from oracle import mx as oracle

# cut along K into tiles of 32, 64 and 128 rows
CUT = [(1, 20000, 48), (20, 20000, 3000), (60, 20000, 2000), (64, 8192, 4096), (100, 9000, 70), (129, 30000, 130), (512, 40000, 512)]
WHOLE = [(16, 12000, 500), (31, 4000, 20000), (64, 4100, 4099), (300, 9000, 9000), (2300, 5000, 2300)]


@pytest.mark.gpu
@pytest.mark.parametrize("m,k,n", CUT + WHOLE, ids=str)
def test_sums_that_fp32_holds(m, k, n):
    """Positive codes of one scale: multiples of a quarter below 2^22, whatever the order."""
    import torch
    from paper_2510_08874_amd import binding
    from tests.test_gpu_mx import Form, whole
    g = torch.Generator(device="cuda").manual_seed(k)
    table = torch.from_numpy(oracle.VALUES).cuda()

    def codes(d, along, size):
        form, code = Form(d, along), torch.randint(1, 8, size, generator=g, dtype=torch.uint8, device="cuda")
        padded = torch.nn.functional.pad(code, (0, -k % 128))
        form.codes[0].copy_(padded[:, 0::2] | padded[:, 1::2] << 4)
        form.scales[0].zero_()
        form.scales[0][:, :-(-k // 32)] = 127
        return form, table[code.int()]

    (a, A), (b, B) = codes(whole(m, k), 1, (m, k)), codes(whole(k, n), 2, (n, k))
    plan = binding.Plan(whole(m, k), whole(k, n), whole(m, n), 1)
    want = A @ B.t().contiguous()
    for dtype, flags in ((torch.float32, 0), (torch.bfloat16, binding.DMM_C_BF16)):
        c = torch.zeros(m, n, dtype=dtype, device="cuda")
        plan.execute_mx(a.table(), b.table(), binding.tile_table([c], [n]), flags, torch.cuda.current_stream().cuda_stream)
        assert torch.equal(c, want.to(dtype))


@pytest.mark.gpu
@pytest.mark.parametrize("m,k,n", CUT, ids=str)
def test_random_sums(m, k, n):
    import torch
    from paper_2510_08874_amd import binding
    from tests.test_gpu_mx import made, whole
    (a, A), (b, B) = made(m, k, 1, m), made(k, n, 2, k)
    c = torch.zeros(m, n, device="cuda")
    binding.Plan(whole(m, k), whole(k, n), whole(m, n), 1).execute_mx(a.table(), b.table(), binding.tile_table([c], [n]),
                                                                     stream=torch.cuda.current_stream().cuda_stream)
    A, B, c = (x.double().cpu().numpy() for x in (A, B, c))
    assert np.linalg.norm(c - A @ B) <= oracle.sum_limit(A, B)
