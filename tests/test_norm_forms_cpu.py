"""That the sizes of the GPU tests of layer norm run every kernel that there is for it. No GPU."""
from tests.linear_launches import launches
from tests.norm_forms import back_calls, norm_calls

OURS = ("norm_kernel<", "norm_wave_kernel<", "norm_long_kernel<", "back_kernel<", "back_long_kernel<", "gains_kernel<")


def test_every_kernel_is_tested(tmp_path):
    calls = [c for bf16 in (0, 1) for c in norm_calls(bf16) + back_calls(bf16)]
    out, known = launches(tmp_path, calls)
    assert all(out)
    wanted = {k for k in known if k.startswith(OURS)}
    assert len(wanted) > 200 and wanted - {n for names in out for n in names} == set()
