"""The experts' norm at widths that lead to each number of threads and chunks a row."""
import pytest

from test_gpu_experts import test_norm as check

pytestmark = pytest.mark.gpu


# bf16 rows of 4104 to 8192 are four chunks a thread of 256, fp32 ones four of 512
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,E,d,mode", [(50, 3, 4104, "plain"), (33, 2, 8192, "gather"),
                                        (61, 4, 6008, "ragged"), (700, 1, 5000, "shared"),
                                        (7, 300, 8184, "plain")])
def test_wide_rows(N, E, d, mode, dtype):
    check(N, E, d, mode, dtype)
