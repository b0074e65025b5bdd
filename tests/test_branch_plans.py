"""What plans of matrix products say of themselves, against what the calls then do; no GPU is needed, nothing is launched."""
import pytest

import paper_2002_00552_amd as dwm

ONE = 4096  # an address no call reads
TYPES = [dwm.DWM_F16, dwm.DWM_BF16]


class Product:
    def __init__(self, M, N, K, type=dwm.DWM_BF16, flags=0, operands=None):
        self.plan = dwm.dwm_matmul_plan_create(M, N, K, type if operands is None else operands, type, dwm.DWM_F32, 0, flags)

    def __enter__(self):
        return self.plan

    def __exit__(self, *_):
        dwm.dwm_matmul_plan_destroy(self.plan)


def says(plan):
    info = dwm.dwm_matmul_plan_info(plan)
    return info.kernel, info.splits, dwm.dwm_matmul_workspace_bytes(plan)


SIZES = [(300, 300, 500), (300, 300, 501), (5, 12289, 4097), (16001, 333, 1111), (100, 200, 3000), (40, 24, 5000), (1, 4096, 4096), (1030, 1029, 1027), (512, 512, 16384), (7, 9, 0)]


@pytest.mark.parametrize("flags", range(4))
@pytest.mark.parametrize("type", TYPES)
@pytest.mark.parametrize("M, N, K", SIZES)
def test_asking_for_the_planners_parts_changes_nothing(M, N, K, type, flags):
    with Product(M, N, K, type, flags) as plan:
        was = says(plan)
        dwm.dwm_matmul_set_variant(plan, "splits", -1)
        assert says(plan) == was
        dwm.dwm_matmul_set_variant(plan, "splits", 5)
        assert says(plan)[1] == 5
        dwm.dwm_matmul_set_variant(plan, "splits", -1)
        assert says(plan) == was
        dwm.dwm_matmul_set_variant(plan, "kernel", 3)
        assert says(plan)[0] == 3
        dwm.dwm_matmul_set_variant(plan, "splits", 2)
        assert says(plan)[:2] == (3, 2)
        dwm.dwm_matmul_set_variant(plan, "splits", -1)  # of that kernel
        assert says(plan)[0] == 3
        dwm.dwm_matmul_set_variant(plan, "kernel", -1)
        assert says(plan) == was


@pytest.mark.parametrize("M, N, K", [(300, 300, 500), (300, 300, 501)])
def test_one_part_asks_for_no_copies(M, N, K):
    """Rows of odd lengths that the planner does not lay out anew stay where they lie, in however many parts."""
    with Product(M, N, K) as plan:
        assert says(plan)[2] == 0
        dwm.dwm_matmul_set_variant(plan, "splits", 1)
        assert says(plan)[1:] == (1, 0)
        dwm.dwm_matmul_set_variant(plan, "splits", 2)
        assert says(plan)[2] == 2 * M * 320 * 4  # sums of parts alone


def test_parts_where_few_rows_have_a_kernel_of_their_own():
    with Product(1, 4096, 4096) as plan:
        assert says(plan)[:2] == (5, 1)
        dwm.dwm_matmul_set_variant(plan, "splits", 3)  # by tiles
        kernel, splits, bytes_ = says(plan)
        assert 2 <= kernel <= 4 and splits == 3 and bytes_ == 3 * 4096 * 4
        dwm.dwm_matmul_set_variant(plan, "splits", 1)
        assert says(plan) == (5, 1, 0)
        dwm.dwm_matmul_set_variant(plan, "kernel", 5)
        with pytest.raises(dwm.DwmError) as e:
            dwm.dwm_matmul_set_variant(plan, "splits", 3)
        assert e.value.status == dwm.DWM_ERR_INVALID_ARG


def refused(status, f, *args):
    with pytest.raises(dwm.DwmError) as e:
        f(*args)
    assert e.value.status == status


@pytest.mark.parametrize("M, N, K", [(8, 8, (1 << 20) + 1), (1, 1, 1 << 24), (1 << 24, 8, 1 << 17), (8, 1 << 24, 1 << 17)])
def test_packed_operands_that_cannot_be_made_are_refused(M, N, K):
    assert dwm.dwm_packed_codes_bytes(M, K) == 0 or dwm.dwm_packed_codes_bytes(N, K) == 0
    refused(dwm.DWM_ERR_UNSUPPORTED, dwm.dwm_matmul_plan_create, M, N, K, dwm.DWM_PACKED, dwm.DWM_BF16, dwm.DWM_F32, 0, 0)


@pytest.mark.parametrize("M, N, K", [(8, 8, 1 << 20), (1 << 20, 16, 1 << 20), (8, 8, 0)])
def test_the_largest_packed_operands(M, N, K):
    with Product(M, N, K, operands=dwm.DWM_PACKED):
        pass


@pytest.mark.parametrize("operands", [dwm.DWM_BF16, dwm.DWM_PACKED])
def test_packed_results_that_cannot_be_sized_are_refused(operands):
    N, rows = (1 << 20) + 1, dwm.dwm_packed_t(ONE, ONE)
    with Product(4, N, 64, operands=operands) as plan:
        assert dwm.dwm_packed_codes_bytes(4, N) == 0
        f, a = (dwm.dwm_matmul_packed, rows) if operands == dwm.DWM_PACKED else (dwm.dwm_matmul, ONE)
        for packed in ((rows, None), (None, rows)):
            refused(dwm.DWM_ERR_UNSUPPORTED, f, plan, a, a, None, None, ONE, *packed)
            refused(dwm.DWM_ERR_UNSUPPORTED, f, plan, a, a, None, None, None, *packed)
