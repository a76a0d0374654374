"""tdk_kv_attend, many query rows: single parts of many steps, where the step kernel's page lists and registers go round several times."""
import pytest

from test_gpu_kv import FORMATS, check_attend

pytestmark = pytest.mark.gpu


@FORMATS
@pytest.mark.parametrize("T", [16, 32])
@pytest.mark.parametrize("lengths,kw", [([(2500, 40)], {}), ([(1100, 70), (0, 3), (2300, 30)], {}), ([(3900, 30)], dict(window=2600, sink=130)),
                                        ([(3900, 30)], dict(hole=[(1000, 1900)], join=True)), ([(1500, 30)], dict(hole=[(0, 60)])),
                                        ([(4000, 30)], dict(window=1500, sink=1200)), ([(64 * 17 - 30, 30)], {}), ([(64 * 16 - 30, 30)], {}),
                                        ([(64 * 33 - 30, 31)], {})])
def test_one_part_of_many_steps(fmt, T, lengths, kw):
    """Five query heads per KV head: 150 rows of a sequence and more (blocks of 128 rows in both formats); no more tokens expected than one, so a
    sequence is one part of up to 64 steps of 64 tokens."""
    check_attend(fmt, 2, 5, T, lengths, max_len=1, **kw)
