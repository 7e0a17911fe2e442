"""kv_write where the parts of a token change in number, by the wave of each type's own kernel."""
import pytest
import torch

from paper_2608_24658_gb300 import build
from tests.test_kv_gpu import check_write

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()
    torch.cuda.init()


# waves of 2432 (fp32, 128, halves) and 3040 warps, and what is a half or a third of them
@pytest.mark.parametrize("mode,d,kind", [("fp32", 128, (128, 1, False)), ("fp32", 128, (128, 1, True)),
                                         ("fp32", 64, (64, 1, False)), ("fp8", 128, (128, 1, False))])
@pytest.mark.parametrize("tokens", [811, 1217, 1521, 2433, 3041])
def test_tokens_around_a_wave(mode, d, kind, tokens):
    check_write(tokens, mode, 16, 4, d, tokens, kind)
