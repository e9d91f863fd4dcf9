"""The gated projection of few tokens through wide layers, where each wavefront goes through many batches of loads."""
import pytest

from test_gpu_gated import run_case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tokens,c,hidden", [
    (1, 4096, 64), (8, 4096, 40), (5, 16392, 17), (1, 1544, 515), (3, 2040, 33),          # weights in halves of rows, one token group
    (9, 5128, 24), (16, 8200, 40), (16, 1600, 131), (12, 2056, 1),                        # two
    (17, 2048, 48), (32, 4096, 48), (24, 776, 100),                                       # whole rows, two groups
    (33, 2056, 40), (64, 4104, 24), (50, 1040, 260), (64, 8192, 16)])                     # four
def test_few_tokens_through_wide_layers(tokens, c, hidden, dtype):
    run_case(tokens, c, hidden, dtype, "silu", bias=hidden % 2 == 0, seed=14)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tokens,c,hidden", [(1, 4097, 33), (16, 4095, 40), (20, 4096, 4104), (64, 2048, 5640)])
def test_few_tokens_on_the_product_for_every_size(tokens, c, hidden, dtype):
    # rows of no whole 16-byte units; more weights than few tokens are worth reading all tokens for
    run_case(tokens, c, hidden, dtype, "gelu", bias=True, seed=15)
