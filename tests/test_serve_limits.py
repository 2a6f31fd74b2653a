"""Limits of the attention calls and how they are told, without a GPU: what is refused here is refused before any HIP call."""
import pytest

from paper_2311_10359_amd import binding
from test_serve_refusals import FAKE, append, plan, vectors

UNSUPPORTED = binding.FIKIT_UNSUPPORTED
MOST = (1 << 24) - 1          # workgroups of 256 threads of a launch, which may have fewer than 2^32 threads


def prompt(prompts, tokens, q_heads):
    return binding.load().fikit_prompt_attention(vectors(), vectors(), vectors(), q_heads, 1, 64, 0, 0.1, FAKE, prompts, tokens, FAKE + 4096, None, FAKE, None)


def test_more_workgroups_than_a_launch_takes():
    assert prompt(262144, 262144, 64) == UNSUPPORTED                  # one-token prompts: 262,144 + 2048 times 64
    assert prompt(MOST + 1, 1, 1) == UNSUPPORTED and prompt(1, MOST, 256) == UNSUPPORTED
    assert append(n_tokens=1 << 30, n_pieces=MOST + 1) == UNSUPPORTED
    assert append(n_tokens=1 << 30, n_pieces=(1 << 31) - 1) == UNSUPPORTED


def test_what_unsupported_is_called():
    """The calls that return it take different things: its text fits all of them."""
    text = binding.status_string(UNSUPPORTED)
    assert "limit" in text and "size" in text and "scenario" not in text


def apart():
    """Arguments of a plan of 4 requests and 9 tokens, each in memory of its own."""
    names = ("cached", "added", "table", "free", "lengths", "offsets", "slots", "pieces", "counts", "status", "ws")
    return {name: FAKE + 4096 * i for i, name in enumerate(names)}


@pytest.mark.parametrize("output, at", [("lengths", "cached"), ("lengths", "added"), ("offsets", "cached"), ("offsets", "added"), ("counts", "cached"),
                                        ("counts", "free"), ("slots", "added"), ("pieces", "free"), ("lengths", "offsets"), ("pieces", "slots")])
@pytest.mark.parametrize("shift", [0, 1])
def test_outputs_of_a_plan_over_what_it_reads(output, at, shift):
    """Every workgroup reads the requests while the first one writes: in place there would be a race."""
    a = apart()
    a[output] = a[at] + 16 * shift if output == "pieces" or shift == 0 else a[at] + 8
    assert plan(**a) == binding.FIKIT_INVALID_ARG


def test_a_prompts_output_over_its_inputs():
    """Rows with values that are not finite are done again, from the queries."""
    q, k, v, offsets, status = (FAKE + 4096 * i for i in range(5))
    for out in (q, k, v):
        assert binding.load().fikit_prompt_attention(vectors(q), vectors(k), vectors(v), 4, 2, 64, 0, 0.1, offsets, 2, 9, out, None, status,
                                                     None) == binding.FIKIT_INVALID_ARG


@pytest.mark.parametrize("dim", [0, 32, 80, 96, 256])
def test_no_workspace_for_head_sizes_that_are_not_taken(dim):
    assert binding.fikit_cache_attention_workspace_bytes(1, 8, 8, dim, 100000) == 0
