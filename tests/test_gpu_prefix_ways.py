"""spec_prefix_attn's two ways, whatever the planner would choose: a launch of its own for the prefixes (few rows and many), and every
request through its whole context."""
import pytest
import torch  # noqa: F401  (its GPU runtime is loaded before the library, which the switch loads)

import test_gpu_cache_batches as batches
import test_gpu_prefix_attn as prefix

pytestmark = pytest.mark.gpu

WAYS = pytest.mark.parametrize("shared", [1, 0], ids=["shared", "whole"])


@pytest.fixture
def way(tuning, shared):
    tuning("SPEC_VERIFY_PREFIX_SHARED", shared)


@WAYS
@pytest.mark.parametrize("kind", prefix.KINDS)
@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("name,groups,Hq,Hkv,d,scale", prefix.CASES, ids=[c[0] for c in prefix.CASES])
def test_matches_the_definition(way, name, groups, Hq, Hkv, d, scale, out, kind):
    prefix.test_matches_the_definition(name, groups, Hq, Hkv, d, scale, out, kind)


@WAYS
@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("kind", prefix.KINDS)
@pytest.mark.parametrize("name,G,n,prefix_len,q_len,own,Hq,Hkv,d", batches.GROUPS, ids=[g[0] for g in batches.GROUPS])
def test_groups_that_fill_the_device(way, name, G, n, prefix_len, q_len, own, Hq, Hkv, d, kind, out):
    batches.test_groups_that_fill_the_device(name, G, n, prefix_len, q_len, own, Hq, Hkv, d, kind, out)


@WAYS
@pytest.mark.parametrize("kind", prefix.KINDS)
def test_many_groups(way, kind):
    prefix.test_many_groups(kind)


@WAYS
@pytest.mark.parametrize("kind", prefix.KINDS)
def test_a_bucket_serves_other_lengths(way, kind):
    prefix.test_a_bucket_serves_other_lengths(kind)


@WAYS
def test_what_does_not_fit_is_left_out_and_counted(way):
    prefix.test_what_does_not_fit_is_left_out_and_counted()


@WAYS
@pytest.mark.parametrize("kind", ["tiles", "tokens"])
@pytest.mark.parametrize("out", ["f32", "bf16"])
def test_infinities_and_nan_where_rows_do_not_see_them(way, kind, out):
    prefix.test_infinities_and_nan_where_rows_do_not_see_them(kind, out)


@WAYS
@pytest.mark.parametrize("kind", prefix.KINDS)
def test_replays_of_a_graph(way, kind):
    prefix.test_replays_of_a_graph(kind)


@WAYS
@pytest.mark.parametrize("kind", ["tiles", "e4m3"])
def test_two_runs_agree_to_the_bit(way, kind):
    batches.test_two_runs_agree_to_the_bit(kind)


@WAYS
def test_a_table_entry_outside_the_pool_reads_as_zeros_anywhere(way):
    batches.test_a_table_entry_outside_the_pool_reads_as_zeros_anywhere()
