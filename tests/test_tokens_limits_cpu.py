"""Refusals at the limits of the token calls (include/az_tokens.h), before any CUDA call."""
import paper_2609_37447_b200 as az


def test_the_status_self_test_knows_two_parts():
    assert az._lib.az_selftest_tokens_timeout(2, None) == az.AZ_ERR_BAD_ARG
    assert az._lib.az_selftest_tokens_timeout(-1, None) == az.AZ_ERR_BAD_ARG
