"""gg_product_status without a device."""


def test_a_missing_context_is_an_argument_error():
    import __graft_entry__ as entry
    entry.build()
    from paper_2506_00486_b200 import binding
    assert binding.lib().gg_product_status(None) == 1
