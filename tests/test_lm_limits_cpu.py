"""Sizes that the operators refuse before they touch a device."""
import ctypes


def test_gradients_of_more_tokens_than_places_are_refused():
    """Ends of chunks of the sorted list are 32-bit numbers."""
    from paper_1511_00175_amd import _fc_lm
    for tokens in ((1 << 30) + 1, (1 << 31) - 32, (1 << 31) - 1, 1 << 31):
        plan = ctypes.c_void_p()
        assert _fc_lm.lib.fc_embed_create(ctypes.byref(plan), 10, 1, tokens) == -1 and not plan.value, tokens
