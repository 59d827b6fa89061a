"""What the Python classes of the learning operators refuse without a GPU."""
import pytest


@pytest.mark.parametrize("name", ["m", "v", "m_exp", "v_exp", "new_m", "new_v", "new_m_exp", "new_v_exp"])
def test_moments_are_not_replaced(name):
    """The plan holds the moments' places: another tensor in their name would be left unread."""
    import torch
    from paper_2608_16329_amd import AdamW
    opt = object.__new__(AdamW)
    with pytest.raises(AttributeError):
        setattr(opt, name, torch.zeros(4))
