"""The form that the library gives an 8-bit product, from the debug build's host-only hook (no GPU needed; 256 compute units are assumed
where there is none)."""
from tests.plan_util import debug_lib

INT8_FORMS = ("few rows", "32, shared k", "64, shared k", "64", "128", "256 x 192", "256 x 256")


def int8_form(rows, in_features, out_features):
    return INT8_FORMS[debug_lib().dit_debug_int8_form(rows, in_features, out_features)]
