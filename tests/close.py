"""A comparison whose mask comes from the wanted values, never from the computed ones."""
import torch

# From here on half a step and the errors before it may round a value to binary16's infinity (its largest number is 65504).
FP16_MAY_OVERFLOW = 65000.0


def settled(got, want, bound, dtype):
    """True where got (of type dtype) is within bound of want (float64).  Not a number never is; an infinity is where binary16 has no number for the wanted
    value, and of its sign."""
    got = got.double()
    ok = torch.isfinite(got) & ((got - want).abs() <= bound)
    if dtype == "fp16":
        ok |= (want.abs() >= FP16_MAY_OVERFLOW) & torch.isinf(got) & (torch.sign(got) == torch.sign(want))
    return ok
