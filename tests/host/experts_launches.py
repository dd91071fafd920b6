"""Calls of the experts' entry points beside a stand-in for the launch (experts_recorder.cpp): what each would launch, as JSON.

argv: the stand-in, the library, a JSON list of [function, arguments]; of the arguments "p" is a pointer on 16 bytes, "odd" one that is not, null none, a list
[n] a long long, a number with a point a float.  The stand-in is loaded first, so the library's launches go to it; no memory is touched.
"""
import ctypes
import json
import sys

recorder = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
lib = ctypes.CDLL(sys.argv[2])
recorded, name = (ctypes.c_int * 4).in_dll(recorder, "recorded"), (ctypes.c_char * 512).in_dll(recorder, "recorded_name")


def argument(v):
    if isinstance(v, list):
        return ctypes.c_longlong(v[0])
    if isinstance(v, str):
        return ctypes.c_void_p((1 << 20) + (v == "odd") * 4)
    return ctypes.c_float(v) if isinstance(v, float) else v


out = []
for function, arguments in json.loads(sys.argv[3]):
    before = recorded[0]
    rc = getattr(lib, function)(*map(argument, arguments))
    out.append(dict(rc=rc, launches=recorded[0] - before, workgroups=recorded[1], threads=recorded[2], way=recorded[3], kernel=name.value.decode()))
print(json.dumps(out))
