// What the stand-ins of operator_stubs.cpp count.
#pragma once
struct OperatorStubs {
    int turned = 0, turned_back = 0, in_place = 0, joins = 0, joins_with_norm = 0, joins_back = 0, distillations = 0;
};
extern OperatorStubs operator_stubs;
